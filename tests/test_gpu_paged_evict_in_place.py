"""Eviction in place, where strides of a dimension of one entry mean nothing."""
import ctypes

import pytest
import torch

import paper_2601_07353_amd as T
from paper_2601_07353_amd.binding import _CPagedCache
from tests.paged_harness import Pages

P = 0x7000000


@pytest.mark.parametrize("B,Hkv,sb,sh,nsb,nsh,fine", [(1, 2, 640, 320, 200, 320, True), (1, 1, 640, 320, 200, 100, True), (2, 1, 640, 320, 640, 100, True),
                                                      (2, 1, 640, 320, 320, 320, False), (1, 2, 640, 320, 640, 300, False), (2, 2, 640, 320, 640, 640, False)])
def test_strides_that_count(B, Hkv, sb, sh, nsb, nsh, fine):
    """Weights in place need one set of strides, where there is more than one entry.  (No GPU: what passes is refused for a
    destination in place whose pages are of another size, before anything is launched.)"""
    lib = T.load_library()
    cache = lambda page: _CPagedCache(B, Hkv, 128, 1, 64, page, 320 // page, 16 * 256, 256, 128, P, P + 0x1000000, P + 4, P + 8)
    src, dst = cache(16), cache(8)
    rc = lib.talon_paged_evict(ctypes.byref(src), ctypes.byref(dst), P, 300, P + 128, sb, sh, 100, 0, 0, P, P + 64, P + 128, nsb, nsh, None)
    said = lib.talon_last_error_string().decode()
    assert rc == T.TALON_ERR_INVALID_ARG and ("same cache" if fine else "one set of strides") in said, said


@pytest.mark.gpu
def test_the_first_rows_of_the_weights_as_new_weights():
    pages = Pages([300], 2, 64, torch.bfloat16)
    w = torch.rand(1, 2, 300, device="cuda")
    old = w.clone()
    kept = torch.zeros(1, 2, 100, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(1, dtype=torch.int32, device="cuda")
    length = torch.tensor([300], dtype=torch.int32, device="cuda")
    T.talon_paged_evict(pages.cache, length, 300, w, 100, kept, new_len, n_recent=1, new_weights=w[:, :, :100])
    assert torch.equal(w[:, :, :100], torch.gather(old, 2, kept.long())) and torch.equal(w[:, :, 100:], old[:, :, 100:])


@pytest.mark.gpu
def test_the_same_single_page_with_another_stride():
    """A pool of one page through two handles: the same rows, so it is in place."""
    k, v = (torch.randn(1, 512, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    far = lambda x: x.as_strided(x.shape, (2 * x.stride(0), *x.stride()[1:]))
    old = [x.clone() for x in (k, v)]
    w = torch.rand(1, 2, 400, device="cuda")
    kept = torch.zeros(1, 2, 100, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(1, dtype=torch.int32, device="cuda")
    length = torch.tensor([400], dtype=torch.int32, device="cuda")
    T.talon_paged_evict(T.PagedCache(k, v, table), length, 400, w, 100, kept, new_len, dst=T.PagedCache(far(k), far(v), table))
    for x, was in zip((k, v), old):
        for h in range(2):
            assert torch.equal(x[0, :100, h], was[0, kept[0, h].long(), h])
