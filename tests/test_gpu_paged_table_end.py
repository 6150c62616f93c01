"""Rows beyond the end of a page table are reported by every call that would read them: tokens that do not fit behind the prefix, a
prefix or a length that is longer than the table."""
import pytest
import torch

import paper_2601_07353_amd as T
from tests.paged_harness import Pages
from tests.test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu
BAD = T.TALON_STATUS_BAD_PAGE

SHAPES = {
    "few rows": dict(n=3, Hq=8, Hkv=2, Dh=128),
    "few rows, short": dict(n=3, Hq=8, Hkv=2, Dh=64, prefix=20),
    "many rows": dict(n=40, Hq=8, Hkv=2, Dh=128),
    "many rows, heads of 256": dict(n=40, Hq=4, Hkv=2, Dh=256),
    "many rows, 8 wavefronts": dict(n=150, Hq=8, Hkv=2, Dh=64),
    "many rows, nothing cut": dict(n=20, Hq=8, Hkv=2, Dh=64, prefix=40),
}


def past_the_end(n, Hq, Hkv, Dh, prefix=1000, B=4):
    """Sequence 0 fits to its last row, the last one too, sequence 1 lacks a row, sequence 2 begins beyond the table."""
    page = 16
    c = Case([prefix] * B, [n] * B, Hq, Hkv, Dh, page=page)
    room = c.pages.max_pages * page
    c.full = [x.clone() for x in c.run()]
    c.p[1] = room - n + 1
    c.p[2] = room + 50
    c.most = room + 100
    c.ws = torch.empty(T.talon_paged_attention_workspace_bytes(B, n, Hq, Hkv, Dh, c.most), dtype=torch.uint8, device="cuda")
    c.pages.cache.status.zero_()
    return c, room


@pytest.mark.parametrize("name", SHAPES)
def test_attention(name):
    print("case", name, flush=True)
    c, room = past_the_end(**SHAPES[name])
    c.run()
    assert c.pages.cache.status.tolist() == [0, BAD, BAD, 0]
    # (rows are cut by all lengths of the batch: low bits may differ)
    assert (c.out[0].float() - c.full[0][0].float()).abs().max() < 0.05 and (c.lse[0] - c.full[1][0]).abs().max() < 1e-4
    assert torch.isfinite(c.out[3].float()).all()


@pytest.mark.parametrize("name", SHAPES)
def test_weights(name):
    print("case", name, flush=True)
    c, room = past_the_end(**SHAPES[name])
    w = torch.full((4, c.Hkv, room + 3), 7.0, device="cuda")
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, c.full[1], w, **c.how)
    assert c.pages.cache.status.tolist() == [0, BAD, BAD, 0]
    assert (w[:, :, room:] == 7.0).all()


def test_the_last_of_many_sequences():
    for n in (1, 40):
        c, room = past_the_end(n, 4, 2, 64, B=130)
        c.p[1:129] = 30
        c.p[129] = room - n + 1
        c.run()
        assert c.pages.cache.status.tolist() == [0] * 129 + [BAD]
        c.pages.cache.status.zero_()
        w = torch.zeros(130, 2, room, device="cuda")
        T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, c.full[1], w, **c.how)
        assert c.pages.cache.status.tolist() == [0] * 129 + [BAD]


def test_a_bound_of_the_call_is_no_end_of_the_table():
    """Prefixes above max_prefix_len and more tokens than N count as these; all of that fits."""
    c = Case([100, 100], [8, 8], 4, 2, 64)
    c.p[0], c.n[1] = 2 ** 31 - 1, 2 ** 31 - 1
    c.run()
    w = torch.zeros(2, 2, 120, device="cuda")
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, c.lse, w, **c.how)
    assert not c.pages.cache.status.any()


@pytest.mark.parametrize("budget", [20, 500])
def test_eviction(budget):
    pages = Pages([90, 90, 90], 2, 64, torch.bfloat16, page=16)      # six pages: 96 rows
    w = torch.rand(3, 2, 96, device="cuda")
    kept = torch.zeros(3, 2, budget, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(3, dtype=torch.int32, device="cuda")
    length = torch.tensor([96, 97, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    T.talon_paged_evict(pages.cache, length, 200, w, budget, kept, new_len)
    assert pages.cache.status.tolist() == [0, BAD, BAD] and new_len.tolist() == [min(budget, 96)] * 3
    pages.cache.status.zero_()
    T.talon_paged_evict(pages.cache, length, 96, w, budget, kept, new_len)   # the nearest bound fits
    assert not pages.cache.status.any()
