"""Scales and caps whose products and quotients no 32-bit number holds are refused (they would make scores of 0 into NaN)."""
import ctypes

import pytest

import paper_2601_07353_amd as T
from paper_2601_07353_amd.binding import _CPagedCache, _CScores, _CView

P = 0x7000000


def call(name, scale, cap):
    lib = T.load_library()
    c = ctypes.byref(_CPagedCache(2, 2, 128, 1, 64, 16, 20, 16 * 256, 256, 128, P, P + 0x1000000, P + 4, P + 8))
    v = ctypes.byref(_CView(P, 10 * 1024, 1024, 128))
    s = ctypes.byref(_CScores(None, None, None, scale, cap, 0))
    if name == "attention":   # (a workspace of nothing: what passes the scores is refused for it)
        rc = lib.talon_paged_attention(c, v, 10, 8, P, P, 300, s, v, None, P, 0, None)
    else:                     # (no lse)
        rc = lib.talon_paged_weights(c, v, 10, 8, P, P, 300, s, None, 1.0, None, P, 640, 320, None)
    return rc, lib.talon_last_error_string().decode()


@pytest.mark.parametrize("name", ["attention", "weights"])
@pytest.mark.parametrize("scale,cap", [(3e38, 0.0), (0.0, 3e38), (0.0, 1e-42), (1e30, 1e-10), (1e-10, 1e30), (0.0, 2e37)])
def test_refused(name, scale, cap):
    rc, said = call(name, scale, cap)
    assert rc == T.TALON_ERR_INVALID_ARG and "32-bit" in said, said


@pytest.mark.parametrize("name", ["attention", "weights"])
@pytest.mark.parametrize("scale,cap", [(0.0, 0.0), (2e38, 0.0), (1e-45, 0.0), (0.0, 1e-38), (0.0, 1e36), (1.0, 1e37), (1e30, 1e30), (0.125, 50.0)])
def test_not_refused(name, scale, cap):
    rc, said = call(name, scale, cap)
    assert (rc, "workspace" in said) == (T.TALON_ERR_WORKSPACE, True) if name == "attention" else "lse / weights is NULL" in said, said


def test_weights_of_more_rows_than_a_launch_covers():
    """Many queries over 2^29 rows and more: a workgroup of 512 threads for 64 of them is 2^32 threads, refused like other sizes."""
    lib = T.load_library()
    c = ctypes.byref(_CPagedCache(1, 1, 64, 1, 64, 1 << 20, 1024, 64 << 20, 64, 64, P, P + 0x1000000, P + 4, P + 8))
    v = ctypes.byref(_CView(P, 0, 64, 64))
    for most in ((1 << 29), (1 << 30)):
        rc = lib.talon_paged_weights(c, v, 33, 1, P, P, most, None, P, 1.0, None, P, 1 << 30, 1 << 30, None)
        assert rc == T.TALON_ERR_UNSUPPORTED and "rows" in lib.talon_last_error_string().decode()
