"""Scores capped far above what they reach (cap * tanh(x / cap) is then close to x) and at large scores: attention and weights to the
accuracy of 32-bit scores, whatever the cap."""
import math

import pytest
import torch

import paper_2601_07353_amd as T
from tests import paged_harness, test_gpu_paged_attention
from tests.paged_harness import assert_close
from tests.test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def capped_scores(q, k, sees, scale, cap=0.0, slopes=None, window=0, pos_q=None, pos_k=None):
    """As paged_harness.scores_of, but the cap's error is relative to the score.  cap * tanh(x / cap) does not enlarge the product's error;
    x / cap, a quotient of two polynomials of three and four terms (a half step for each of their operations, two for a reciprocal) and the product
    with cap are at most 20 half steps of 2^-24."""
    x, off = paged_harness_scores(q, k, sees, scale, 0.0, None, 0, pos_q, pos_k)
    x = torch.matmul(q.double().permute(1, 0, 2), k.double().repeat_interleave(q.shape[1] // k.shape[1], 1).permute(1, 2, 0).contiguous()) * scale
    x = cap * torch.tanh(x / cap)
    off = off + x.abs() * 20 * 2.0 ** -24
    away = (pos_q[:, None] - pos_k[None]).double()
    if slopes is not None:
        bias = slopes.double()[:, None, None] * away.abs()
        x = x - bias
        off = off + (bias + x.abs()) * 2.0 ** -21
    s = sees if not window else sees & (away < window)
    return x.masked_fill(~s, -math.inf), off.masked_fill(~s, 0.0)


paged_harness_scores = paged_harness.scores_of


def close(got, want, tol, what=""):
    # exp of less than -87.3 is less than 2^-126, the least normal number in 32 bits, and becomes 0; a weight has less than 2^10 summands
    assert_close(got, want, tol + 2.0 ** -116, what)


@pytest.fixture(autouse=True)
def tight(monkeypatch):
    monkeypatch.setattr(test_gpu_paged_attention, "assert_close", close)
    monkeypatch.setattr(paged_harness, "scores_of", capped_scores)
    monkeypatch.setattr(test_gpu_paged_attention, "scores_of", capped_scores)


SHAPES = {
    "one token": dict(prefix=[1500, 63], fresh=[1, 1], Hq=8, Hkv=2, Dh=128),
    "one token, fp16, heads of 64": dict(prefix=[1500, 63], fresh=[1, 1], Hq=8, Hkv=2, Dh=64, dtype=F16),
    "some tokens, distance, window": dict(prefix=[900], fresh=[7], Hq=8, Hkv=2, Dh=128, slopes=True, window=500, dtype=F16),
    "few rows, heads of 256": dict(prefix=[300], fresh=[8], Hq=4, Hkv=2, Dh=256, dtype=F16),
    "tree": dict(prefix=[700, 20], fresh=[60, 33], Hq=8, Hkv=2, Dh=128, new="tree", dtype=F16),
    "chunk, 8 wavefronts": dict(prefix=[600], fresh=[150], Hq=16, Hkv=4, Dh=128, dtype=F16),
    "chunk, distance": dict(prefix=[600, 0], fresh=[70, 70], Hq=8, Hkv=4, Dh=64, slopes=True),
    "chunk, 8 wavefronts, distance, window": dict(prefix=[400], fresh=[180], Hq=16, Hkv=4, Dh=128, slopes=True, window=128, dtype=F16),
    "chunk, heads of 256": dict(prefix=[300], fresh=[70], Hq=4, Hkv=2, Dh=256, dtype=F16),
}


@pytest.mark.parametrize("cap,spread", [(65.0, 2.0), (1e3, 2.0), (1e3, 300.0), (1e4, 2.0), (1e6, 4.0), (1e30, 2.0)])
@pytest.mark.parametrize("name", SHAPES)
def test_large_caps(name, cap, spread):
    print("case", name, cap, spread, flush=True)
    c = Case(**SHAPES[name], cap=cap, spread=spread, seed=len(name))
    c.run()
    c.check()
    c.check_weights()


@pytest.mark.parametrize("cap", [50.0, 1e3, 1e5])
@pytest.mark.parametrize("name", SHAPES)
def test_the_weights_of_a_token_add_up_to_one(name, cap):
    """exp(score - lse) with the lse that attention gives.  Scores of both calls are off by 32-bit arithmetic (`off`), in attention up to a
    cap of 64 by 2^-22 of it besides."""
    print("case", name, cap, flush=True)
    c = Case(**SHAPES[name], cap=cap, seed=len(name))
    _, lse = c.run()
    w = torch.zeros(c.B, c.Hkv, c.most + c.N, device="cuda")
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, lse, w, **c.how)
    for b in range(c.B):
        q, k, v, sees, how = c.of(b)
        _, off = capped_scores(q, k, sees, **how)
        far = 2 * float(off.max()) + (2.0 ** -22 * cap if cap <= 64 else 0.0) + 2.0 ** -19
        total = float(w[b].double().sum())
        assert abs(total - c.fresh[b] * c.Hq) <= far * c.fresh[b] * c.Hq, (total, c.fresh[b] * c.Hq, far)
