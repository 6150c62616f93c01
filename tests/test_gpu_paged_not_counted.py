"""talon_paged_weights: a token whose lse is +inf counts nothing, whatever its query and its own row hold."""
import math

import pytest
import torch

import paper_2601_07353_amd as T
from tests.paged_harness import assert_close, scores_of
from tests.test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16

CASES = {
    "few rows": dict(prefix=[300, 40], fresh=[8, 5], Hq=8, Hkv=2, Dh=128, new="tree"),
    "few rows, causal, distance, fp16": dict(prefix=[300], fresh=[7], Hq=4, Hkv=2, Dh=64, slopes=True, dtype=F16),
    "few rows, capped, window, heads of 256": dict(prefix=[300], fresh=[8], Hq=8, Hkv=2, Dh=256, cap=20.0, window=100),
    "tree": dict(prefix=[300, 127], fresh=[64, 60], Hq=8, Hkv=2, Dh=128, new="tree"),
    "chunk of whole tiles": dict(prefix=[500], fresh=[128], Hq=8, Hkv=2, Dh=64, dtype=F16),
    "chunk, capped, distance": dict(prefix=[500], fresh=[100], Hq=8, Hkv=2, Dh=128, cap=20.0, slopes=True),
    "chunk, heads of 256": dict(prefix=[200], fresh=[70], Hq=4, Hkv=2, Dh=256, window=150),
}


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("name", CASES)
def test_not_counted(name, bad):
    print("case", name, bad, flush=True)
    c = Case(**CASES[name], seed=len(name))
    _, lse = c.run()
    lse = lse.clone()
    g = torch.Generator(device="cuda").manual_seed(9)
    out = torch.rand(c.B, c.N, device="cuda", generator=g) < 0.5
    out[:, 0], out[:, 1] = False, True
    lse[out] = math.inf
    c.q[out] = bad
    for b in range(c.B):          # rows of tokens that count nothing: every token that sees one counts nothing either
        k, v = c.pages.rows(b, c.prefix[b] + c.fresh[b])
        for i in range(c.fresh[b]):
            seen_by = c.of(b)[3][:, c.prefix[b] + i]
            if bool(out[b, i]) and bool(out[b, :c.fresh[b]][seen_by].all()):
                row = c.prefix[b] + i
                c.pages.put(b, row, k[row:row + 1] * 0 + bad, v[row:row + 1])
    W = c.most + c.N + 2
    prior = torch.rand(c.B, c.Hkv, W, device="cuda", generator=g)
    got = torch.full((c.B, c.Hkv, W), 7.0, device="cuda")
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, lse, got, decay=0.5, prior=prior, **c.how)
    want, tol = got.double() * 0 + 7.0, torch.zeros_like(got).double()
    for b in range(c.B):
        P, n = c.prefix[b], c.fresh[b]
        want[b, :, :P + n] = 0.0
        want[b, :, :P] = 0.5 * prior[b, :, :P].double()
        tol[b, :, :P + n] = 2.0 ** -22 * want[b, :, :P + n]
        q, k, v, sees, how = c.of(b)
        keep = ~out[b, :n]
        k = k.nan_to_num(nan=0.0, posinf=0.0, neginf=0.0)      # (none of the tokens that count sees such a row)
        how["pos_q"] = how["pos_q"][keep]
        x, off = scores_of(q[keep], k, sees[keep], **how)
        x = x - lse[b, :n][keep].double().T[:, :, None]
        p = torch.exp(x)
        # as in Case.check_weights: scores, their difference to lse, sums
        rel = 2 * off + 2.0 ** -21 * (1 + x.abs().nan_to_num(posinf=0.0)) + 2.0 ** -19
        want[b, :, :P + n] += p.view(c.Hkv, -1, P + n).sum(1)
        tol[b, :, :P + n] += (p * rel).view(c.Hkv, -1, P + n).sum(1)
    assert_close(got, want, tol, "weights")
