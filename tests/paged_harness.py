"""References in 64 bits for the calls on a paged cache, and the errors that the calls' arithmetic allows for."""
import math

import torch

import paper_2601_07353_amd as T

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Pages:
    """A pool of more pages than are used, in random order, filled with NaN where nothing was put."""

    def __init__(self, lens, Hkv, Dh, dtype, page=16, spare=3, head_major=False, seed=0, device="cuda", room=0):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        self.page, self.B, self.Hkv, self.Dh, self.dtype = page, B, Hkv, Dh, dtype
        self.max_pages = max(1, max((n + room + page - 1) // page for n in lens))
        pages = B * self.max_pages + spare
        shape = (pages, Hkv, page, Dh) if head_major else (pages, page, Hkv, Dh)
        self.k = torch.full(shape, math.nan, dtype=dtype, device=device)
        self.v = torch.full(shape, math.nan, dtype=dtype, device=device)
        if head_major:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        order = torch.randperm(pages, generator=g)[:B * self.max_pages]
        self.table = order.view(B, self.max_pages).to(torch.int32).to(device)
        self.cache = T.PagedCache(self.k, self.v, self.table)
        self.g = torch.Generator(device=device).manual_seed(seed + 1)
        for b, n in enumerate(lens):
            self.put(b, 0, torch.randn(n, Hkv, Dh, device=device, generator=self.g), torch.randn(n, Hkv, Dh, device=device, generator=self.g))

    def at(self, b, rows):
        return self.table[b].long()[rows // self.page], rows % self.page

    def put(self, b, first, k, v):
        rows = torch.arange(first, first + k.shape[0], device=self.k.device)
        p, s = self.at(b, rows)
        self.k[p, s] = k.to(self.dtype)
        self.v[p, s] = v.to(self.dtype)

    def rows(self, b, n):
        p, s = self.at(b, torch.arange(n, device=self.k.device))
        return self.k[p, s], self.v[p, s]


def causal_or_mask(mask_bool, n, P):
    """[n][P + n] whether new token i sees row j."""
    sees = torch.ones(n, P + n, dtype=torch.bool, device="cuda")
    sees[:, P:] = torch.ones(n, n, dtype=torch.bool, device="cuda").tril() if mask_bool is None else mask_bool[:n, :n]
    return sees


def words_of(mask_bool):
    """bool [B][N][N] -> int64 [B][N][ceil(N/64)]"""
    B, N, _ = mask_bool.shape
    W = (N + 63) // 64
    bits = torch.zeros(B, N, W * 64, dtype=torch.int64, device=mask_bool.device)
    bits[:, :, :N] = mask_bool.long()
    return (bits.view(B, N, W, 64) << torch.arange(64, device=mask_bool.device)).sum(-1)


def scores_of(q, k, sees, scale, cap=0.0, slopes=None, window=0, pos_q=None, pos_k=None):
    """q [n][Hq][D], k [L][Hkv][D] -> scores [Hq][n][L] in 64 bits (-inf where not seen) and how far 32 bits may be off."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    kk = k.double().repeat_interleave(G, 1).permute(1, 2, 0).contiguous()      # [Hq][D][L]
    qq = q.double().permute(1, 0, 2).contiguous()
    x = torch.matmul(qq, kk) * scale
    # a sum of D products in 32 bits: D half steps of the sum of absolute values; a few more for scale, base 2 and differences
    off = torch.matmul(qq.abs(), kk.abs()) * scale * (D + 8) * 2.0 ** -24 + x.abs() * 2.0 ** -22
    if cap:
        x = cap * torch.tanh(x / cap)
        off = off + cap * 2.0 ** -21
    away = (pos_q[:, None] - pos_k[None]).double()
    if slopes is not None:
        bias = slopes.double()[:, None, None] * away.abs()
        x = x - bias
        off = off + bias * 2.0 ** -21
    s = sees if not window else sees & (away < window)
    return x.masked_fill(~s, -math.inf), off.masked_fill(~s, 0.0)


def attention_of(q, k, v, *how, **more):
    """(out, lse, tolerance of out, tolerance of lse), [n][Hq][...], for storage type q.dtype."""
    x, off = scores_of(q, k, *how, **more)
    G = q.shape[1] // k.shape[1]
    vv = v.double().repeat_interleave(G, 1).permute(1, 0, 2).contiguous()
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    w = torch.where(total > 0, p / total, torch.zeros_like(p))
    vv = torch.where((p > 0).any(1)[..., None], vv, torch.zeros_like(vv)) if not torch.isfinite(vv).all() else vv
    out = torch.matmul(w, vv)
    u = HALF_STEP[q.dtype]
    far = off.amax(-1, keepdim=True)
    # probabilities rounded to the storage type (relative u, or half of fp16's smallest step against a maximum of 1), scores off
    # by `far` (relative 2 * far in a weight), the result rounded once
    tol = u * out.abs() + torch.matmul(w, vv.abs()) * (u + 2 * far + 2.0 ** -18) + 2.0 ** -25 * vv.abs().sum(1)[:, None] + 2.0 ** -25
    lse = (top + torch.log(total))[..., 0]
    return out.permute(1, 0, 2), lse.T, tol.permute(1, 0, 2), (far[..., 0] + 2.0 ** -20 * (1 + lse.abs().nan_to_num(posinf=0.0))).T


def assert_close(got, want, tol, what=""):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN"
    fine = ~torch.isnan(want)
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what + ": infinities"
    fine &= ~inf
    bad = ((got - want).abs() > tol) & fine
    assert not bad.any(), "%s: %d of %d off, worst by %.3g (allowed there %.3g)" % (
        what, int(bad.sum()), bad.numel(), float((got - want).abs()[bad].max()), float(tol.expand_as(want)[bad].max()))
