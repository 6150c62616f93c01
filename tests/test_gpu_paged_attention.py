"""talon_paged_attention and talon_paged_weights against references in 64 bits: lengths from none to long ones, head layouts, page sizes and
orders, masks that leave a row empty, values that are no finite numbers where nobody looks, streams, graphs and bad pages."""
import math

import pytest
import torch

import paper_2601_07353_amd as T
from tests.paged_harness import HALF_STEP, Pages, assert_close, attention_of, causal_or_mask, scores_of, words_of

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def tree_mask(B, N, g):
    """Ancestor masks and depths of random trees whose parents come before them."""
    mask = torch.zeros(B, N, N, dtype=torch.bool)
    depth = torch.zeros(B, N, dtype=torch.int32)
    for b in range(B):
        for i in range(N):
            if i:
                p = int(torch.randint(0, i, (1,), generator=g))
                mask[b, i] = mask[b, p]
                depth[b, i] = depth[b, p] + 1
            mask[b, i, i] = True
    return mask.cuda(), depth.cuda()


class Case:
    def __init__(self, prefix, fresh, Hq, Hkv, Dh, dtype=BF, page=16, new="causal", cap=0.0, slopes=False, window=0, head_major=False,
                 scale=0.0, seed=0, spread=2.0, strided=False, N=None):
        g = torch.Generator().manual_seed(seed + 17)
        self.prefix, self.fresh, self.B = prefix, fresh, len(prefix)
        self.N = N = max(fresh) if N is None else N
        N = self.N = max(1, N)
        self.Hq, self.Hkv, self.Dh, self.dtype = Hq, Hkv, Dh, dtype
        self.pages = Pages([p + n for p, n in zip(prefix, fresh)], Hkv, Dh, dtype, page, head_major=head_major, seed=seed)
        gg = torch.Generator(device="cuda").manual_seed(seed + 5)
        x = (torch.randn(self.B, N, Hq + 2, Dh, device="cuda", generator=gg) * spread).to(dtype)
        self.q = x[:, :, 1:1 + Hq] if strided else x[:, :, :Hq].contiguous()
        self.mask = self.offset = None
        if new == "tree":
            self.mask, self.offset = tree_mask(self.B, N, g)
        elif new == "random":      # any pattern, some rows without a bit
            self.mask = torch.rand(self.B, N, N, generator=g).cuda() < 0.4
            self.mask[:, ::3] = False
        elif new == "offsets":     # causal, several tokens at one place
            self.offset = (torch.arange(N) // 3).expand(self.B, N).to(torch.int32).contiguous().cuda()
        self.slopes = (2.0 ** -(1 + 6 * torch.rand(Hq, generator=g))).cuda() if slopes else None
        self.cap, self.window, self.scale = cap, window, scale or 1 / math.sqrt(Dh)
        self.n = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        self.p = torch.tensor(prefix, dtype=torch.int32, device="cuda")
        self.most = max(prefix)
        self.how = dict(mask=None if self.mask is None else words_of(self.mask), offset=self.offset, scale=scale, softcap=cap,
                        slopes=self.slopes, window=window)
        nb = T.talon_paged_attention_workspace_bytes(self.B, N, Hq, Hkv, Dh, self.most)
        self.ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        self.out = torch.full((self.B, N, Hq, Dh), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((self.B, N, Hq), 7.0, device="cuda")

    def run(self, **kw):
        T.talon_paged_attention(self.pages.cache, self.q, self.n, self.p, self.most, self.out, self.lse, self.ws, **self.how, **kw)
        return self.out, self.lse

    def positions(self, b):
        P, n = self.prefix[b], self.fresh[b]
        off = torch.arange(n, device="cuda") if self.offset is None else self.offset[b, :n].long()
        return P + off, torch.cat([torch.arange(P, device="cuda"), P + off])

    def of(self, b):
        P, n = self.prefix[b], self.fresh[b]
        k, v = self.pages.rows(b, P + n)
        pq, pk = self.positions(b)
        sees = causal_or_mask(None if self.mask is None else self.mask[b], n, P)
        return self.q[b, :n], k, v, sees, dict(scale=self.scale, cap=self.cap, slopes=self.slopes, window=self.window, pos_q=pq, pos_k=pk)

    def check(self):
        torch.cuda.synchronize()
        for b in range(self.B):
            n = self.fresh[b]
            assert (self.out[b, n:] == 7.0).all() and (self.lse[b, n:] == 7.0).all(), "rows behind the last token were written"
            if n == 0:
                continue
            q, k, v, sees, how = self.of(b)
            out, lse, tol, tol_lse = attention_of(q, k, v, sees, **how)
            assert_close(self.out[b, :n], out, tol, "out of sequence %d" % b)
            assert_close(self.lse[b, :n], lse, tol_lse, "lse of sequence %d" % b)
        assert not self.pages.cache.status.any()

    def check_weights(self, decay=0.75):
        W = self.most + self.N + 3
        prior = torch.rand(self.B, self.Hkv, W, device="cuda")
        got = torch.full((self.B, self.Hkv, W), 7.0, device="cuda")
        lse = torch.zeros(self.B, self.N, self.Hq, device="cuda")
        want, tols = got.double(), torch.zeros_like(got).double()
        for b in range(self.B):
            P, n = self.prefix[b], self.fresh[b]
            want[b, :, :P + n] = 0.0
            want[b, :, :P] = decay * prior[b, :, :P].double()
            tols[b, :, :P + n] = 2.0 ** -22 * want[b, :, :P + n]
            if n:
                q, k, v, sees, how = self.of(b)
                x, off = scores_of(q, k, sees, **how)
                lse[b, :n] = torch.logsumexp(x, -1).T.float()
                p = torch.exp(x - lse[b, :n].double().T[:, :, None]).nan_to_num(nan=0.0)
                rel = 2 * off + 2.0 ** -21 * (1 + x.abs().nan_to_num(posinf=0.0)) + 2.0 ** -19   # scores, their difference to lse, sums
                want[b, :, :P + n] += p.view(self.Hkv, -1, P + n).sum(1)
                tols[b, :, :P + n] += (p * rel).view(self.Hkv, -1, P + n).sum(1)
        T.talon_paged_weights(self.pages.cache, self.q, self.n, self.p, self.most, lse, got, decay=decay, prior=prior, **self.how)
        assert_close(got, want, tols, "weights")


CASES = {
    "one token, one row": dict(prefix=[0], fresh=[1], Hq=4, Hkv=4, Dh=64),
    "one token": dict(prefix=[2048], fresh=[1], Hq=32, Hkv=8, Dh=128),
    "one token, a group of 5": dict(prefix=[1000, 0, 37], fresh=[1, 1, 1], Hq=20, Hkv=4, Dh=128, dtype=F16, page=32),
    "one token, one KV head for 48": dict(prefix=[777, 64], fresh=[1, 1], Hq=48, Hkv=1, Dh=64, page=1),
    "one token, one KV head for 128": dict(prefix=[500], fresh=[3], Hq=128, Hkv=1, Dh=64, dtype=F16, page=128),
    "one token, heads of 256": dict(prefix=[1500, 63, 64], fresh=[1, 1, 1], Hq=8, Hkv=4, Dh=256, page=64),
    "seventy sequences": dict(prefix=[(37 * i * i) % 1900 for i in range(70)], fresh=[1] * 70, Hq=8, Hkv=2, Dh=128, slopes=True),
    "some without new tokens": dict(prefix=[300, 500, 0, 900, 20], fresh=[0, 5, 0, 17, 0], Hq=6, Hkv=2, Dh=64, dtype=F16, page=8),
    "none has new tokens": dict(prefix=[300, 500], fresh=[0, 0], Hq=4, Hkv=2, Dh=64, N=4),
    "short, not cut": dict(prefix=[0, 100, 190], fresh=[60, 7, 60], Hq=12, Hkv=4, Dh=128),
    "chunk from the start": dict(prefix=[0, 0], fresh=[513, 200], Hq=8, Hkv=2, Dh=128, page=64),
    "chunk behind a prefix, 8 wavefronts": dict(prefix=[1000, 333], fresh=[300, 257], Hq=16, Hkv=4, Dh=128),
    "chunk, fp16, head-major": dict(prefix=[700], fresh=[190], Hq=8, Hkv=8, Dh=128, dtype=F16, page=32, head_major=True),
    "chunk, heads of 256": dict(prefix=[130, 5], fresh=[70, 33], Hq=4, Hkv=2, Dh=256, head_major=True),
    "chunk, heads of 64, 8 wavefronts": dict(prefix=[400], fresh=[180], Hq=9, Hkv=3, Dh=64, strided=True),
    "capped": dict(prefix=[900, 30], fresh=[40, 40], Hq=8, Hkv=2, Dh=128, cap=5.0),
    "capped hard, 8 wavefronts": dict(prefix=[600], fresh=[150], Hq=16, Hkv=4, Dh=128, cap=0.5, dtype=F16),
    "distance": dict(prefix=[800, 77], fresh=[50, 31], Hq=8, Hkv=4, Dh=64, slopes=True),
    "distance, 8 wavefronts, offsets": dict(prefix=[500], fresh=[140], Hq=16, Hkv=4, Dh=128, slopes=True, new="offsets"),
    "window of one": dict(prefix=[300, 0], fresh=[20, 20], Hq=4, Hkv=2, Dh=64, window=1),
    "window of 100": dict(prefix=[1000, 50, 0], fresh=[130, 130, 130], Hq=8, Hkv=2, Dh=128, window=100),
    "window, one token": dict(prefix=[5000, 63, 64, 65], fresh=[1, 1, 1, 1], Hq=8, Hkv=2, Dh=128, window=64),
    "window, all of it": dict(prefix=[700], fresh=[150], Hq=16, Hkv=4, Dh=128, window=150, cap=20.0, slopes=True, dtype=F16),
    "window wider than the rows": dict(prefix=[200], fresh=[10], Hq=4, Hkv=4, Dh=64, window=2 ** 31 - 1),
    "tree": dict(prefix=[2000, 100, 1], fresh=[60, 64, 33], Hq=32, Hkv=8, Dh=128, new="tree"),
    "tree, 8 wavefronts, window, distance": dict(prefix=[1000, 200], fresh=[130, 129], Hq=16, Hkv=4, Dh=128, new="tree", slopes=True, window=90),
    "tree, capped, heads of 256": dict(prefix=[400], fresh=[100], Hq=4, Hkv=2, Dh=256, new="tree", cap=30.0, window=37),
    "any mask": dict(prefix=[65, 0, 127], fresh=[129, 70, 200], Hq=4, Hkv=2, Dh=64, new="random"),
    "any mask, window": dict(prefix=[65, 0], fresh=[129, 70], Hq=8, Hkv=4, Dh=128, new="random", window=50, dtype=F16),
    "a large scale": dict(prefix=[300], fresh=[9], Hq=4, Hkv=2, Dh=64, scale=2.0),
    "long": dict(prefix=[20011, 40000], fresh=[2, 1], Hq=8, Hkv=2, Dh=64, page=256, spread=4.0),
}


@pytest.mark.parametrize("name", CASES)
def test_attention(name):
    print("case", name, flush=True)
    c = Case(**CASES[name], seed=len(name))
    c.run()
    c.check()


@pytest.mark.parametrize("name", CASES)
def test_weights(name):
    print("case", name, flush=True)
    Case(**CASES[name], seed=len(name)).check_weights()


def test_a_call_repeats_itself_and_needs_no_lse():
    c = Case([900, 33], [70, 70], 16, 4, 128, new="tree")
    out, lse = (x.clone() for x in c.run())
    for _ in range(3):
        c.out.fill_(7.0)
        T.talon_paged_attention(c.pages.cache, c.q, c.n, c.p, c.most, c.out, None, c.ws, **c.how)
        assert torch.equal(c.out.view(torch.int16), out.view(torch.int16))


def test_what_a_token_does_not_see_has_no_effect():
    """NaN and infinities in masked rows of K and V, in queries and rows beyond the lengths (which the pool holds anyway)."""
    for bad in (math.nan, math.inf, -math.inf):
        for new, window in (("causal", 0), ("random", 0), ("causal", 40)):
            c = Case([130, 64], [100, 100], 8, 2, 128, new=new, window=window, seed=3)
            i, j = 20, 60                                    # token j's rows, seen by few
            sees = [causal_or_mask(None if c.mask is None else c.mask[b], 100, c.prefix[b]) for b in range(2)]
            for b in range(2):
                if window:
                    pq, pk = c.positions(b)
                    sees[b] &= (pq[:, None] - pk[None]) < window
            want = [x.clone() for x in c.run()]
            for b in range(2):
                row = c.prefix[b] + j
                k, v = c.pages.rows(b, row + 1)
                c.pages.put(b, row, k[row:] * 0 + bad, v[row:] * 0 + bad)
            early = 5                                        # a row that the window hides from later tokens
            if window:
                for b in range(2):
                    k, v = c.pages.rows(b, early + 1)
                    c.pages.put(b, early, k[early:] * 0 + bad, v[early:] * 0 + bad)
            c.run()
            for b in range(2):
                blind = ~sees[b][:, c.prefix[b] + j]
                if window:
                    blind &= ~sees[b][:, early]
                assert 0 < int(blind.sum()) < 100
                assert torch.equal(c.out[b][blind], want[0][b][blind]) and torch.equal(c.lse[b][blind], want[1][b][blind])
                if bad != -math.inf:                          # (a key of -inf times a query of either sign: not always NaN)
                    assert not torch.isfinite(c.out[b][~blind].float()).all(-1).any()


def test_a_value_that_is_not_finite_reaches_who_sees_it():
    for Dh, dtype in ((64, F16), (128, BF), (256, BF)):
        c = Case([70], [40], 4, 2, Dh, dtype, seed=1)
        k, v = c.pages.rows(0, 91)
        bad = v[90:].clone()
        bad[0, 0, 7] = math.inf                              # token 20, KV head 0
        c.pages.put(0, 90, k[90:], bad)
        c.run()
        fine = torch.isfinite(c.out[0].float()).all(-1)      # [token][head]
        assert fine[:20].all() and fine[:, 2:].all() and not fine[20:, :2].any()
        assert torch.isfinite(c.lse[0][:20]).all()


def test_views_of_a_wider_tensor_and_streams():
    c = Case([500, 20], [30, 9], 8, 4, 64, strided=True, head_major=True)
    wide = torch.full((2, 30, 10, 3 * 64), 7.0, dtype=BF, device="cuda")
    c.out = wide[:, :, 1:9, 64:128]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    c.check()
    assert (wide[:, :, 0] == 7.0).all() and (wide[:, :, 9] == 7.0).all() and (wide[..., :64] == 7.0).all() and (wide[..., 128:] == 7.0).all()


def test_captured_and_replayed_between_other_work():
    c = Case([900, 100, 5], [64, 64, 64], 16, 4, 128, new="tree", cap=20.0)
    W = c.most + 64
    weights = torch.zeros(3, 4, W, device="cuda")
    c.run()
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, c.lse, weights, **c.how)
    want = [x.clone() for x in (c.out, c.lse, weights)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
        T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, c.lse, weights, **c.how)
    for _ in range(3):
        for x in (c.out, c.lse, weights):
            x.fill_(7.0 if x is not weights else 0.0)
        graph.replay()
        (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
        for x, y in zip((c.out, c.lse, weights), want):
            assert torch.equal(x, y)
    c.n.copy_(torch.tensor([1, 40, 0], dtype=torch.int32))   # lengths are read by the replay
    c.p.copy_(torch.tensor([200, 37, 5], dtype=torch.int32))
    c.fresh, c.prefix = [1, 40, 0], [200, 37, 5]
    c.out.fill_(7.0)
    c.lse.fill_(7.0)
    graph.replay()
    c.check()


@pytest.mark.parametrize("entry", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_a_page_outside_the_pool_is_reported(entry):
    c = Case([200, 200, 200], [3, 3, 3], 8, 2, 128)
    want = c.run()[0].clone()
    c.pages.table[1, 7] = entry
    lse = c.lse.clone()
    weights = torch.zeros(3, 2, 203, device="cuda")
    c.run()
    assert c.pages.cache.status.tolist() == [0, T.TALON_STATUS_BAD_PAGE, 0]
    assert torch.equal(c.out[0], want[0]) and torch.equal(c.out[2], want[2])
    c.pages.cache.status.zero_()
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, lse, weights, **c.how)
    assert c.pages.cache.status.tolist() == [0, T.TALON_STATUS_BAD_PAGE, 0]
    # entries behind a sequence's last row are not looked at
    c = Case([200, 20], [3, 3], 8, 2, 128)
    c.pages.table[1, 2:] = entry
    c.run()
    c.check()


def test_lengths_outside_their_bounds_are_the_nearest_bound():
    c = Case([100, 64], [8, 8], 4, 2, 64)
    want = [x.clone() for x in c.run()]
    c.n.copy_(torch.tensor([10 ** 9, 8], dtype=torch.int32))
    c.p.copy_(torch.tensor([2 ** 31 - 1, 64], dtype=torch.int32))
    c.run()
    assert torch.equal(c.out, want[0])
    c.n.copy_(torch.tensor([-5, 8], dtype=torch.int32))
    c.p.copy_(torch.tensor([-1, 64], dtype=torch.int32))
    c.out.fill_(7.0)
    c.run()
    assert (c.out[0] == 7.0).all() and torch.equal(c.out[1], want[0][1])


def test_a_pool_beyond_32_bit_offsets():
    """5 GiB per tensor, the rows on its last pages."""
    Hkv, Dh, page = 8, 128, 64
    pages = (5 << 30) // (page * Hkv * Dh * 2)
    k = torch.empty(pages, page, Hkv, Dh, dtype=BF, device="cuda")
    v = torch.empty(pages, page, Hkv, Dh, dtype=BF, device="cuda")
    L = 500
    table = (pages - 1 - torch.arange(8, device="cuda") * 3).to(torch.int32).view(1, 8)
    cache = T.PagedCache(k, v, table)
    c = Case([L], [4], 16, Hkv, Dh)
    c.pages.k, c.pages.v, c.pages.table, c.pages.cache, c.pages.page = k, v, table, cache, page
    c.pages.put(0, 0, torch.randn(L + 4, Hkv, Dh, device="cuda"), torch.randn(L + 4, Hkv, Dh, device="cuda"))
    c.run()
    c.check()
    c.check_weights()


def test_a_token_that_was_not_accepted_counts_nothing():
    c = Case([300], [20], 8, 2, 64, new="tree")
    _, lse = c.run()
    keep = torch.rand(1, 20, 1, device="cuda") < 0.5
    keep[0, 0] = True
    a, b = torch.zeros(1, 2, 320, device="cuda"), torch.zeros(1, 2, 320, device="cuda")
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, torch.where(keep, lse, torch.full_like(lse, math.inf)), a, **c.how)
    total = a.sum().item()
    assert abs(total - 8 * int(keep.sum())) < 1e-3 * total    # every row that counts gives every head a weight of one
    T.talon_paged_weights(c.pages.cache, c.q, c.n, c.p, c.most, torch.where(keep, lse, torch.full_like(lse, math.inf)), a, decay=-1.0, prior=a, **c.how)
    assert a[..., :300].abs().max() < 1e-5


def test_the_dense_call_agrees():
    """The same tree over the same rows through talon_tree_attention."""
    c = Case([1000], [64], 32, 8, 128, new="tree")
    c.run()
    k, v = c.pages.rows(0, 1064)
    out = torch.zeros(1, 64, 32, 128, dtype=BF, device="cuda")
    lse = torch.zeros(1, 64, 32, device="cuda")
    ws = torch.empty(T.talon_tree_attention_workspace_bytes(1, 64, 32, 8, 128, 1000), dtype=torch.uint8, device="cuda")
    T.talon_tree_attention(c.q, k[None, :1000], v[None, :1000], k[None, 1000:].contiguous(), v[None, 1000:].contiguous(), c.how["mask"], c.n, c.p,
                           1000, out, lse, ws)
    assert (lse - c.lse).abs().max() < 1e-4
    big = v.float().abs().max().item()
    assert (out.float() - c.out.float()).abs().max() < 4 * HALF_STEP[BF] * big   # two roundings of each, at most, of a mean of values
