"""talon_rotary_store, talon_paged_evict and talon_paged_compact: moves of rows bit for bit, rotations against 64 bits; and the calls
on a paged cache together, as a decoding step makes them."""
import math

import numpy as np
import pytest
import torch

import paper_2601_07353_amd as T
from tests.paged_harness import HALF_STEP, Pages, assert_close, attention_of

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def bits(x):
    return x.view(torch.int16)


# ---------------------------------------------------------------------------------- rotary store
STORES = {
    "one token": dict(prefix=[2048], fresh=[1], Hq=32, Hkv=8, Dh=128),
    "nothing cached": dict(prefix=[0, 0], fresh=[3, 0], Hq=4, Hkv=4, Dh=64, dtype=F16),
    "a chunk across pages": dict(prefix=[13, 100], fresh=[77, 50], Hq=8, Hkv=2, Dh=128, page=8),
    "interleaved": dict(prefix=[13, 100], fresh=[40, 50], Hq=6, Hkv=3, Dh=64, interleaved=True, dtype=F16),
    "three axes": dict(prefix=[13, 100], fresh=[40, 50], Hq=6, Hkv=3, Dh=128, axes=3),
    "four axes, interleaved, fused tensor": dict(prefix=[5], fresh=[90], Hq=6, Hkv=2, Dh=128, axes=4, interleaved=True, fused=True, head_major=True),
    "some of the head": dict(prefix=[7, 9], fresh=[20, 33], Hq=4, Hkv=2, Dh=128, pairs=32),
    "some of the head, pairs no multiple of eight": dict(prefix=[7, 9], fresh=[20, 33], Hq=4, Hkv=2, Dh=96, pairs=13),
    "the same, interleaved": dict(prefix=[7, 9], fresh=[20, 33], Hq=4, Hkv=2, Dh=80, pairs=9, interleaved=True, dtype=F16),
    "one pair": dict(prefix=[7], fresh=[20], Hq=2, Hkv=1, Dh=8, pairs=1),
    "no pairs": dict(prefix=[7, 9], fresh=[20, 33], Hq=4, Hkv=2, Dh=64, pairs=0),
    "a head of 8": dict(prefix=[7], fresh=[20], Hq=4, Hkv=2, Dh=8, page=1),
    "heads of 256, in place": dict(prefix=[70, 3], fresh=[21, 22], Hq=8, Hkv=4, Dh=256, in_place=True),
    "in place, odd pairs": dict(prefix=[70], fresh=[21], Hq=8, Hkv=4, Dh=64, pairs=11, in_place=True),
    "far positions": dict(prefix=[70], fresh=[21], Hq=4, Hkv=4, Dh=128, far=2 ** 30, dtype=F16),
    "many tokens": dict(prefix=[100, 7, 0], fresh=[1500, 900, 1], Hq=4, Hkv=2, Dh=128, axes=2, page=64),
    "many tokens, odd": dict(prefix=[3], fresh=[2051], Hq=3, Hkv=1, Dh=72, fused=True),
}


@pytest.mark.parametrize("name", STORES)
def test_rotary_store(name):
    print("case", name, flush=True)
    store_case(**STORES[name])


def store_case(prefix, fresh, Hq, Hkv, Dh, dtype=BF, page=16, axes=1, interleaved=False, pairs=None, fused=False, in_place=False, far=0,
               head_major=False):
    B, N = len(prefix), max(fresh)
    pages = Pages(prefix, Hkv, Dh, dtype, page, head_major=head_major, room=N, seed=N)
    g = torch.Generator(device="cuda").manual_seed(Dh + N)
    x = torch.randn(B, N, Hq + 2 * Hkv, Dh, device="cuda", generator=g).to(dtype)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q_in = q.clone()
    out = q if in_place else torch.full((B, N, Hq, Dh), 7.0, dtype=dtype, device="cuda")
    pairs = Dh // 2 if pairs is None else pairs
    freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(1, pairs))).float().cuda()
    pos = torch.randint(0, 5000, (axes, B, N), device="cuda", generator=g, dtype=torch.int32) + (far if far else 0)
    axis = torch.randint(0, axes, (pairs,), device="cuda", generator=g, dtype=torch.int32) if axes > 1 else None
    base = torch.randint(0, 100, (B,), device="cuda", generator=g, dtype=torch.int32) + (far - 200 if far else 0)
    old_k, old_v = pages.k.clone(), pages.v.clone()
    n, p = torch.tensor(fresh, dtype=torch.int32, device="cuda"), torch.tensor(prefix, dtype=torch.int32, device="cuda")
    T.talon_rotary_store(pages.cache, q, k, v, out, n, p, pos, freq if pairs else None, pos_base=base, pair_axis=axis, interleaved=interleaved)
    torch.cuda.synchronize()
    u = HALF_STEP[dtype]
    one = torch.arange(pairs, device="cuda")
    one, two = (2 * one, 2 * one + 1) if interleaved else (one, one + pairs)
    for b in range(B):
        m = fresh[b]
        at = base[b].double() + pos[:, b, :m].double()
        angle = (at[axis.long()].T if axis is not None else at[0][:, None]) * freq.double()
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

        def turned(y):
            y = y[b, :m].double()
            z, tol = y.clone(), torch.zeros_like(y)
            a1, a2 = y[..., one], y[..., two]
            z[..., one], z[..., two] = a1 * c - a2 * s, a2 * c + a1 * s
            # sine and cosine good to 2^-21 (argument and value in 32 bits), two products and a sum, one rounding
            near = (a1.abs() + a2.abs()) * (2.0 ** -21 + 2.0 ** -22)
            tol[..., one], tol[..., two] = near, near
            return z, tol + z.abs() * u * (tol > 0) * (1 + 2.0 ** -12) + 2.0 ** -25 * (tol > 0)

        z, tol = turned(q_in)
        assert_close(out[b, :m], z, tol, "q")
        assert torch.equal(bits(out[b, m:]), bits(q_in[b, m:] if in_place else torch.full_like(out[b, m:], 7.0)))
        z, tol = turned(k)
        pg, sl = pages.at(b, torch.arange(prefix[b], prefix[b] + m, device="cuda"))
        assert_close(pages.k[pg, sl], z, tol, "k")
        assert torch.equal(bits(pages.v[pg, sl]), bits(v[b, :m]))
        old_k[pg, sl], old_v[pg, sl] = pages.k[pg, sl], pages.v[pg, sl]
    assert torch.equal(bits(pages.k), bits(old_k)) and torch.equal(bits(pages.v), bits(old_v))   # nothing else was written
    assert not pages.cache.status.any()


def test_store_rows_without_a_place_are_not_written_and_reported():
    pages = Pages([30, 30, 30], 2, 64, BF, page=16)           # two pages each: 32 rows
    x = torch.randn(3, 5, 2, 64, device="cuda").to(BF)
    out = torch.zeros_like(x)
    freq = torch.ones(32, device="cuda")
    pos = torch.zeros(1, 3, 5, dtype=torch.int32, device="cuda")
    n = torch.tensor([2, 5, 2], dtype=torch.int32, device="cuda")
    p = torch.tensor([30, 30, 30], dtype=torch.int32, device="cuda")
    pages.table[2, 1] = pages.k.shape[0]
    old = pages.k.clone()
    T.talon_rotary_store(pages.cache, x, x, x, out, n, p, pos, freq)
    assert pages.cache.status.tolist() == [0, T.TALON_STATUS_BAD_PAGE, T.TALON_STATUS_BAD_PAGE]
    for b in range(2):
        pg, sl = pages.at(b, torch.arange(30, 32, device="cuda"))
        assert torch.equal(pages.k[pg, sl], x[b, :2])         # position 0 turns nothing
        old[pg, sl] = x[b, :2]
    assert torch.equal(bits(pages.k), bits(old))


# ---------------------------------------------------------------------------------- eviction
def evict_reference(w, n, budget, sink, recent):
    """Rows that stay, ascending (numpy)."""
    if n <= budget:
        return np.arange(n)
    w = w[:n].astype(np.float64)
    assert not np.isnan(w).any()
    forced = (np.arange(n) < sink) | (np.arange(n) >= n - recent)
    order = np.lexsort((np.arange(n), -w))                    # largest weight first, then the lowest row
    order = [r for r in order if not forced[r]][:budget - sink - recent]
    return np.sort(np.concatenate([np.nonzero(forced)[0], np.array(order, dtype=np.int64)]))


EVICTIONS = {
    "ordinary": dict(lens=[500, 300, 64], budget=100, sink=4, recent=16, Hkv=2, Dh=64),
    "in order of weight alone": dict(lens=[1000], budget=250, Hkv=4, Dh=128, dtype=F16),
    "one row stays": dict(lens=[100, 1, 0], budget=1, Hkv=2, Dh=64),
    "first and last alone": dict(lens=[200, 50], budget=20, sink=5, recent=15, Hkv=2, Dh=64),
    "all but one": dict(lens=[513], budget=512, sink=1, recent=1, Hkv=1, Dh=256),
    "shorter sequences": dict(lens=[100, 99, 101], budget=100, Hkv=2, Dh=64),
    "all weights alike": dict(lens=[3000], budget=700, sink=3, recent=7, kind="zero", Hkv=2, Dh=64),
    "few values": dict(lens=[3000, 2999], budget=1111, kind="few", Hkv=2, Dh=64, page=64),
    "not numbers, infinities, zeros of both signs, negative": dict(lens=[2000], budget=1500, kind="odd", Hkv=3, Dh=64),
    "more than a workgroup holds": dict(lens=[40000, 17000, 16385], budget=9000, sink=4, recent=64, Hkv=2, Dh=64, page=64, kind="few"),
    "more than a workgroup holds, spread": dict(lens=[33000], budget=16500, sink=4, recent=64, Hkv=1, Dh=64, page=256),
    "to other pages": dict(lens=[500, 300, 64, 0], budget=100, sink=4, recent=16, Hkv=2, Dh=64, apart=True),
    "to other pages, long, other sizes": dict(lens=[5000, 100], budget=2000, Hkv=2, Dh=128, page=16, apart=True, page2=64, head_major=True),
    "a head of 72": dict(lens=[700], budget=333, Hkv=2, Dh=72),
    "many": dict(lens=[1200 - 7 * i for i in range(33)], budget=600, sink=2, recent=2, Hkv=4, Dh=64),
}


@pytest.mark.parametrize("place", ["new weights", "weights in place", "no weights"])
@pytest.mark.parametrize("name", EVICTIONS)
def test_evict(name, place):
    print("case", name, place, flush=True)
    evict_case(place=place, **EVICTIONS[name])


def evict_case(lens, budget, Hkv, Dh, sink=0, recent=0, dtype=BF, page=16, kind="spread", apart=False, page2=None, head_major=False, place="new weights"):
    B, L = len(lens), max(lens)
    pages = Pages(lens, Hkv, Dh, dtype, page, head_major=head_major, seed=L)
    rng = np.random.default_rng(L + budget)
    w = np.exp(2.0 * rng.standard_normal((B, Hkv, L + 5))).astype(np.float32)
    if kind == "zero":
        w[:] = 0.0
    elif kind == "few":
        w = rng.integers(0, 4, w.shape).astype(np.float32) * np.float32(0.5)
    elif kind == "odd":
        w[rng.random(w.shape) < 0.2] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = -np.inf
        w[rng.random(w.shape) < 0.2] = -0.0
        w[rng.random(w.shape) < 0.2] = 0.0
        w[rng.random(w.shape) < 0.1] *= -1
    weights = torch.from_numpy(w).cuda()
    dst = None
    to = pages
    if apart:
        to = Pages([min(budget, L)] * B, Hkv, Dh, dtype, page2 or page, seed=1)
        dst = to.cache
    kept = torch.full((B, Hkv, budget), -7, dtype=torch.int32, device="cuda")
    new_len = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    old = [pages.rows(b, n) for b, n in enumerate(lens)]
    old_pools = [pages.k.clone(), pages.v.clone()]
    new_w = torch.full((B, Hkv, L + 1), 7.0, device="cuda") if place == "new weights" else (weights if place == "weights in place" else None)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    T.talon_paged_evict(pages.cache, length, L, weights, budget, kept, new_len, n_sink=sink, n_recent=recent, dst=dst, new_weights=new_w)
    torch.cuda.synchronize()
    assert new_len.tolist() == [min(n, budget) for n in lens]
    got = kept.cpu().numpy()
    for b, n in enumerate(lens):
        m = min(n, budget)
        k, v = to.rows(b, m)
        for h in range(Hkv):
            want = evict_reference(order_of(w[b, h]), n, budget, sink, recent)
            assert (got[b, h, :m] == want).all() and (got[b, h, m:] == -1).all()
            rows = torch.from_numpy(want).cuda()
            assert torch.equal(bits(k[:, h]), bits(old[b][0][rows, h])) and torch.equal(bits(v[:, h]), bits(old[b][1][rows, h]))
            if new_w is not None:
                np.testing.assert_array_equal(new_w[b, h, :m].cpu().numpy(), w[b, h, want])
    if apart:
        assert torch.equal(bits(pages.k), bits(old_pools[0])) and torch.equal(bits(pages.v), bits(old_pools[1]))
    if place == "new weights":
        assert (new_w[:, :, min(budget, L):] == 7.0).all()
    assert not pages.cache.status.any() and not to.cache.status.any()


def order_of(w):
    """Numbers in the order of the weights, what is no number least of all."""
    order = np.unique(np.where(np.isnan(w), 0.0, w + 0.0))
    return np.where(np.isnan(w), -1.0, np.searchsorted(order, np.where(np.isnan(w), 0.0, w + 0.0)).astype(np.float64))


def test_evict_reports_pages_outside_the_pool():
    pages = Pages([300, 300], 2, 64, BF)
    w = torch.rand(2, 2, 300, device="cuda")
    pages.table[1, 3] = -1
    kept = torch.zeros(2, 2, 100, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    T.talon_paged_evict(pages.cache, torch.tensor([300, 300], dtype=torch.int32, device="cuda"), 300, w, 100, kept, new_len, n_recent=1)
    assert pages.cache.status.tolist() == [0, T.TALON_STATUS_BAD_PAGE] and new_len.tolist() == [100, 100]


def test_evict_again_and_again_in_a_graph():
    """In place, replayed on what the replay before left (in the same places: lengths stay the longer ones)."""
    pages = Pages([900], 2, 64, BF, page=32)
    w = torch.rand(1, 2, 900, device="cuda")
    kept = torch.zeros(1, 2, 500, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(1, dtype=torch.int32, device="cuda")
    length = torch.tensor([900], dtype=torch.int32, device="cuda")
    call = lambda: T.talon_paged_evict(pages.cache, length, 900, w, 500, kept, new_len, n_sink=2, n_recent=3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        w.copy_(torch.rand(1, 2, 900, device="cuda"))
        old = pages.rows(0, 900)
        graph.replay()
        torch.cuda.synchronize()
        for h in range(2):
            want = evict_reference(w[0, h].cpu().numpy(), 900, 500, 2, 3)
            assert (kept[0, h].cpu().numpy() == want).all()
            assert torch.equal(bits(pages.rows(0, 500)[0][:, h]), bits(old[0][torch.from_numpy(want).cuda(), h]))


# ---------------------------------------------------------------------------------- compaction
@pytest.mark.parametrize("B,N,Hkv,Dh,page,dtype,head_major", [(1, 64, 8, 128, 16, BF, False), (5, 64, 2, 64, 8, F16, True), (3, 256, 2, 256, 64, BF, False),
                                                              (2, 1, 1, 8, 1, BF, False), (7, 100, 3, 72, 32, BF, True)])
@pytest.mark.parametrize("order", ["rising", "any"])
def test_compact(B, N, Hkv, Dh, page, dtype, head_major, order):
    rng = np.random.default_rng(B * N)
    prefix = [int(x) for x in rng.integers(0, 300, B)]
    pages = Pages([p + N for p in prefix], Hkv, Dh, dtype, page, head_major=head_major, seed=N)
    path = np.full((B, N), -1, dtype=np.int32)
    lens = [N - 1] + [int(x) for x in rng.integers(0, N, B - 1)]
    for b in range(B):
        if order == "rising":
            path[b, :lens[b] + 1] = np.concatenate([[0], np.sort(rng.choice(np.arange(1, N), lens[b], replace=False))]) if N > 1 else 0
        else:
            path[b, :lens[b] + 1] = rng.permutation(N)[:lens[b] + 1]
    rows = pages.max_pages * page
    w = torch.rand(B, Hkv, rows + 2, device="cuda")
    want_w, want_k, want_v = w.clone(), pages.k.clone(), pages.v.clone()
    for b in range(B):
        j = torch.arange(lens[b] + 1, device="cuda")
        src = prefix[b] + torch.from_numpy(path[b, :lens[b] + 1]).cuda().long()
        (p1, s1), (p2, s2) = pages.at(b, src), pages.at(b, prefix[b] + j)
        want_k[p2, s2], want_v[p2, s2] = pages.k[p1, s1], pages.v[p1, s1]
        want_w[b][:, prefix[b] + j] = w[b][:, src]
    new = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    T.talon_paged_compact(pages.cache, torch.from_numpy(path).cuda(), i32(lens), i32(prefix), new, weights=w)
    assert new.tolist() == [p + n + 1 for p, n in zip(prefix, lens)]
    assert torch.equal(bits(pages.k), bits(want_k)) and torch.equal(bits(pages.v), bits(want_v)) and torch.equal(w, want_w)
    assert not pages.cache.status.any()


def test_compact_with_fewer_weights_than_rows():
    pages = Pages([16], 1, 64, BF, page=16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    wide = torch.arange(20.0, device="cuda").view(1, 1, 20)
    new = i32([0])
    T.talon_paged_compact(pages.cache, i32([[0, 2, 5, -1, -1, -1]]), i32([2]), i32([4]), new, weights=wide[:, :, :9])
    assert new.tolist() == [7] and wide[0, 0].tolist() == [0, 1, 2, 3, 4, 6] + list(range(6, 20))   # row 9 is beyond the nine


def test_compact_at_the_end_of_the_table_and_on_bad_input():
    pages = Pages([40, 40, 40], 2, 64, BF, page=16)           # three pages: 48 rows
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    path = i32([[0, 2, 9, -1], [0, 2, 3, 300], [0, -5, 3, -1]])
    pages.table[2, 2] = 999                                   # where rows 40 .. 43 of sequence 2 would be
    old = pages.k.clone()
    new = i32([0, 0, 0])
    T.talon_paged_compact(pages.cache, path, i32([2, 3, 2]), i32([46, 36, 40]), new)
    # sequence 0: rows 46 and 47 have a place, 48 has none; node 300 and node -5 are none of four; sequence 2's page is outside the pool
    assert new.tolist() == [48, 40, 43]
    assert pages.cache.status.tolist() == [T.TALON_STATUS_BAD_PAGE, 0, T.TALON_STATUS_BAD_PAGE]
    (p1, s1), (p2, s2) = pages.at(1, torch.tensor([38, 39], device="cuda")), pages.at(1, torch.tensor([37, 38], device="cuda"))
    want = old.clone()
    want[p2, s2] = old[p1, s1]
    assert torch.equal(bits(pages.k), bits(want))


# ---------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", [BF, F16])
def test_a_decoding_loop_on_a_paged_cache(dtype):
    """A prompt in two chunks, then steps of: draft tree -> rotated rows into the pages -> tree attention -> accepted path -> weights ->
    compaction, and an eviction between them, against a plain cache that the test keeps in 64-bit-checked form."""
    B, Hq, Hkv, Dh, V, N, page = 2, 8, 2, 64, 500, 20, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)
    rows = 64 * 5
    pages = Pages([rows] * B, Hkv, Dh, dtype, page)
    cache = pages.cache
    st = T.TreeState(B, N)
    Np = st.N_pad
    cand = T.Candidates(B, Np, 4)
    ws = T.make_expand_workspace(B, Np, V, 4, T.TALON_DTYPE_F32)
    vws = T.make_verify_workspace(B, Np, V, T.TALON_DTYPE_F32)
    mask = torch.zeros(B, Np, 1, dtype=torch.int64, device="cuda")
    freq = (10000.0 ** (-torch.arange(Dh // 2, dtype=torch.float64) / (Dh // 2))).float().cuda()
    i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device="cuda")
    length, true_len, new_len = i32(B), i32(B), i32(B)
    aws = torch.empty(max(T.talon_paged_attention_workspace_bytes(B, n, Hq, Hkv, Dh, rows) for n in (Np, 70)), dtype=torch.uint8, device="cuda")
    weights = torch.zeros(B, Hkv, rows, device="cuda")
    path, accept, bonus, target, bad = i32(B, Np), i32(B), i32(B), i32(B, Np), i32(B)
    held = [[] for _ in range(B)]        # the test's own rows: (k, v) of every row of the cache, as stored

    def forward(n, pos, mask_words=None, offset=None):
        Nq = pos.shape[1]
        x = rand(B, Nq, Hq + 2 * Hkv, Dh).to(dtype)
        q = torch.empty(B, Nq, Hq, Dh, dtype=dtype, device="cuda")
        out, lse = torch.zeros_like(q), torch.zeros(B, Nq, Hq, device="cuda")
        T.talon_rotary_store(cache, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], q, n, length, pos[None], freq, pos_base=true_len)
        T.talon_paged_attention(cache, q, n, length, rows, out, lse, aws, mask=mask_words, offset=offset, softcap=20.0)
        for b in range(B):
            m, P = int(n[b]), int(length[b])
            k, v = pages.rows(b, P + m)
            if P:
                assert torch.equal(bits(k[:P]), bits(torch.stack([r[0] for r in held[b]]))) and torch.equal(bits(v[:P]), bits(torch.stack([r[1] for r in held[b]])))
            sees = torch.ones(m, P + m, dtype=torch.bool, device="cuda")
            if mask_words is None:
                sees[:, P:] = torch.ones(m, m, dtype=torch.bool, device="cuda").tril()
            else:
                sees[:, P:] = (mask_words[b, :m, :1] >> torch.arange(m, device="cuda")) & 1 > 0
            where = torch.arange(P + m, device="cuda")
            want, want_lse, tol, tol_lse = attention_of(q[b, :m], k, v, sees, 1 / math.sqrt(Dh), cap=20.0, pos_q=where[P:], pos_k=where)
            assert_close(out[b, :m], want, tol, "out")
            assert_close(lse[b, :m], want_lse, tol_lse, "lse")
        return q, lse

    def hold(b, first, count):
        p, s = pages.at(b, torch.arange(first, first + count, device="cuda"))
        held[b] += [(pages.k[pp, ss].clone(), pages.v[pp, ss].clone()) for pp, ss in zip(p.tolist(), s.tolist())]

    for n in (i32(B, v=70), torch.tensor([33, 1], dtype=torch.int32, device="cuda")):     # the prompt
        q, lse = forward(n, torch.arange(70, device="cuda", dtype=torch.int32).expand(B, 70).contiguous())
        T.talon_paged_weights(cache, q, n, length, rows, lse, weights, prior=weights, softcap=20.0)
        for b in range(B):
            hold(b, int(length[b]), int(n[b]))
        length, true_len = length + n, true_len + n
    accepted = 0
    for step in range(4):
        logits = rand(B, Np, V) * 4.0
        T.talon_build_tree(i32(B, v=1), logits, st, 4, 0.03, 4, 1, 8, cand, ws, mask)
        q, lse = forward(st.n_nodes, st.depth, mask, st.depth)
        T.talon_target_argmax(logits + 0.3 * rand(B, Np, V), st, target, None, bad, vws)
        T.talon_greedy_accept(st, target, bad, path, accept, bonus)
        on_path = torch.zeros(B, Np, dtype=torch.bool, device="cuda")
        for b in range(B):
            on_path[b, path[b, :int(accept[b]) + 1].long()] = True
        counts = torch.where(on_path[:, :, None], lse, torch.full_like(lse, math.inf))
        T.talon_paged_weights(cache, q, st.n_nodes, length, rows, counts, weights, prior=weights, mask=mask, offset=st.depth, softcap=20.0)
        for b in range(B):
            P = int(length[b])
            p, s = pages.at(b, P + path[b, :int(accept[b]) + 1].long())
            held[b] += [(pages.k[pp, ss].clone(), pages.v[pp, ss].clone()) for pp, ss in zip(p.tolist(), s.tolist())]
            accepted += int(accept[b])
        T.talon_paged_compact(cache, path, accept, length, new_len, weights=weights)
        true_len = true_len + accept + 1
        length = new_len.clone()
        assert length.tolist() == [len(h) for h in held]
        if step == 1:
            kept = i32(B, Hkv, 60)
            before = [list(h) for h in held]
            w = weights.clone()
            T.talon_paged_evict(cache, length, rows, weights, 60, kept, new_len, n_sink=2, n_recent=8, new_weights=weights)
            for b in range(B):
                keep = [evict_reference(w[b, h].cpu().numpy(), int(length[b]), 60, 2, 8) for h in range(Hkv)]
                assert [list(x) for x in keep] == [list(x) for x in kept[b].cpu().numpy()]
                held[b] = [tuple(torch.stack([before[b][keep[h][m]][t][h] for h in range(Hkv)]) for t in range(2)) for m in range(60)]
            length = new_len.clone()
    assert accepted > 0 and not cache.status.any() and not (st.status & T.TALON_STATUS_BAD_ROW).any()
