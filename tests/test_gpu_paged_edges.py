"""The calls on a paged cache at the ends of what they allow: the largest batch, masks of more than four words, single heads and 128 of
them, broadcast queries, calls at the same time on two streams, one captured step replayed with other tokens, lengths beyond budgets."""
import math

import pytest
import torch

import paper_2601_07353_amd as T
from tests.paged_harness import Pages
from tests.test_gpu_paged_attention import Case
from tests.test_gpu_paged_rows import evict_case

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16

CASES = {
    "256 sequences, one token": dict(prefix=[(31 * i * i) % 700 for i in range(256)], fresh=[i % 2 for i in range(256)], Hq=4, Hkv=2, Dh=64),
    "256 sequences, some tokens": dict(prefix=[(17 * i) % 400 for i in range(256)], fresh=[1 + i % 20 for i in range(256)], Hq=8, Hkv=2, Dh=128, dtype=F16),
    "a mask of five words": dict(prefix=[100, 65], fresh=[300, 257], Hq=4, Hkv=2, Dh=64, new="random"),
    "a mask of five words, window": dict(prefix=[300], fresh=[290], Hq=8, Hkv=2, Dh=128, new="random", window=33, dtype=F16),
    "128 heads of their own": dict(prefix=[200], fresh=[3], Hq=128, Hkv=128, Dh=64, page=2),
    "one KV head for 128, heads of 256": dict(prefix=[300, 1], fresh=[5, 9], Hq=128, Hkv=1, Dh=256, page=2),
    "33 rows": dict(prefix=[900], fresh=[11], Hq=6, Hkv=2, Dh=128),
    "32 rows, heads of 256": dict(prefix=[900, 2000], fresh=[8, 3], Hq=8, Hkv=2, Dh=256, cap=9.0, slopes=True),
    "a page for all": dict(prefix=[900], fresh=[70], Hq=8, Hkv=2, Dh=64, page=4096),
    "nothing cached, a tree of one": dict(prefix=[0], fresh=[1], Hq=8, Hkv=2, Dh=128, new="tree"),
    "511 and 512 rows": dict(prefix=[130, 129], fresh=[128, 127], Hq=16, Hkv=4, Dh=128),
}


@pytest.mark.parametrize("name", CASES)
def test_ends(name):
    print("case", name, flush=True)
    c = Case(**CASES[name], seed=len(name))
    c.run()
    c.check()
    Case(**CASES[name], seed=len(name)).check_weights()


@pytest.mark.parametrize("what", ["sequences", "heads", "tokens"])
def test_a_query_for_all(what):
    """q broadcast along one of its dimensions (a stride of zero)."""
    c = Case([300, 40], [12, 12], 8, 2, 64)
    q = {"sequences": c.q[:1], "tokens": c.q[:, :1], "heads": c.q[:, :, :1]}[what].expand_as(c.q)
    c.q = q.contiguous()
    want = [x.clone() for x in c.run()]
    c.q = q
    c.out.fill_(7.0)
    c.run()
    assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])


def test_two_calls_at_once():
    """Two caches, two streams, a workspace each; one cache's readers share it."""
    a = Case([3000, 100], [64, 64], 16, 4, 128, new="tree")
    b = Case([2000, 1999], [1, 1], 32, 8, 128, dtype=F16)
    want = [x.clone() for c in (a, b) for x in c.run()]
    other = Case([2000, 1999], [1, 1], 32, 8, 128, dtype=F16)     # the same queries on the same pages
    other.pages = b.pages
    torch.cuda.synchronize()
    for c in (a, b, other):
        c.out.fill_(7.0)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for c, s in zip((a, b, other), streams):
            c.run(stream=s)
    for s in streams:
        s.synchronize()
    for c, (out, lse) in zip((a, b, other), (want[:2], want[2:], want[2:])):
        assert torch.equal(c.out.view(torch.int16), out.view(torch.int16)) and torch.equal(c.lse, lse)


def test_a_captured_step_with_other_tokens():
    """Rotary store, attention, weights and compaction in one graph: every replay on new tokens does what eager calls do."""
    B, N, Hq, Hkv, Dh = 2, 32, 8, 2, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    worlds = []
    for _ in range(2):
        pages = Pages([200, 90], Hkv, Dh, BF, room=400, seed=4)
        w = dict(pages=pages, out=torch.zeros(B, N, Hq, Dh, dtype=BF, device="cuda"), lse=torch.zeros(B, N, Hq, device="cuda"),
                 weights=torch.zeros(B, Hkv, 700, device="cuda"), len=torch.tensor([200, 90], dtype=torch.int32, device="cuda"),
                 new=torch.zeros(B, dtype=torch.int32, device="cuda"), qr=torch.zeros(B, N, Hq, Dh, dtype=BF, device="cuda"),
                 ws=torch.empty(T.talon_paged_attention_workspace_bytes(B, N, Hq, Hkv, Dh, 500), dtype=torch.uint8, device="cuda"))
        worlds.append(w)
    qkv = torch.zeros(B, N, Hq + 2 * Hkv, Dh, dtype=BF, device="cuda")
    n = torch.tensor([N, N - 3], dtype=torch.int32, device="cuda")
    pos = torch.arange(N, dtype=torch.int32, device="cuda").expand(1, B, N).contiguous()
    inv_freq = 10000.0 ** (-torch.arange(Dh // 2, device="cuda") / (Dh // 2))
    path = torch.zeros(B, N, dtype=torch.int32, device="cuda")
    accept = torch.zeros(B, dtype=torch.int32, device="cuda")

    def step(w):
        cache = w["pages"].cache
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        T.talon_rotary_store(cache, q, k, v, w["qr"], n, w["len"], pos, inv_freq, pos_base=w["len"])
        T.talon_paged_attention(cache, w["qr"], n, w["len"], 500, w["out"], w["lse"], w["ws"])
        T.talon_paged_weights(cache, w["qr"], n, w["len"], 500, w["lse"], w["weights"], decay=0.9, prior=w["weights"])
        T.talon_paged_compact(cache, path, accept, w["len"], w["new"], weights=w["weights"])
        w["len"].copy_(w["new"])

    def fill():
        qkv.copy_(torch.randn(qkv.shape, device="cuda", generator=g))
        accept.copy_(torch.randint(1, 8, (B,), device="cuda", generator=g))
        path.copy_(torch.cat([torch.zeros(B, 1, device="cuda"), torch.sort(torch.randperm(28, device="cuda", generator=g)[:N - 5] + 1)[0].expand(B, -1),
                              torch.full((B, 4), -1.0, device="cuda")], -1).to(torch.int32))

    fill()
    for w in worlds:
        step(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(worlds[0])
    for _ in range(4):
        fill()
        graph.replay()
        (torch.randn(500, 500, device="cuda") @ torch.randn(500, 500, device="cuda")).sum().item()
        step(worlds[1])
        torch.cuda.synchronize()
        a, b = worlds
        for k in ("out", "lse", "weights", "len", "qr"):
            assert torch.equal(a[k], b[k]), k
        for x, y in ((a["pages"].k, b["pages"].k), (a["pages"].v, b["pages"].v)):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    assert not worlds[0]["pages"].cache.status.any() and worlds[0]["len"].min() > 90


EVICTIONS = {
    "as many rows as a thread has four of": dict(lens=[4096, 4095, 1025], budget=1000, sink=3, recent=5, kind="few", Hkv=2, Dh=64, page=64),
    "one more": dict(lens=[4097, 4096], budget=4095, sink=3, recent=5, kind="few", Hkv=2, Dh=64, page=64),
    "as many as lie in registers": dict(lens=[16384, 16383], budget=8191, kind="few", Hkv=1, Dh=64, page=64),
    "zeros, more than lie in registers": dict(lens=[16390], budget=16389, kind="zero", Hkv=2, Dh=8, page=64),
    "a budget of more than there is": dict(lens=[100, 3], budget=500, sink=100, recent=400, Hkv=2, Dh=64),
    "not numbers, more than lie in registers": dict(lens=[20000], budget=15000, sink=1, recent=1, kind="odd", Hkv=1, Dh=64, page=64),
    "a head of 1024, in rows": dict(lens=[300], budget=77, Hkv=1, Dh=1024),
    "many heads, in whole rows": dict(lens=[400] * 16, budget=130, Hkv=8, Dh=128, sink=1, recent=9),
}


@pytest.mark.parametrize("place", ["new weights", "weights in place"])
@pytest.mark.parametrize("name", EVICTIONS)
def test_evictions(name, place):
    print("case", name, place, flush=True)
    evict_case(place=place, **EVICTIONS[name])


def test_eviction_of_lengths_outside_their_bounds():
    """Above max_len: max_len; below zero: no rows."""
    pages = Pages([300, 300], 2, 64, BF)
    w = torch.rand(2, 2, 300, device="cuda")
    kept = torch.full((2, 2, 100), -7, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    length = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")
    old = [x.clone() for x in pages.rows(1, 300)]
    T.talon_paged_evict(pages.cache, length, 200, w, 100, kept, new_len, n_recent=1)
    assert new_len.tolist() == [100, 0] and (kept[1] == -1).all() and (kept[0, :, -1] == 199).all()
    want = torch.sort(torch.sort(-w[0, :, :199], dim=-1, stable=True)[1][:, :99], -1)[0]
    assert torch.equal(kept[0, :, :99].long(), want)
    assert all(torch.equal(x, y) for x, y in zip(old, pages.rows(1, 300)))


def test_rows_on_another_stream():
    """A store, an eviction and a compaction on a stream that is not the current one, behind work that they depend on."""
    pages = Pages([500], 2, 64, F16, room=20, seed=2)
    again = Pages([500], 2, 64, F16, room=20, seed=2)
    n = torch.tensor([20], dtype=torch.int32, device="cuda")
    P = torch.tensor([500], dtype=torch.int32, device="cuda")
    x = torch.randn(1, 20, 8, 64, device="cuda").half()
    w = torch.rand(1, 2, 520, device="cuda")
    pos = torch.arange(20, dtype=torch.int32, device="cuda").view(1, 1, 20)
    inv_freq = torch.rand(32, device="cuda")
    path = torch.arange(0, 20, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    path[0, 0] = 0
    acc = torch.tensor([7], dtype=torch.int32, device="cuda")

    def rows(p, stream=None):
        out = dict(q=torch.zeros(1, 20, 4, 64, dtype=F16, device="cuda"), len=torch.zeros(1, dtype=torch.int32, device="cuda"),
                   kept=torch.zeros(1, 2, 100, dtype=torch.int32, device="cuda"), cut=torch.zeros(1, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        T.talon_rotary_store(p.cache, x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], out["q"], n, P, pos, inv_freq, stream=stream)
        T.talon_paged_compact(p.cache, path, acc, P, out["len"], stream=stream)
        T.talon_paged_evict(p.cache, out["len"], 520, w, 100, out["kept"], out["cut"], stream=stream)
        torch.cuda.synchronize()
        return out

    want = rows(pages)
    got = rows(again, torch.cuda.Stream())
    assert all(torch.equal(got[k], want[k]) for k in want) and got["len"].item() == 508 and got["cut"].item() == 100
    assert torch.equal(pages.k.view(torch.int16), again.k.view(torch.int16)) and torch.equal(pages.v.view(torch.int16), again.v.view(torch.int16))
