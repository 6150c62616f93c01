"""The paged-cache calls of a speculative decoding server, as they are measured.

A case is one of five kinds of call on a cache kept in pages, each as a serving loop makes it:

  store    talon_rotary_store: the new tokens' queries and keys rotated, keys and values written into the pages
  attend   talon_paged_attention: the new tokens (one token, a tree, a chunk of a prompt) over the paged cache
  weigh    talon_paged_weights: the attention weight that every cached row has received, added up
  evict    talon_paged_evict: the rows of least weight dropped, the others moved together
  compact  talon_paged_compact: the rows of the accepted path moved behind the prefix

Shapes are those of workloads/configs.py (8B-class and 70B-class targets: 32 or 64 query and 8 KV heads of
128; heads of 64; prefixes of 2048 to 16384; trees of 60 to 256 nodes) and generic ones around them.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # one chat turn decodes one token: nothing but the latency of a launch
        dict(_STORE, name="store-1", B=1, N=1, L=2048),
        # prompts with pictures, four sequences: positions in time, height and width, keys laid out head by head
        dict(_STORE, name="store-images-x4", B=4, N=2048, L=1000, axes=3, ragged=True, page=64, head_major=True, interleaved=True),
        # one token of one sequence of an 8B-class target at a 2k prefix
        dict(_ATTEND, name="attend-1", B=1, N=1, L=2048),
        # a full batch decodes: ragged prefixes up to 8k, a score that falls with the distance, fp16
        dict(_ATTEND, name="attend-x64-distance", B=64, N=1, L=8192, ragged=True, dtype="f16", slopes=True),
        # four trees of 128 nodes verified at 4k, scores capped
        dict(_ATTEND, name="attend-trees-x4-capped", B=4, N=128, L=4096, new="tree", cap=30.0, ragged=True),
        # two prompts prefilled by chunks of 2048 tokens behind up to 8k that are in the cache
        dict(_ATTEND, name="attend-chunk-x2", B=2, N=2048, L=8192, ragged=True, page=64),
        # the weight that eight sequences' rows get from one decoded token, at 16k
        dict(_WEIGH, name="weigh-x8", B=8, N=1, L=16384),
        # ... and from a chunk of 512 tokens at 8k
        dict(_WEIGH, name="weigh-chunk", B=1, N=512, L=8192, ragged=True, page=64),
        # one sequence's cache cut from 4k rows to 1k, in place
        dict(_EVICT, name="evict-1", B=1, L=4096, budget=1024),
        # sixteen sequences cut from up to 16k to 4k, into other pages (theirs are shared)
        dict(_EVICT, name="evict-x16", B=16, L=16384, budget=4096, ragged=True, apart=True),
        # the accepted path of one tree of 60 nodes
        dict(_COMPACT, name="compact-1", B=1, N=64, L=2048),
        # ... and of sixteen of 256, deep ones, with the rows' weights
        dict(_COMPACT, name="compact-x16", B=16, N=256, L=4096, deep=True, ragged=True, page=64),
    ]


_HEADS = dict(Hq=32, Hkv=8, Dh=128, dtype="bf16", page=16, head_major=False, ragged=False)
_SCORES = dict(new="causal", cap=0.0, slopes=False, window=0)
_STORE = dict(_HEADS, kind="store", axes=1, interleaved=False, partial=False)
_ATTEND = dict(_HEADS, **_SCORES, kind="attend")
_WEIGH = dict(_HEADS, **_SCORES, kind="weigh")
_EVICT = dict(_HEADS, kind="evict", apart=False)
_COMPACT = dict(_HEADS, kind="compact", deep=False)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_MOST_FLOPS = 4.0 * 2 * 2048 * 32 * 128 * 8192     # products of the listed chunk (causal half of its own tokens aside)
_MOST_SCORES = 2 * 2048 * 32 * 8192                # its scores, which the plain form holds
_MOST_ROWS = 64 * 8192                             # cached rows of the widest batch


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "attend", "weigh", "evict", "compact"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 16])
    c = dict(_HEADS, Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 3, 4, 4, 5, 8, 8]), Dh=rng.choice([64, 128, 128, 128, 256]),
             dtype=rng.choice(["bf16", "bf16", "f16"]), page=rng.choice([8, 16, 16, 32, 64, 128, 256]),
             head_major=rng.random() < 0.3, ragged=rng.random() < 0.6, kind=kind)
    row = Hkv * c["Dh"] / 1024.0                   # a cached row against the listed ones'
    if kind == "store":
        c.update(N=_log_int(rng, 1, 4096), L=_log_int(rng, 1, 8192), axes=rng.choice([1, 1, 2, 3, 4]),
                 interleaved=rng.random() < 0.4, partial=rng.random() < 0.3)
        c["B"] = _cap(rng, 64, 16384 * 1024 * 5 / (c["N"] * (c["Hq"] + 2 * Hkv) * c["Dh"]), _MOST_ROWS / (row * (c["N"] + c["L"])))
    elif kind in ("attend", "weigh"):
        new = rng.choice(["causal", "causal", "tree", "causal"])
        N = _log_int(rng, 2, 256) if new == "tree" else rng.choice([1, 1, _log_int(rng, 2, 2048)])
        c.update(new=new, N=N, L=_log_int(rng, 1, 16384), cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                 slopes=rng.random() < 0.25, window=rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]))
        pairs = c["N"] * c["Hq"] * (c["L"] + c["N"])
        c["N"] = max(1, int(c["N"] * min(1.0, _MOST_SCORES / pairs, _MOST_FLOPS / (4.0 * pairs * c["Dh"]))))
        pairs = c["N"] * c["Hq"] * (c["L"] + c["N"])
        c["B"] = _cap(rng, 64, min(_MOST_SCORES / pairs, _MOST_FLOPS / (4.0 * pairs * c["Dh"])), _MOST_ROWS / (row * (c["N"] + c["L"])))
    elif kind == "evict":
        c.update(L=_log_int(rng, 16, 65536), apart=rng.random() < 0.5)
        c["budget"] = max(8, int(c["L"] * rng.choice([0.1, 0.25, 0.5, 0.9])))
        c["B"] = _cap(rng, 32, 16 * 16384 / (row * c["L"]))
    else:
        c.update(N=64 * rng.randint(1, 4), L=_log_int(rng, 1, 8192), deep=rng.random() < 0.5)
        c["B"] = _cap(rng, 64, _MOST_ROWS / (row * (c["N"] + c["L"])))
    return c


def _cap(rng, most, *limits):
    b = _log_int(rng, 1, most)
    for x in limits:
        b = min(b, int(x))
    return max(1, b)


# ---------------------------------------------------------------------------------- inputs
_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# the first rows and the last ones stay whatever they weigh
_SINK, _RECENT = 4, 32


def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) % (2 ** 62))
    return g


def _randn(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def _pool(case, pages, dtype, g):
    """[pages][page_size][Hkv][Dh], the heads of a page together or its tokens."""
    p, H, D = case["page"], case["Hkv"], case["Dh"]
    if case["head_major"]:
        return _randn((pages, H, p, D), dtype, g).transpose(1, 2)
    return _randn((pages, p, H, D), dtype, g)


def _lengths(case, most, g, least=1):
    B = case["B"]
    if not case["ragged"]:
        return torch.full((B,), most, dtype=torch.int32, device="cuda")
    n = torch.randint(max(least, most // 4), most + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    n[0] = most
    return n


def prepare(case, seed):
    g = _generator(seed, 7)
    B, Hq, Hkv, D, L = case["B"], case["Hq"], case["Hkv"], case["Dh"], case["L"]
    N = case.get("N", 0)
    dt = _DTYPES[case["dtype"]]
    per_seq = (L + N + case["page"] - 1) // case["page"]
    tables = 2 if case.get("apart") else 1
    pages = B * per_seq * tables
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    s = {"case": case, "k": _pool(case, pages, dt, g), "v": _pool(case, pages, dt, g),
         "table": order[:B * per_seq].view(B, per_seq).contiguous(), "prefix": _lengths(case, L, g)}
    if tables == 2:
        s["table2"] = order[B * per_seq:].view(B, per_seq).contiguous()
    kind = case["kind"]
    if kind in ("store", "attend", "weigh"):
        s["n"] = _lengths(case, N, g)
    if kind == "store":
        fused = _randn((B, N, Hq + 2 * Hkv, D), dt, g)      # what one projection writes
        s["q"], s["key"], s["value"] = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:]
        s["q_out"] = torch.zeros(B, N, Hq, D, dtype=dt, device="cuda")
        pairs = D // 4 if case["partial"] else D // 2
        s["inv_freq"] = (500000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()
        step = torch.arange(N, device="cuda", dtype=torch.int32)
        if case["axes"] == 1:
            s["pos"] = step.expand(1, B, N).contiguous()
            s["axis"] = None
        else:                                               # pictures of 28 x 28 patches: time, height, width, ...
            place = [step // 784, step // 28 % 28, step % 28, step % 7]
            s["pos"] = torch.stack([p.expand(B, N) for p in place[:case["axes"]]]).contiguous()
            s["axis"] = (torch.arange(pairs, device="cuda") % case["axes"]).to(torch.int32)
        s["base"] = s["prefix"] + torch.randint(0, 100000, (B,), device="cuda", generator=g, dtype=torch.int32)
    elif kind in ("attend", "weigh"):
        s["q"] = _randn((B, N, Hq, D), dt, g, 2.0)
        s["mask"] = s["offset"] = s["slopes"] = None
        if case["new"] == "tree":
            s["mask"], s["offset"] = _tree(B, N, g)
        if case["slopes"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq)
        s["out"] = torch.zeros(B, N, Hq, D, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(B, N, Hq, device="cuda")
        if kind == "weigh":
            s["lse"] = _plain_attend(s)[1]
            s["prior"] = torch.rand(B, Hkv, L + N, device="cuda", generator=g) * 4.0
            s["weights"] = torch.zeros(B, Hkv, L + N, device="cuda")
    elif kind == "evict":
        s["weights"] = torch.exp(2.0 * torch.randn(B, Hkv, L, device="cuda", generator=g))
        s["new_weights"] = torch.zeros(B, Hkv, L, device="cuda")
        s["kept"] = torch.zeros(B, Hkv, case["budget"], dtype=torch.int32, device="cuda")
        s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["recent"] = min(_RECENT, case["budget"] - _SINK)
    else:
        most = min(N - 1, 60) if case["deep"] else min(N - 1, 8)
        skip = torch.randint(1, max(2, (N - 1) // most + 1), (B, most), device="cuda", generator=g)
        path = torch.cat([torch.zeros_like(skip[:, :1]), skip.cumsum(1)], 1)
        s["accept"] = torch.randint(0, most + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
        s["accept"][0] = most
        s["path"] = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
        j = torch.arange(most + 1, device="cuda")
        s["path"][:, :most + 1] = torch.where(j <= s["accept"][:, None], path, -1).to(torch.int32)
        s["weights"] = torch.rand(B, Hkv, L + N, device="cuda", generator=g)
        s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if own:   # the handle and the scratch that a server keeps
        import paper_2601_07353_amd as T
        s["cache"] = T.PagedCache(s["k"], s["v"], s["table"])
        if tables == 2:
            s["cache2"] = T.PagedCache(s["k"], s["v"], s["table2"])
        if kind == "attend":
            nb = T.talon_paged_attention_workspace_bytes(B, N, Hq, Hkv, D, L)
            s["workspace"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
    return s


def _tree(B, N, g):
    """Trees of N nodes whose parents come before them: ancestor words [B][N][ceil(N/64)] and depths [B][N]."""
    i = torch.arange(N, device="cuda")
    parent = (torch.rand(B, N, device="cuda", generator=g) * i).long().clamp(max=N - 1)
    parent[:, 0] = 0
    reach = torch.zeros(B, N, N, dtype=torch.float32, device="cuda")
    reach.scatter_(2, parent[:, :, None], 1.0)
    reach = ((reach + torch.eye(N, device="cuda")) > 0).float()
    for _ in range(8):                                     # paths of up to 256 edges
        reach = (torch.matmul(reach, reach) > 0).float()
    words = (N + 63) // 64
    bits = torch.zeros(B, N, words * 64, dtype=torch.int64, device="cuda")
    bits[:, :, :N] = reach.long()
    shift = torch.arange(64, device="cuda")
    mask = (bits.view(B, N, words, 64) << shift).sum(-1)
    return mask, (reach.sum(-1) - 1).to(torch.int32)


# ---------------------------------------------------------------------------------- plain forms
def _rows(pool, table, page, W):
    """Rows 0 .. W-1 of every sequence: [B][W][Hkv][Dh]."""
    j = torch.arange(W, device="cuda")
    return pool[table[:, j // page].long(), (j % page).expand(table.shape[0], W)]


def _allowed(s, W):
    """[B][N][W] whether new token i sees row j, and [B][N][W] how far apart they stand."""
    case, N = s["case"], s["case"]["N"]
    P = s["prefix"].long()[:, None, None]
    n = s["n"].long()[:, None, None]
    i = torch.arange(N, device="cuda")[None, :, None]
    j = torch.arange(W, device="cuda")[None, None, :]
    fresh = (j - P).clamp(0, N - 1)
    if s["mask"] is None:
        sees = (j <= P + i).expand(-1, N, W)
    else:
        at = fresh.expand(-1, N, W)
        word = torch.gather(s["mask"], 2, at >> 6)
        sees = (j < P) | (((word >> (at & 63)) & 1) > 0)
    if s["offset"] is None:
        apart = P + i - j
    else:
        off = s["offset"].long()
        there = torch.where(j < P, j, P + torch.gather(off, 1, fresh[:, 0])[:, None])
        apart = P + off[:, :, None] - there
    sees = sees & (j < P + n) & (i < n)
    if case["window"]:
        sees = sees & (apart < case["window"])
    return sees, apart


def _plain_scores(s):
    """Scores [B][Hkv][N][G][W] in 32 bits, -inf where a token does not see a row; rows' keys in 32 bits."""
    case = s["case"]
    B, N, Hq, Hkv, D = case["B"], case["N"], case["Hq"], case["Hkv"], case["Dh"]
    G, W = Hq // Hkv, case["L"] + N
    k = _rows(s["k"], s["table"], case["page"], W).float().permute(0, 2, 3, 1).contiguous()
    q = s["q"].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    x = torch.matmul(q, k).view(B, Hkv, N, G, W) * (1.0 / math.sqrt(D))
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    sees, apart = _allowed(s, W)
    if case["slopes"]:
        x = x - s["slopes"].view(Hkv, 1, G, 1) * apart.abs().float()[:, None, :, None]
    return x.masked_fill(~sees[:, None, :, None], -math.inf)


def _plain_attend(s):
    case = s["case"]
    B, N, Hq, Hkv, D = case["B"], case["N"], case["Hq"], case["Hkv"], case["Dh"]
    G, W = Hq // Hkv, case["L"] + N
    x = _plain_scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x = torch.exp(x - top)
    total = x.sum(-1, keepdim=True)
    v = _rows(s["v"], s["table"], case["page"], W).float().transpose(1, 2).contiguous()
    o = torch.matmul(x.view(B, Hkv, N * G, W), v).view(B, Hkv, N, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + torch.log(total))[..., 0].permute(0, 2, 1, 3).reshape(B, N, Hq)
    real = (torch.arange(N, device="cuda") < s["n"][:, None])[:, :, None]
    out = o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).to(s["q"].dtype)
    return (torch.where(real[..., None], out, torch.zeros_like(out)), torch.where(real, lse, torch.zeros_like(lse)))


def _plain_weigh(s):
    case = s["case"]
    B, N, Hq, Hkv = case["B"], case["N"], case["Hq"], case["Hkv"]
    W = case["L"] + N
    lse = s["lse"].view(B, N, Hkv, Hq // Hkv).permute(0, 2, 1, 3)[..., None]
    got = torch.exp(_plain_scores(s) - lse).sum((2, 3))
    j = torch.arange(W, device="cuda")
    P = s["prefix"][:, None, None]
    new = torch.where(j < P, 0.9 * s["prior"], torch.zeros_like(s["prior"])) + got
    return torch.where(j < P + s["n"][:, None, None], new, s["weights"])


def _turned(x, cos, sin, pairs, interleaved):
    """x [B][N][H][Dh] in 32 bits with the first 2 * pairs values of a head rotated."""
    y = x.clone()
    a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    u, w = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2] = u, w
    else:
        y[..., :pairs], y[..., pairs:2 * pairs] = u, w
    return y


def _plain_store(s):
    case = s["case"]
    N, page, f = case["N"], case["page"], s["inv_freq"]
    pos = s["pos"] + s["base"][:, None]                                            # [axes][B][N]
    pos = pos[0][:, :, None] if s["axis"] is None else pos[s["axis"].long()].permute(1, 2, 0)
    angle = pos.double() * f.double()                                              # 64 bits: far positions
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    real = torch.arange(N, device="cuda") < s["n"][:, None]
    q = _turned(s["q"].float(), cos, sin, f.numel(), case["interleaved"]).to(s["q"].dtype)
    k = _turned(s["key"].float(), cos, sin, f.numel(), case["interleaved"]).to(s["q"].dtype)
    s["q_out"] = torch.where(real[:, :, None, None], q, s["q_out"])
    row = s["prefix"].long()[:, None] + torch.arange(N, device="cuda")
    at = torch.gather(s["table"].long(), 1, row // page), row % page
    at = at[0][real], at[1][real]
    s["k"][at], s["v"][at] = k[real], s["value"][real]
    return s["q_out"], s["k"], s["v"]


def _plain_evict(s):
    case = s["case"]
    B, Hkv, L, M, page = case["B"], case["Hkv"], case["L"], case["budget"], case["page"]
    j = torch.arange(L, device="cuda")
    n = s["prefix"].long()[:, None, None]
    w = torch.where((j < _SINK) | (j >= n - s["recent"]), torch.full_like(s["weights"], math.inf), s["weights"])
    w = torch.where(j < n, w, torch.full_like(w, -1.0))
    best = torch.sort(w, dim=-1, descending=True, stable=True)[1][..., :M]         # ties: the lowest row
    live = torch.arange(M, device="cuda") < torch.clamp(n, max=M)
    rows = torch.sort(torch.where(live, best, torch.full_like(best, L)), dim=-1)[0]
    kept = torch.where(live, rows, torch.full_like(rows, -1))
    src = rows.clamp(max=L - 1)
    s["new_weights"][..., :M] = torch.where(live, torch.gather(s["weights"], 2, src), s["new_weights"][..., :M])
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
    to = s["table2"] if case["apart"] else s["table"]
    m = torch.arange(M, device="cuda").expand(B, Hkv, M)
    src_at = (s["table"][b, src // page].long(), src % page, h.expand(B, Hkv, M))
    dst_at = (to[b, m // page].long(), m % page, h.expand(B, Hkv, M))
    k, v = s["k"][src_at][live.expand(B, Hkv, M)], s["v"][src_at][live.expand(B, Hkv, M)]
    dst_at = tuple(t[live.expand(B, Hkv, M)] for t in dst_at)
    s["k"][dst_at], s["v"][dst_at] = k, v
    return kept.to(torch.int32), torch.clamp(s["prefix"], max=M), s["new_weights"], s["k"], s["v"]


def _plain_compact(s):
    case = s["case"]
    B, N, page = case["B"], case["N"], case["page"]
    j = torch.arange(N, device="cuda")
    live = j <= s["accept"][:, None]
    P = s["prefix"].long()[:, None]
    src = P + s["path"].long().clamp(min=0)
    dst = P + j.expand(B, N)
    src_at = (torch.gather(s["table"].long(), 1, src // page), src % page)
    dst_at = (torch.gather(s["table"].long(), 1, dst // page), dst % page)
    k, v = s["k"][src_at][live], s["v"][src_at][live]
    s["k"][dst_at[0][live], dst_at[1][live]], s["v"][dst_at[0][live], dst_at[1][live]] = k, v
    at = torch.arange(B, device="cuda")[:, None].expand(B, N)[live]
    s["weights"][at, :, dst[live]] = s["weights"][at, :, src[live]]
    return s["k"], s["v"], s["weights"], s["prefix"] + s["accept"] + 1


# ---------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"store": _plain_store, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict, "compact": _plain_compact}[kind](s)
    import paper_2601_07353_amd as T
    if kind == "store":
        T.talon_rotary_store(s["cache"], s["q"], s["key"], s["value"], s["q_out"], s["n"], s["prefix"], s["pos"], s["inv_freq"],
                             pos_base=s["base"], pair_axis=s["axis"], interleaved=case["interleaved"])
        return s["q_out"], s["k"], s["v"]
    if kind == "attend":
        T.talon_paged_attention(s["cache"], s["q"], s["n"], s["prefix"], case["L"], s["out"], s["lse"], s["workspace"], mask=s["mask"],
                                offset=s["offset"], softcap=case["cap"], slopes=s["slopes"], window=case["window"])
        return s["out"], s["lse"]
    if kind == "weigh":
        T.talon_paged_weights(s["cache"], s["q"], s["n"], s["prefix"], case["L"], s["lse"], s["weights"], prior=s["prior"], decay=0.9,
                              mask=s["mask"], offset=s["offset"], softcap=case["cap"], slopes=s["slopes"], window=case["window"])
        return s["weights"]
    if kind == "evict":
        T.talon_paged_evict(s["cache"], s["prefix"], case["L"], s["weights"], case["budget"], s["kept"], s["new_len"], n_sink=_SINK,
                            n_recent=s["recent"], dst=s.get("cache2"), new_weights=s["new_weights"])
        return s["kept"], s["new_len"], s["new_weights"], s["k"], s["v"]
    T.talon_paged_compact(s["cache"], s["path"], s["accept"], s["prefix"], s["new_len"], weights=s["weights"])
    return s["k"], s["v"], s["weights"], s["new_len"]


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    B, Hq, Hkv, D, L = case["B"], case["Hq"], case["Hkv"], case["Dh"], case["L"]
    N, kind = case.get("N", 0), case["kind"]
    full = 0.625 if case["ragged"] else 1.0               # mean length against the largest one, but for the first
    mean = lambda most: most * (1.0 + (B - 1) * full) / B  # noqa: E731
    n, l = mean(N), mean(L)
    row = Hkv * D * 2.0                                     # one tensor's row of one token
    if kind == "store":
        return {"bytes": B * n * 2 * (Hq * D * 2.0 + 2 * row), "flops": B * n * (Hq + Hkv) * D * 3.0}
    if kind in ("attend", "weigh"):
        reach = min(l, case["window"]) if case["window"] else l
        pairs = B * Hq * n * (reach + (n + 1) / 2)
        if kind == "attend":
            return {"bytes": B * (2 * row * (min(l, reach + n) + n) + n * Hq * (D * 4.0 + 4)), "flops": pairs * D * 4.0}
        return {"bytes": B * (row * (min(l, reach + n) + n) + n * Hq * (D * 2.0 + 4) + Hkv * (l + l + n) * 4.0), "flops": pairs * D * 2.0}
    if kind == "evict":
        kept = min(case["budget"], l)
        return {"bytes": B * (4 * row * kept + Hkv * (4.0 * l + 12.0 * kept)), "flops": 0.0}
    moved = mean(min(N - 1, 60) if case["deep"] else min(N - 1, 8)) / (1.0 if B == 1 else 1.25)
    return {"bytes": B * moved * (4 * row + 8.0 * Hkv + 4.0), "flops": 0.0}


# ---------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """Attention, weights and rotation from their definitions, one sequence and KV head after the other; the moves of
    rows compute nothing."""
    kind = case["kind"]
    if kind in ("evict", "compact"):
        return None
    s = prepare(case, seed)
    B, N, Hq, Hkv, D, page = case["B"], case["N"], case["Hq"], case["Hkv"], case["Dh"], case["page"]
    G = Hq // Hkv
    lens, news, table = s["prefix"].tolist(), s["n"].tolist(), s["table"].long()
    if kind == "store":
        q_out, kp, vp = torch.zeros(B, N, Hq, D, dtype=torch.float64, device="cuda"), s["k"].double(), s["v"].double()
        f = s["inv_freq"].double()
        axis = torch.zeros(f.numel(), dtype=torch.long, device="cuda") if s["axis"] is None else s["axis"].long()
        one, two = torch.arange(f.numel(), device="cuda"), torch.arange(f.numel(), device="cuda")
        one, two = (2 * one, 2 * two + 1) if case["interleaved"] else (one, two + f.numel())
        for b in range(B):
            m, P = news[b], lens[b]
            place = (s["pos"][:, b, :m].double() + s["base"][b].double())[axis].T        # [m][pairs]
            turn = torch.polar(torch.ones_like(place * f), place * f)[:, None]
            rows = torch.arange(P, P + m, device="cuda")
            pg, sl = table[b, rows // page], rows % page
            for x, to in ((s["q"], "q"), (s["key"], "k")):
                y = x[b, :m].double()
                z = torch.complex(y[..., one], y[..., two]) * turn
                y[..., one], y[..., two] = z.real, z.imag
                if to == "q":
                    q_out[b, :m] = y
                else:
                    kp[pg, sl] = y
            vp[pg, sl] = s["value"][b, :m].double()
        return q_out, kp, vp
    if 2.0 * B * N * Hq * (case["L"] + N) * D > 4e12:
        return None
    out = torch.zeros(B, N, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, N, Hq, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if kind == "weigh" else None
    for b in range(B):
        m, P = news[b], lens[b]
        T = P + m
        rows = torch.arange(T, device="cuda")
        pg, sl = table[b, rows // page], rows % page
        off = torch.arange(m, device="cuda") if s["offset"] is None else s["offset"][b, :m].long()
        where = torch.cat([torch.arange(P, device="cuda"), P + off])
        away = (P + off)[:, None] - where[None]
        sees = torch.ones(m, T, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            sees[:, P:] = torch.ones(m, m, dtype=torch.bool, device="cuda").tril()
        else:
            bit = torch.arange(m, device="cuda")
            sees[:, P:] = (s["mask"][b, :m][:, bit // 64] >> (bit % 64)) & 1 == 1
        if case["window"]:
            sees &= away < case["window"]
        for g in range(Hkv):
            key, value = s["k"][pg, sl, g].double(), s["v"][pg, sl, g].double()
            for h in range(g * G, (g + 1) * G):
                x = s["q"][b, :m, h].double() @ key.T / math.sqrt(D)
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if case["slopes"]:
                    x = x - s["slopes"][h].double() * away.abs()
                x[~sees] = -math.inf
                if kind == "attend":
                    lse[b, :m, h] = torch.logsumexp(x, -1)
                    out[b, :m, h] = torch.nan_to_num(torch.softmax(x, -1), nan=0.0) @ value
                else:
                    if h == g * G:
                        weights[b, g, :T] = 0.0
                        weights[b, g, :P] = 0.9 * s["prior"][b, g, :P].double()
                    weights[b, g, :T] += torch.exp(x - s["lse"][b, :m, h].double()[:, None]).sum(0)
    return (out, lse) if kind == "attend" else weights
