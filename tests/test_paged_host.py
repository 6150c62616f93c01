"""The calls on a paged cache on a machine without a GPU: what is refused, by the C ABI and by the Python binding, before anything is
launched (the pointers are made up; validation never dereferences them), and the launch plan."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2601_07353_amd as T
from paper_2601_07353_amd import build as B
from paper_2601_07353_amd.binding import _CPagedCache, _CScores, _CView

P = 0x7000000
INVALID, UNSUPPORTED, WORKSPACE = T.TALON_ERR_INVALID_ARG, T.TALON_ERR_UNSUPPORTED, T.TALON_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return T.load_library()


def cache(**kw):
    d = dict(B=2, Hkv=2, Dh=128, dtype=1, num_pages=64, page_size=16, max_pages=20, stride_page=16 * 256, stride_token=256, stride_head=128,
             k=P, v=P + 0x1000000, page_table=P + 4, status=P + 8)
    d.update(kw)
    return _CPagedCache(*[d[name] for name, _ in _CPagedCache._fields_])


def view(data=P, sb=10 * 1024, st=1024, sh=128):
    return _CView(data, sb, st, sh)


def scores(mask=None, offset=None, slopes=None, scale=0.0, softcap=0.0, window=0):
    return _CScores(mask, offset, slopes, scale, softcap, window)


def said(lib):
    return lib.talon_last_error_string().decode()


def calls(lib):
    """One call of each entry point that all checks pass but those of the arguments that are changed: name -> f(**changes)."""
    ref = lambda x: None if x is None else ctypes.byref(x)

    def store(c=None, q=None, k=None, v=None, o=None, N=10, Hq=8, n=P, p=P, pos=P, axes=1, base=None, freq=P, pairs=64, axis=None):
        return lib.talon_rotary_store(ref(c or cache()), ref(q or view()), ref(k or view()), ref(v or view()), ref(o or view()), N, Hq, n, p, pos, axes,
                                      base, freq, pairs, axis, 0, None)

    def attend(c=None, q=None, o=None, N=10, Hq=8, n=P, p=P, most=300, s=None, lse=None, ws=P, nb=1 << 40):
        return lib.talon_paged_attention(ref(c or cache()), ref(q or view()), N, Hq, n, p, most, ref(s), ref(o or view()), lse, ws, nb, None)

    def weigh(c=None, q=None, N=10, Hq=8, n=P, p=P, most=300, s=None, lse=P, decay=1.0, prior=None, w=P, sb=640, sh=320):
        return lib.talon_paged_weights(ref(c or cache()), ref(q or view()), N, Hq, n, p, most, ref(s), lse, decay, prior, w, sb, sh, None)

    def evict(c=None, dst=None, n=P, most=300, w=P, sb=640, sh=320, budget=100, sink=0, recent=0, kept=P, new=P + 64, nw=None, nsb=0, nsh=0):
        return lib.talon_paged_evict(ref(c or cache()), ref(dst), n, most, w, sb, sh, budget, sink, recent, kept, new, nw, nsb, nsh, None)

    def compact(c=None, N=10, path=P, accept=P, p=P, new=P + 64, w=None, rows=320, sb=640, sh=320):
        return lib.talon_paged_compact(ref(c or cache()), N, path, accept, p, new, w, rows, sb, sh, None)
    return dict(store=store, attend=attend, weigh=weigh, evict=evict, compact=compact)


BAD_CACHES = [(dict(B=0), INVALID, "B=0"), (dict(B=257), INVALID, "B=257"), (dict(dtype=0), UNSUPPORTED, "dtype 0"), (dict(dtype=3), UNSUPPORTED, "dtype"),
              (dict(Hkv=0), INVALID, "Hkv=0"), (dict(Hkv=129), UNSUPPORTED, "Hkv=129"), (dict(Dh=0), INVALID, "Dh=0"), (dict(Dh=100), INVALID, "Dh=100"),
              (dict(Dh=1032), UNSUPPORTED, "Dh"), (dict(page_size=0), INVALID, "page_size"), (dict(page_size=24), INVALID, "page_size=24"),
              (dict(page_size=-16), INVALID, "page_size"), (dict(num_pages=0), INVALID, "num_pages"), (dict(max_pages=0), INVALID, "max_pages"),
              (dict(max_pages=1 << 30), UNSUPPORTED, "rows per sequence"), (dict(k=0), INVALID, "NULL"), (dict(v=0), INVALID, "NULL"),
              (dict(page_table=0), INVALID, "NULL"), (dict(status=0), INVALID, "NULL"), (dict(k=P + 8), INVALID, "aligned"),
              (dict(page_table=P + 2), INVALID, "misaligned"), (dict(stride_token=129), INVALID, "strides"), (dict(stride_head=64), INVALID, "strides"),
              (dict(stride_page=-4096), INVALID, "strides"), (dict(num_pages=1 << 30, stride_page=1 << 20), UNSUPPORTED, "64 GiB")]


@pytest.mark.parametrize("name", ["store", "attend", "weigh", "evict", "compact"])
def test_caches_that_are_refused(lib, name):
    call = calls(lib)[name]
    for change, code, text in BAD_CACHES:
        assert call(c=cache(**change)) == code and text in said(lib), (change, said(lib))
    assert getattr(lib, {"store": "talon_rotary_store"}.get(name, "talon_paged_attention")) is not None


def test_null_cache(lib):
    v = ctypes.byref(view())
    assert lib.talon_paged_attention(None, v, 10, 8, P, P, 300, None, v, None, P, 1 << 40, None) == INVALID and "NULL" in said(lib)
    assert lib.talon_paged_compact(None, 10, P, P, P, P + 64, None, 0, 0, 0, None) == INVALID


@pytest.mark.parametrize("name", ["store", "attend", "weigh"])
def test_new_tokens_that_are_refused(lib, name):
    call = calls(lib)[name]
    for change, code, text in [(dict(N=0), INVALID, "N=0"), (dict(N=65537), INVALID, "N=65537"), (dict(n=None), INVALID, "n_new"), (dict(p=None), INVALID, "prefix_len"),
                               (dict(n=P + 2), INVALID, "misaligned"), (dict(Hq=0), INVALID, "Hq=0"), (dict(q=view(data=0)), INVALID, "q is NULL"),
                               (dict(q=view(data=P + 8)), INVALID, "q is not 16-byte"), (dict(q=view(sh=12)), INVALID, "q: strides"), (dict(q=view(st=-1024)), INVALID, "q: strides")]:
        assert call(**change) == code and text in said(lib), (change, said(lib))


@pytest.mark.parametrize("name", ["attend", "weigh"])
def test_scores_that_are_refused(lib, name):
    call = calls(lib)[name]
    nan, inf = float("nan"), float("inf")
    for change, code, text in [(dict(s=scores(scale=-1.0)), INVALID, "scale"), (dict(s=scores(scale=nan)), INVALID, "scale"), (dict(s=scores(scale=inf)), INVALID, "scale"),
                               (dict(s=scores(softcap=-1.0)), INVALID, "softcap"), (dict(s=scores(softcap=nan)), INVALID, "softcap"), (dict(s=scores(softcap=inf)), INVALID, "softcap"),
                               (dict(s=scores(window=-1)), INVALID, "window"), (dict(s=scores(mask=P + 4)), INVALID, "mask"), (dict(s=scores(offset=P + 2)), INVALID, "offset"),
                               (dict(s=scores(slopes=P + 2)), INVALID, "slopes"), (dict(most=-1), INVALID, "max_prefix_len"), (dict(c=cache(Dh=96)), UNSUPPORTED, "Dh=96"),
                               (dict(Hq=7), UNSUPPORTED, "multiple"), (dict(Hq=258), UNSUPPORTED, "above 128")]:
        assert call(**change) == code and text in said(lib), (change, said(lib))


def test_what_else_is_refused(lib):
    c = calls(lib)
    for name, change, code, text in [
            ("store", dict(o=view(sh=0)), INVALID, "q_out: strides"), ("store", dict(k=view(data=0)), INVALID, "k is NULL"), ("store", dict(v=view(st=3)), INVALID, "v: strides"),
            ("store", dict(pairs=65), INVALID, "pairs=65"), ("store", dict(pairs=-1), INVALID, "pairs"), ("store", dict(axes=0), INVALID, "axes"), ("store", dict(axes=9), INVALID, "axes"),
            ("store", dict(pos=None), INVALID, "pos"), ("store", dict(freq=None), INVALID, "inv_freq"), ("store", dict(base=P + 1), INVALID, "misaligned"),
            ("store", dict(q=view(sh=256)), INVALID, "in place"), ("store", dict(o=view(st=8192)), INVALID, "in place"),
            ("attend", dict(o=view(st=0)), INVALID, "out: strides"), ("attend", dict(lse=P + 1), INVALID, "out_lse"), ("attend", dict(ws=None), INVALID, "workspace"),
            ("attend", dict(ws=P + 8), INVALID, "workspace"), ("attend", dict(nb=1000), WORKSPACE, "smaller"),
            ("weigh", dict(lse=None), INVALID, "lse"), ("weigh", dict(w=None), INVALID, "weights"), ("weigh", dict(prior=P + 2), INVALID, "misaligned"),
            ("weigh", dict(decay=float("nan")), INVALID, "decay"), ("weigh", dict(decay=1.5), INVALID, "decay"), ("weigh", dict(sh=309), INVALID, "strides"), ("weigh", dict(sb=0), INVALID, "strides"),
            ("evict", dict(n=None), INVALID, "NULL"), ("evict", dict(w=None), INVALID, "NULL"), ("evict", dict(kept=None), INVALID, "NULL"), ("evict", dict(new=P), INVALID, "new_len"),
            ("evict", dict(budget=0), INVALID, "budget=0"), ("evict", dict(sink=60, recent=41), INVALID, "n_sink"), ("evict", dict(sink=-1), INVALID, "n_sink"),
            ("evict", dict(most=-1), INVALID, "max_len"), ("evict", dict(sh=299), INVALID, "stride"), ("evict", dict(nw=P, nsb=640, nsh=99), INVALID, "stride"),
            ("evict", dict(nw=P, nsb=6400, nsh=320), INVALID, "one set of strides"), ("evict", dict(dst=cache(Dh=64, page_table=P + 16)), INVALID, "dst must have"),
            ("evict", dict(dst=cache(max_pages=6, page_table=P + 16)), INVALID, "dst holds 96"), ("evict", dict(dst=cache(page_size=8, max_pages=40)), INVALID, "same cache"),
            ("evict", dict(dst=cache(B=0)), INVALID, "dst: B=0"),
            ("compact", dict(N=0), INVALID, "N=0"), ("compact", dict(N=257), INVALID, "N=257"), ("compact", dict(path=None), INVALID, "NULL"), ("compact", dict(new=P), INVALID, "new_prefix_len"),
            ("compact", dict(w=P, sh=319), INVALID, "strides"), ("compact", dict(w=P, rows=-1), INVALID, "rows")]:
        assert c[name](**change) == code and text in said(lib), (name, change, said(lib))


def test_workspace_sizes(lib):
    size = lib.talon_paged_attention_workspace_bytes
    assert size(1, 1, 32, 8, 128, 700) == 256 and size(1, 60, 32, 8, 128, 100) == 256                   # nothing is cut
    assert 0 < size(1, 1, 32, 8, 128, 2048) < size(1, 64, 32, 8, 128, 2048) <= size(64, 2048, 32, 8, 128, 8192) < 80 << 20
    for bad in [(0, 1, 8, 8, 128, 0), (1, 0, 8, 8, 128, 0), (1, 1, 8, 0, 128, 0), (1, 1, 0, 8, 128, 0), (1, 1, 8, 8, 96, 0), (1, 1, 8, 8, 128, -1), (1, 1, 9, 8, 128, 0),
                (256, 65536, 128, 1, 128, 1 << 30)]:
        assert size(*bad) == 0
        with pytest.raises(T.TalonError):
            T.talon_paged_attention_workspace_bytes(*bad)


# ---------------------------------------------------------------------------------- the binding
def small(dtype=torch.bfloat16, B=2, Hkv=2, Dh=64):
    k = torch.zeros(8, 16, Hkv, Dh, dtype=dtype)
    return T.PagedCache(k, torch.zeros_like(k), torch.zeros(B, 4, dtype=torch.int32))


def refused(code, text, call):
    with pytest.raises(T.TalonError) as e:
        call()
    assert e.value.code == code and text in str(e.value), str(e.value)


def test_handles_that_are_refused():
    k, t = torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 4, dtype=torch.int32)
    refused(INVALID, "one type", lambda: T.PagedCache(k, k.half(), t))
    refused(INVALID, "one set of strides", lambda: T.PagedCache(k, torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16).transpose(1, 2), t))
    refused(INVALID, "one set", lambda: T.PagedCache(k[0], k[0], t))
    refused(INVALID, "contiguous", lambda: T.PagedCache(k[..., ::2], k[..., ::2], t))
    refused(UNSUPPORTED, "float32", lambda: T.PagedCache(k.float(), k.float(), t))
    refused(INVALID, "page_table", lambda: T.PagedCache(k, k, t.long()))
    refused(INVALID, "page_table", lambda: T.PagedCache(k, k, t[:, ::2]))
    refused(INVALID, "status", lambda: T.PagedCache(k, k, t, torch.zeros(3, dtype=torch.int32)))


def test_tensors_that_are_refused():
    c = small()
    q = torch.zeros(2, 10, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(2, 10, 2, 64, dtype=torch.bfloat16)
    n, p = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pos, freq, lse, w = torch.zeros(1, 2, 10, dtype=torch.int32), torch.zeros(32), torch.zeros(2, 10, 4), torch.zeros(2, 2, 64)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    attend = lambda c=c, q=q, n=n, p=p, o=q, lse=lse, ws=ws, **kw: T.talon_paged_attention(c, q, n, p, 30, o, lse, ws, stream=0, **kw)
    refused(INVALID, "on the current GPU", attend)                # everything else is right: host memory is refused
    refused(INVALID, "q must be torch.bfloat16", lambda: attend(q=q.half()))
    refused(INVALID, "q must be torch.float16", lambda: attend(c=small(torch.float16)))
    refused(INVALID, "q has another shape", lambda: attend(q=q[:1]))
    refused(INVALID, "q has another shape", lambda: attend(q=q[0]))
    refused(INVALID, "q has another shape", lambda: attend(q=torch.zeros(2, 10, 4, 128, dtype=torch.bfloat16)))
    refused(INVALID, "contiguous heads", lambda: attend(q=torch.zeros(2, 10, 64, 4, dtype=torch.bfloat16).transpose(2, 3)))
    refused(INVALID, "out has another shape", lambda: attend(o=q[:, :9]))
    refused(INVALID, "out is None", lambda: attend(o=None))
    refused(INVALID, "n_new must be torch.int32", lambda: attend(n=n.long()))
    refused(INVALID, "n_new has another shape", lambda: attend(n=torch.zeros(3, dtype=torch.int32)))
    refused(INVALID, "prefix_len must be contiguous", lambda: attend(p=torch.zeros(4, dtype=torch.int32)[::2]))
    refused(INVALID, "out_lse", lambda: attend(lse=lse[:, :, :2]))
    refused(INVALID, "out_lse must be torch.float32", lambda: attend(lse=lse.double()))
    refused(INVALID, "mask", lambda: attend(mask=torch.zeros(2, 10, 2, dtype=torch.int64)))
    refused(INVALID, "mask must be torch.int64", lambda: attend(mask=torch.zeros(2, 10, 1, dtype=torch.bool)))
    refused(INVALID, "offset", lambda: attend(offset=torch.zeros(2, 9, dtype=torch.int32)))
    refused(INVALID, "slopes", lambda: attend(slopes=torch.zeros(3)))
    for bad in (lambda: attend(c=object()), lambda: attend(window="x"), lambda: attend(softcap="x"), lambda: attend(window=1.5)):
        with pytest.raises((TypeError, AttributeError)):
            bad()
    st = T.TreeState(2, 10, device="cpu")
    with pytest.raises(TypeError):                                # a struct of another kind
        st.get_device = lambda: 0
        T.talon_paged_attention(st, q, n, p, 30, q, lse, ws, stream=0)
    store = lambda q=q, k=kv, v=kv, o=q, pos=pos, freq=freq, **kw: T.talon_rotary_store(c, q, k, v, o, n, p, pos, freq, stream=0, **kw)
    refused(INVALID, "on the current GPU", store)
    refused(INVALID, "k has another shape", lambda: store(k=kv[:, :, :1]))
    refused(INVALID, "v has another shape", lambda: store(v=kv[:, :9]))
    refused(INVALID, "pos must be torch.int32", lambda: store(pos=pos.long()))
    refused(INVALID, "pos has another shape", lambda: store(pos=pos[0]))
    refused(INVALID, "inv_freq must be torch.float32", lambda: store(freq=freq.double()))
    refused(INVALID, "pair_axis has another shape", lambda: store(pair_axis=torch.zeros(31, dtype=torch.int32)))
    refused(INVALID, "pos_base", lambda: store(pos_base=torch.zeros(1, dtype=torch.int32)))
    weigh = lambda lse=lse, w=w, prior=None, **kw: T.talon_paged_weights(c, q, n, p, 30, lse, w, prior=prior, stream=0, **kw)
    refused(INVALID, "on the current GPU", weigh)
    refused(INVALID, "lse is None", lambda: weigh(lse=None))
    refused(INVALID, "weights has fewer rows", lambda: weigh(w=w[:, :, :39]))
    refused(INVALID, "prior must have the strides", lambda: weigh(prior=torch.zeros(2, 2, 65)))
    refused(INVALID, "weights must have contiguous rows", lambda: weigh(w=torch.zeros(2, 64, 2).transpose(1, 2)))
    kept, new = torch.zeros(2, 2, 20, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    evict = lambda kept=kept, new=new, w=w, budget=20, **kw: T.talon_paged_evict(c, n, 64, w, budget, kept, new, stream=0, **kw)
    refused(INVALID, "on the current GPU", evict)
    refused(INVALID, "kept has another shape", lambda: evict(budget=21))
    refused(INVALID, "kept must be contiguous", lambda: evict(kept=torch.zeros(2, 2, 40, dtype=torch.int32)[:, :, ::2]))
    refused(INVALID, "weights has fewer rows", lambda: evict(w=w[:, :, :63]))
    refused(INVALID, "new_weights has fewer rows", lambda: evict(new_weights=w[:, :, :19]))
    path = torch.zeros(2, 10, dtype=torch.int32)
    compact = lambda path=path, new=new, **kw: T.talon_paged_compact(c, path, n, p, new, stream=0, **kw)
    refused(INVALID, "on the current GPU", compact)
    refused(INVALID, "path must be torch.int32", lambda: compact(path=path.long()))
    refused(INVALID, "weights must have contiguous rows", lambda: compact(weights=torch.zeros(2, 64, 2).transpose(1, 2)))


# ---------------------------------------------------------------------------------- the launch plan
def test_plans_stay_within_what_the_kernels_assume(tmp_path):
    """paged_plan over a grid of shapes, in a small C++ program."""
    src = tmp_path / "plan.cpp"
    src.write_text(r'''
#include "paged_plan.h"
#include <stdio.h>
using namespace talon;
int main() {
  int bad = 0, count = 0;
  const int Bs[] = {1, 3, 64, 256}, Ns[] = {1, 2, 60, 64, 257, 2048, 65536}, Gs[] = {1, 3, 8, 48, 128}, Hs[] = {1, 8, 128}, Ds[] = {64, 128, 256},
            Ls[] = {0, 1, 63, 192, 255, 2048, 100000, 1 << 30};
  for (int B : Bs) for (int N : Ns) for (int G : Gs) for (int H : Hs) for (int D : Ds) for (int L : Ls) {
    const PagedPlan p = paged_plan(B, N, G * H, H, D, L);
    if (p.tiles >= 1ll << 30) continue;                       // refused
    ++count;
    const long long rows = (long long)N * G, tile = p.waves ? 32 * p.waves : 32, keys = p.waves ? 64 : 32, items = (long long)B * H * ((rows + tile - 1) / tile);
    const long long most = ((long long)L + N + keys - 1) / keys;
    bool ok = p.slots >= 1 && (p.waves == 4 || p.waves == 8 || (p.waves == 0 && rows <= 32)) && (D != 256 || p.waves != 8) && p.rows_slot <= tile && p.rows_slot <= rows;
    if (p.split) {
      long long share = (p.tiles + p.slots - 1) / p.slots;
      if (share < p.least) share = p.least;  // (p.tiles: with what row tiles cost besides)
      ok = ok && share * p.slots >= p.tiles && p.tiles + share < 1ll << 31;                    // all tiles have a share, in 32 bits
      ok = ok && (long long)p.slots < (1 << 30);                                                // the last share and a slot's bit lie in one word
      ok = ok && p.off_m >= 2ull * p.slots * p.rows_slot * D * 4 && p.off_l - p.off_m >= 2ull * p.slots * p.rows_slot * 4 &&
           p.off_cut - p.off_l >= 2ull * p.slots * p.rows_slot * 4 && p.bytes - p.off_cut >= 16ull * p.slots && p.off_m % 16 == 0 && p.off_cut % 16 == 0;
    } else {
      ok = ok && p.slots == items && most <= (p.waves ? kPagedWholeTiles : kPagedFewWhole);
    }
    if (!ok) { ++bad; printf("B=%d N=%d G=%d H=%d D=%d L=%d\n", B, N, G, H, D, L); }
  }
  printf("%d plans, %d bad\n", count, bad);
  return bad != 0 || count < 1000;
}
''')
    exe = tmp_path / "plan"
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-I", B.CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
