"""The scratch memory of talon_paged_attention: what the size query returns holds for the call of the same arguments, whatever the page
table's capacity, and for every call with shorter prefixes.  (No GPU: the sizes that a call needs are read from its refusal of none.)"""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2601_07353_amd as T
from paper_2601_07353_amd import build as B
from paper_2601_07353_amd.binding import _CPagedCache, _CView

P = 0x7000000
# (B, N, Hq, Hkv, Dh): one token, drafts, trees, chunks; few row tiles, where a longer prefix is cut into larger pieces, and many
SHAPES = [(1, 1, 32, 8, 128), (1, 1, 8, 1, 64), (1, 3, 32, 8, 128), (2, 8, 16, 4, 256), (1, 16, 32, 8, 128), (1, 60, 32, 8, 128), (1, 64, 32, 8, 128), (3, 33, 12, 4, 64),
          (1, 100, 4, 2, 256), (1, 256, 32, 8, 128), (1, 600, 8, 8, 64), (8, 1, 32, 8, 128), (16, 256, 32, 8, 128), (64, 1, 64, 8, 128), (2, 2048, 32, 8, 128)]
LENGTHS = sorted({0, 63, 100, 700, 769, 1000, 2047, 2048, 2945, 4096, 6112, 6400, 8192, 8193, 12345, 16384, 32768, 50000, 131072} | set(range(256, 8192, 416)))


def needed(lib, shape, most, capacity):
    """Bytes that the call asks for (0: it needs no workspace), with a page table of `capacity` rows."""
    b, n, hq, hkv, dh = shape
    c = _CPagedCache(b, hkv, dh, 1, 64, 16, capacity // 16, 16 * hkv * dh, hkv * dh, dh, P, P + 0x1000000, P + 4, P + 8)
    v = _CView(P, n * hq * dh, hq * dh, dh)
    if T.talon_paged_attention_workspace_bytes(b, n, hq, hkv, dh, min(most, capacity)) == 256:
        return 0                                                  # (nothing is cut; nothing to refuse)
    rc = lib.talon_paged_attention(ctypes.byref(c), ctypes.byref(v), n, hq, P, P, most, None, ctypes.byref(v), None, P, 0, None)
    assert rc == T.TALON_ERR_WORKSPACE
    return int(re.search(r"smaller than the (\d+) needed", lib.talon_last_error_string().decode()).group(1))


@pytest.mark.parametrize("shape", SHAPES)
def test_a_workspace_of_the_size_asked_for_serves_any_table(shape):
    lib = T.load_library()
    for most in LENGTHS:
        asked = T.talon_paged_attention_workspace_bytes(*shape, most)
        for capacity in (16, 272, 2944, 4096, 6112, 1 << 20):
            assert needed(lib, shape, most, capacity) <= asked, (most, capacity)


@pytest.mark.parametrize("shape", SHAPES)
def test_a_workspace_for_the_longest_prefix_serves_shorter_ones(shape):
    lib = T.load_library()
    asked = [T.talon_paged_attention_workspace_bytes(*shape, most) for most in LENGTHS]
    assert asked == sorted(asked)
    need = [needed(lib, shape, most, 1 << 20) for most in LENGTHS]
    for i, have in enumerate(asked):
        assert max(need[:i + 1]) <= have, LENGTHS[i]
    assert max(asked) < 80 << 20                                  # still a fixed amount, whatever the lengths


def test_every_shorter_prefix_over_a_grid_of_plans(tmp_path):
    """The same of the plan itself, for every number of key tiles up to 2000."""
    src = tmp_path / "room.cpp"
    src.write_text(r'''
#include "paged_plan.h"
#include <stdio.h>
using namespace talon;
int main() {
  int bad = 0, count = 0;
  const int Bs[] = {1, 2, 5, 64}, Ns[] = {1, 7, 33, 60, 64, 129, 600, 2048}, Gs[] = {1, 4, 5, 8, 40}, Hs[] = {1, 2, 8}, Ds[] = {64, 128, 256};
  for (int B : Bs) for (int N : Ns) for (int G : Gs) for (int H : Hs) for (int D : Ds) {
    size_t most = 0, before = 0;
    for (int t = 0; t <= 2000; ++t) {
      const PagedPlan p = paged_plan(B, N, G * H, H, D, 31 * t);
      most = p.bytes > most ? p.bytes : most;
      ++count;
      if (p.room < most || p.room < before) {
        if (++bad < 10) printf("B=%d N=%d G=%d H=%d D=%d L=%d: %zu of %zu\n", B, N, G, H, D, 31 * t, p.room, most);
      }
      before = p.room;
    }
  }
  printf("%d plans, %d bad\n", count, bad);
  return bad != 0;
}
''')
    exe = tmp_path / "room"
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-I", B.CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
