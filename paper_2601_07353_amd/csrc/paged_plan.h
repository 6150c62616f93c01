// Launch plan of attention over a paged cache.  Host code without HIP, so that tests can evaluate it on a machine without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace talon {

struct PagedPlan {
  int waves;        // wavefronts per workgroup that has rows for each; 0: few rows, the wavefronts share the keys
  int split;        // 1: row tiles are cut into shares; 0: a workgroup per row tile, nothing to join
  int slots;        // workgroups
  int least;        // fewest key tiles of a share
  int extra;        // what a row tile costs besides its key tiles, in tiles
  int rows_slot;    // rows of a partial result
  long long tiles;  // key tiles of the call if every sequence is as long as it may be
  size_t off_m, off_l, off_cut, bytes;   // workspace: outputs, maxima, denominators, cuts
};

constexpr int kPagedTile = 64;
constexpr int kPagedWholeTiles = 4;   // up to so many key tiles a row tile is not cut
constexpr int kPagedLeast = 2;        // fewest key tiles of a share
constexpr int kPagedFewTile = 32;     // the same for few rows
constexpr int kPagedFewWhole = 24;
constexpr int kPagedFewLeast = 8;
constexpr int kPagedPieces = 24;
constexpr int kPagedExtra = 5;
constexpr int kPagedFewExtra = 8;
constexpr int kWeighExtra = 4;

inline PagedPlan paged_plan(int B, int N, int Hq, int Hkv, int Dh, int max_prefix_len) {
  PagedPlan p = {};
  const long long rows = static_cast<long long>(N) * (Hq / Hkv);
  const bool few = rows <= 32;
  p.waves = few ? 0 : (Dh != 256 && rows >= 512 ? 8 : 4);
  const int row_tile = few ? 32 : 32 * p.waves;
  const int tile = few ? kPagedFewTile : kPagedTile;
  const long long items = static_cast<long long>(B) * Hkv * ((rows + row_tile - 1) / row_tile);
  const long long most = (static_cast<long long>(max_prefix_len) + N + tile - 1) / tile;
  p.extra = few ? kPagedFewExtra : kPagedExtra;
  p.tiles = items * (most + p.extra);
  p.rows_slot = static_cast<int>(rows < row_tile ? rows : row_tile);
  p.split = most > (few ? kPagedFewWhole : kPagedWholeTiles) ? 1 : 0;
  if (!p.split) {
    p.slots = static_cast<int>(items < (1ll << 30) ? items : (1ll << 30));
    p.least = 1;
    p.bytes = 256;   // nothing is staged, keep a token size
    return p;
  }
  const long long slots = few ? (Dh == 64 ? 512 : 256) : (p.waves == 8 || Dh == 256 ? 256 : 512);   // workgroups that the device holds at once
  // Few row tiles: as many pieces of each as there are workgroups for, up to what the join reads in three rounds.
  p.least = few ? kPagedFewLeast : kPagedLeast;
  if (items * 8 <= slots) {
    const long long pieces = slots / items < kPagedPieces ? slots / items : kPagedPieces;
    const long long even = (most + pieces - 1) / pieces;
    p.least = static_cast<int>(even > p.least ? even : p.least);
  }
  const long long enough = (p.tiles + p.least - 1) / p.least + items;   // (also as even pieces of the row tiles)
  p.slots = static_cast<int>(enough < slots ? enough : slots);
  const size_t slot_rows = 2 * static_cast<size_t>(p.slots) * p.rows_slot;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.off_m = up(slot_rows * Dh * sizeof(float));
  p.off_l = p.off_m + up(slot_rows * sizeof(float));
  p.off_cut = p.off_l + up(slot_rows * sizeof(float));
  p.bytes = p.off_cut + up(static_cast<size_t>(p.slots) * 16);
  return p;
}

// Attention weights of few queries: the same shares, of all rows of the sequences.
struct WeighPlan {
  int slots, least, extra;
  long long tiles;
};
inline WeighPlan weigh_plan(int B, int Hkv, int Dh, int rows) {
  WeighPlan p = {};
  const long long items = static_cast<long long>(B) * Hkv, most = (static_cast<long long>(rows) + kPagedFewTile - 1) / kPagedFewTile;
  p.least = kPagedFewLeast;
  p.extra = kWeighExtra;
  p.tiles = items * (most + p.extra);
  const long long slots = Dh == 64 ? 512 : 256, enough = (p.tiles + p.least - 1) / p.least + items;
  p.slots = static_cast<int>(enough < slots ? enough : slots);
  return p;
}

}  // namespace talon
