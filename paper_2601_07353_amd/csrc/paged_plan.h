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
  size_t room;      // a workspace that holds this plan and the plans of all shorter prefixes
};

// Which kernel, and how the key tiles of all row tiles are cut into shares (times in us, bf16, heads of 128, 32/8 heads where not
// said otherwise, P rows in the cache):
//   few rows    up to 32 (token, head) rows of a KV head: the wavefronts of a workgroup share the keys of one row tile.  The other
//               kernel, a row tile of 32 rows per wavefront, would leave three quarters of a workgroup without rows.
//   wavefronts  8 from 512 rows on (a K/V tile is read once for 256 rows): a chunk of 2048 512 against 538 with 4, 4 trees of 128
//               nodes 59 against 64; 60 nodes (240 rows) 26.7 against 24.5.  Heads of 256 have registers for 4 only.
//   whole       prefixes of at most that many key tiles are not cut: few rows, 1 x 1000 rows cut 13.2 whole 14.6, but 8 x 1024
//               18.5 and 17.4, and 500 rows 11.2 whole.
//   least       key tiles that a share has at least; a tree of 60 nodes at P = 2048: 2 24.5, 4 22.5, 8 26.3 (few sequences get
//               even pieces instead, below).
//   pieces      most even pieces of a row tile when there are few: one token at P = 2048 8 15.8, 16 14.9, 24 14.7, 32 14.8; at
//               P = 8192 22.3, 20.9, 19.8, 20.7; at P = 32768 62, 43, 39.3, 38.8.
//   extra       what a row tile costs besides its tiles (queries, last stores, partial results), in tiles: 2048 tokens 0 488, 4 479,
//               6 471; 4 trees 65.6, 56, 57.8; few rows, 64 sequences of up to 1024 rows 0 59.3, 4 51, 8 47.1, 16 45.5, and 32 of 4
//               tokens at P = 2048 52, 48.9, 47.7, 49.3.  Attention weights join nothing: half of that.
constexpr int kPagedTile = 64;
constexpr int kPagedWholeTiles = 4;
constexpr int kPagedLeast = 2;
constexpr int kPagedExtra = 5;
constexpr int kPagedFewTile = 32;
constexpr int kPagedFewWhole = 24;
constexpr int kPagedFewLeast = 8;
constexpr int kPagedFewExtra = 8;
constexpr int kPagedPieces = 24;
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
    p.bytes = p.room = 256;   // nothing is staged, keep a token size
    return p;
  }
  const long long slots = few ? 256 : (p.waves == 8 || Dh == 256 ? 256 : 512);   // workgroups that the device holds at once
  // Few row tiles (an eighth of the workgroups): even pieces of each, as many as there are workgroups for, up to what the join reads in
  // three rounds; 8 ragged sequences of up to 8192 rows (a quarter) are better off in equal shares, 45.8 against 50.4.
  const int base = few ? kPagedFewLeast : kPagedLeast;
  p.least = base;
  // Longer prefixes do not always take more workgroups: even pieces get larger, and what a row tile costs besides its tiles (`extra`)
  // weighs less.  With least >= base the number `enough` below is at most what `base` gives, which grows with the
  // prefix; with least >= most / pieces it is at most items * (pieces + extra / base + 1), whatever the prefix.
  long long bound = (p.tiles + base - 1) / base + items;
  if (items * 8 <= slots) {
    const long long pieces = slots / items < kPagedPieces ? slots / items : kPagedPieces;
    const long long even_bound = items * (pieces + (p.extra + base - 1) / base + 1);
    bound = bound < even_bound ? bound : even_bound;
    const long long even = (most + pieces - 1) / pieces;
    p.least = static_cast<int>(even > p.least ? even : p.least);
  }
  const long long enough = (p.tiles + p.least - 1) / p.least + items;   // (also as even pieces of the row tiles)
  p.slots = static_cast<int>(enough < slots ? enough : slots);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  auto lay_out = [&](long long n) {   // of n workgroups
    const size_t slot_rows = 2 * static_cast<size_t>(n) * p.rows_slot;
    p.off_m = up(slot_rows * Dh * sizeof(float));
    p.off_l = p.off_m + up(slot_rows * sizeof(float));
    p.off_cut = p.off_l + up(slot_rows * sizeof(float));
    return p.off_cut + up(static_cast<size_t>(n) * 16);
  };
  p.room = lay_out(bound < slots ? bound : slots);
  p.bytes = lay_out(p.slots);
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
  const long long slots = 256, enough = (p.tiles + p.least - 1) / p.least + items;
  p.slots = static_cast<int>(enough < slots ? enough : slots);
  return p;
}

}  // namespace talon
