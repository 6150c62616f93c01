// What the calls on a paged cache share (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "talon.h"

namespace talon {

// The cache as kernels see it.  Rows are addressed in 16-byte chunks with 32-bit numbers: a tensor of up to 64 GiB (the ABI
// layer refuses larger ones), one 64-bit addition per address.
struct PagedRows {
  void* k;
  void* v;
  const int32_t* table;      // [B][max_pages]
  uint32_t* status;          // [B]
  int max_pages;
  uint32_t num_pages;
  int page_shift;            // page_size = 1 << page_shift
  int capacity;              // rows a sequence can have
  uint32_t page_chunks, token_chunks, head_chunks;   // strides in 16-byte chunks
};

struct RowsView {            // [B][N][H][Dh] of a caller's tensor, strides in elements
  uint16_t* p;
  int64_t sb, st, sh;
};

// Caps up to here are formed by one exponential and a reciprocal in attention (cap - 2 cap / (1 + e^(2x))), which is off by 2^-22 of
// the cap near a score of 0: 2^-16 at most, a 32nd of the half step that a probability is rounded by in fp16, and no more than four times the
// spacing of fp32 numbers near the cap.  Larger ones have kernels of their own, with tanh_of(): a chunk of
// 2048 tokens at 8192 rows, 32/8 heads of 128, 652 us against 394, 4 trees of 128 nodes 78 against 56, 8 tokens at 8192 rows 52.6 against 50.8.
constexpr float kNearCap = 64.f;

// What decides a score besides the product (attention and its weights alike).
struct ScoreArgs {
  const int32_t* n_new;      // [B]
  const int32_t* prefix_len; // [B]
  const uint64_t* mask;      // [B][N][words] or NULL: causal
  const int32_t* offset;     // [B][N] or NULL
  const float* slopes;       // [Hq] or NULL
  int N, words, max_prefix_len, window;
  float scale_log2e;         // scale * log2(e)
  float cap_log2e;           // cap * log2(e); 0: none
  float cap_in;              // with x = scale * product / cap: 2 x log2(e) / product in attention up to kNearCap, else x / product
};

struct PagedAttnArgs {
  PagedRows c;
  ScoreArgs sc;
  RowsView q, out;
  float* lse;                // [B][N][Hq] or NULL (written by attention, read by the weights)
  int B, Hkv, G;
  uint32_t inv_g;            // ceil(2^32 / G)
  int split;                 // 1: shares of the line of key tiles; 0: a row tile per workgroup
  int slots;                 // most workgroups that take a share of the key tiles
  int least;                 // fewest key tiles of a share
  int extra;                 // what a row tile costs besides its key tiles, in tiles
  int rows_slot;             // rows of a partial result
  float* part_o;             // [2 * slots][Dh / 8][rows_slot][8]
  float* part_m;             // [2 * slots][rows_slot]
  float* part_l;
  int4* cut;                 // [slots] the row tile that a share's end cuts, see paged_attention.h; NULL: nothing is joined
};

// Weights of many queries: rows of the cache of a workgroup, and its threads.
constexpr int kWeighRows = 64, kWeighThreads = 512;

struct PagedWeightArgs {
  PagedAttnArgs a;           // cache, scores, queries, lse (read), shares
  const float* prior;        // or NULL
  float* out;
  int64_t stride_b, stride_h;
  float decay;
};

struct RotaryArgs {
  PagedRows c;
  RowsView q, k, v, q_out;
  const int32_t* n_new;
  const int32_t* prefix_len;
  const int32_t* pos;        // [axes][B][N]
  const int32_t* base;       // [B] or NULL
  const int32_t* axis;       // [pairs] or NULL
  const float* inv_freq;     // [pairs]
  int B, N, Hq, Hkv, Dh, pairs, axes, interleaved;
  int units;                 // pieces of a head (set by the launch)
  uint32_t inv_units;        // ceil(2^32 / units), 0 for 1
};

struct EvictArgs {
  PagedRows src, dst;
  const int32_t* len;        // [B]
  int32_t* new_len;          // [B]
  const float* weights;
  float* new_weights;
  int64_t stride_b, stride_h, new_stride_b, new_stride_h;
  int32_t* kept;             // [B][Hkv][budget]
  int B, Hkv, Dh, budget, n_sink, n_recent, max_len;
  int in_place;
};

struct CompactArgs {
  PagedRows c;
  const int32_t* path;       // [B][N]
  const int32_t* accept_len;
  const int32_t* prefix_len;
  int32_t* new_prefix_len;
  float* weights;            // or NULL
  int64_t stride_b, stride_h;
  int weight_rows;
  int B, N, Hkv, Dh;
};

hipError_t launch_paged_attention_bf16_64(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_bf16_128(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_bf16_256(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_f16_64(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_f16_128(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_f16_256(const PagedAttnArgs& a, int waves, hipStream_t s);
hipError_t launch_paged_attention_bf16_far(const PagedAttnArgs& a, int Dh, int waves, hipStream_t s);   // caps above kNearCap
hipError_t launch_paged_attention_f16_far(const PagedAttnArgs& a, int Dh, int waves, hipStream_t s);
hipError_t launch_paged_weights_bf16(const PagedWeightArgs& wa, int Dh, bool few, hipStream_t s);
hipError_t launch_paged_weights_f16(const PagedWeightArgs& wa, int Dh, bool few, hipStream_t s);
hipError_t launch_rotary_store(const RotaryArgs& a, int dtype, hipStream_t s);
hipError_t launch_paged_evict(const EvictArgs& a, hipStream_t s);
hipError_t launch_paged_compact(const CompactArgs& a, hipStream_t s);

}  // namespace talon
