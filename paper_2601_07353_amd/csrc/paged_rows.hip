// Rows of a paged cache: written with rotated keys, moved behind the prefix, dropped and moved together.  All of it is
// bound by the bytes that it moves.
#include "paged_device.h"

namespace talon {

namespace {

__device__ __forceinline__ float to_float(uint16_t v, bool f16) {
  if (f16) return static_cast<float>(__builtin_bit_cast(_Float16, v));
  return __uint_as_float(static_cast<uint32_t>(v) << 16);
}
__device__ __forceinline__ uint16_t from_float(float v, bool f16) {
  if (f16) return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

union Chunk {
  uint4 v;
  uint16_t e[8];
};

// ---- rotary positions and the write into the pages.
// angle(token, f) = (base + pos[axis(f)][token]) * inv_freq[f];  (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin)
// A workgroup takes a token.  The angles' sines and cosines, one f per thread, go to LDS: the product and its
// reduction to one turn are formed in 64 bits (a position of 10^5 in fp32 has lost 2^-8 of a turn), the rest in fp32.  The heads'
// values are two chunks of 16 bytes per thread: the eight first and the eight second values of eight pairs, so that a
// value is read and written by one thread and q may be rotated in place; values that are copied go the same way.  A thread's
// first AHEAD units are on their way while it finds its angles.
// Bound: the bytes (a token's latency when there are few): 4 sequences of up to 2048 tokens, 32/8 heads of 128, interleaved pairs,
// 34 us (4.3 TB/s).  Neighbouring threads have neighbouring chunks (a thread's pairs side by side: 39 us), two units are ahead (one:
// 35, three: 38), and a token per workgroup is as fast as four with many and faster with few (1024 tokens 7.6 us against 10.6).
template <bool F16>
__global__ __launch_bounds__(256) void rotary_store_kernel(RotaryArgs a) {
  extern __shared__ float2 s_turn[];   // [pairs] cosine, sine
  constexpr int AHEAD = 2;
  const int b = blockIdx.y;
  const int i = blockIdx.x;
  const int tid = threadIdx.x;
  int P, n;
  clamped_lengths(a.c, a.prefix_len[b], a.n_new[b], a.c.capacity, a.N, &P, &n);
  if (blockIdx.x == 0 && tid == 0) {
    const int want = a.n_new[b] < a.N ? a.n_new[b] : a.N;
    if (want > n) report(a.c, b, TALON_STATUS_BAD_PAGE);   // rows beyond the page table are not written
  }
  if (i >= n) return;
  // units of a head: groups of eight pairs, then of sixteen values that are copied
  const bool whole = a.pairs % 8 == 0;           // (else value by value)
  const int groups = (a.pairs + 7) / 8;
  const int all = (a.Hq + 2 * a.Hkv) * a.units;

  struct Unit {
    uint4 c1, c2;
    const uint16_t* src;
    uint16_t* dst;     // nullptr: nothing to do
    int unit, one, two;
    bool is_v;
  };
  auto fetch = [&](int x) {
    Unit r;
    int head = a.inv_units != 0u ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), a.inv_units)) : x;
    r.unit = x - head * a.units;
    r.dst = nullptr;
    r.src = nullptr;
    r.is_v = false;
    r.one = r.two = 0;
    r.c1 = r.c2 = make_uint4(0, 0, 0, 0);
    if (x >= all) return r;
    const bool is_q = head < a.Hq;
    if (!is_q) head -= a.Hq;
    r.is_v = !is_q && head >= a.Hkv;
    if (r.is_v) head -= a.Hkv;
    const RowsView& from = is_q ? a.q : (r.is_v ? a.v : a.k);
    r.src = from.p + static_cast<int64_t>(b) * from.sb + static_cast<int64_t>(i) * from.st + static_cast<int64_t>(head) * from.sh;
    // (neighbouring threads have neighbouring chunks, also of interleaved pairs, of which a chunk holds four)
    r.one = r.unit < groups ? 8 * r.unit : 2 * a.pairs + 8 * (r.unit - groups);
    r.two = r.unit < groups ? a.pairs + 8 * r.unit : r.one + 8 * (a.units - groups);   // (beyond the head: only `one`)
    uint32_t entry = 0;
    if (!is_q) entry = page_entry(a.c, b, P + i);
    if (whole) {
      r.c1 = *reinterpret_cast<const uint4*>(r.src + r.one);
      if (r.two < a.Dh) r.c2 = *reinterpret_cast<const uint4*>(r.src + r.two);
    }
    if (is_q) {
      r.dst = a.q_out.p + static_cast<int64_t>(b) * a.q_out.sb + static_cast<int64_t>(i) * a.q_out.st + static_cast<int64_t>(head) * a.q_out.sh;
    } else if (entry < a.c.num_pages) {
      r.dst = chunk_at(static_cast<uint16_t*>(r.is_v ? a.c.v : a.c.k), row_chunk(a.c, entry, P + i, head));
    } else {
      report(a.c, b, TALON_STATUS_BAD_PAGE);   // nowhere to write to
    }
    return r;
  };
  auto finish = [&](const Unit& r) {
    if (r.dst == nullptr) return;
    const bool turned = !r.is_v && r.unit < groups;
    if (whole) {
      Chunk c1, c2, r1, r2;
      c1.v = r.c1;
      c2.v = r.c2;
      r1.v = r.c1;
      r2.v = r.c2;
      if (turned && a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t1 = s_turn[4 * r.unit + e], t2 = s_turn[4 * (groups + r.unit) + e];
          const float x1 = to_float(c1.e[2 * e], F16), y1 = to_float(c1.e[2 * e + 1], F16);
          const float x2 = to_float(c2.e[2 * e], F16), y2 = to_float(c2.e[2 * e + 1], F16);
          r1.e[2 * e] = from_float(x1 * t1.x - y1 * t1.y, F16);
          r1.e[2 * e + 1] = from_float(y1 * t1.x + x1 * t1.y, F16);
          r2.e[2 * e] = from_float(x2 * t2.x - y2 * t2.y, F16);
          r2.e[2 * e + 1] = from_float(y2 * t2.x + x2 * t2.y, F16);
        }
      } else if (turned) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 t1 = s_turn[8 * r.unit + e];
          const float x1 = to_float(c1.e[e], F16), y1 = to_float(c2.e[e], F16);
          r1.e[e] = from_float(x1 * t1.x - y1 * t1.y, F16);
          r2.e[e] = from_float(y1 * t1.x + x1 * t1.y, F16);
        }
      }
      *reinterpret_cast<uint4*>(r.dst + r.one) = r1.v;
      if (r.two < a.Dh) *reinterpret_cast<uint4*>(r.dst + r.two) = r2.v;
    } else if (r.unit < groups) {
      for (int e = 0; e < 8 && 8 * r.unit + e < a.pairs; ++e) {
        const int f = 8 * r.unit + e;
        const int one = a.interleaved ? 2 * f : f, two = a.interleaved ? 2 * f + 1 : f + a.pairs;
        const uint16_t u1 = r.src[one], u2 = r.src[two];
        const float x1 = to_float(u1, F16), y1 = to_float(u2, F16);
        r.dst[one] = turned ? from_float(x1 * s_turn[f].x - y1 * s_turn[f].y, F16) : u1;
        r.dst[two] = turned ? from_float(y1 * s_turn[f].x + x1 * s_turn[f].y, F16) : u2;
      }
    } else {
      for (int e = 2 * a.pairs + r.unit - groups; e < a.Dh; e += a.units - groups) r.dst[e] = r.src[e];
    }
  };

  Unit unit[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) unit[k] = fetch(tid + 256 * k);
  const int base = a.base != nullptr ? a.base[b] : 0;
  for (int f = tid; f < a.pairs; f += 256) {
    int axis = a.axis != nullptr ? a.axis[f] : 0;
    axis = axis < 0 ? 0 : (axis < a.axes ? axis : a.axes - 1);
    const double at = static_cast<double>(base) + static_cast<double>(a.pos[(static_cast<size_t>(axis) * a.B + b) * a.N + i]);
    const double turns = at * (static_cast<double>(a.inv_freq[f]) * 0.15915494309189535);
    float sine, cosine;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sine, &cosine);
    s_turn[f] = make_float2(cosine, sine);
  }
  __syncthreads();
  for (int x = tid;;) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) finish(unit[k]);
    x += 256 * AHEAD;
    if (x >= all) break;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) unit[k] = fetch(x + 256 * k);
  }
}

// ---- the accepted path's rows to their places behind the prefix.
// A workgroup has one (sequence, KV head) and 64 values of the rows of K or of V.  It reads all rows that move before it writes
// any, so the order of the path does not matter; the first row (the root's) is at its place.
constexpr int kPathMost = TALON_N_MAX;
__global__ __launch_bounds__(256) void paged_compact_kernel(CompactArgs a) {
  constexpr int kPer = kPathMost * 8 / 256;   // chunks of 8 values per thread
  const int b = blockIdx.z, g = blockIdx.y;
  const int groups = (a.Dh + 63) / 64;
  const bool is_v = static_cast<int>(blockIdx.x) >= groups;
  const int group = static_cast<int>(blockIdx.x) - (is_v ? groups : 0);
  const int tid = threadIdx.x;
  int len = a.accept_len[b];
  len = len < 0 ? -1 : (len < a.N ? len : a.N - 1);
  int P = a.prefix_len[b];
  P = P < 0 ? 0 : (P < a.c.capacity ? P : a.c.capacity);
  const int room = a.c.capacity - P;
  if (blockIdx.x == 0 && g == 0 && tid == 0) {
    a.new_prefix_len[b] = P + (len + 1 < room ? len + 1 : room);
    if (len + 1 > room) report(a.c, b, TALON_STATUS_BAD_PAGE);
  }
  const int count = len + 1 < room ? len + 1 : room;   // rows 0 .. count - 1 of the path
  uint16_t* const pool = static_cast<uint16_t*>(is_v ? a.c.v : a.c.k);
  uint4 v[kPer];
  uint32_t to[kPer];
  uint32_t moved = 0;
  const int col = group * 8 + (tid & 7);       // 16-byte chunk of the head
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int j = (tid >> 3) + 32 * u;
    to[u] = 0;
    v[u] = make_uint4(0, 0, 0, 0);
    if (j < count && col * 8 < a.Dh) {
      const int node = a.path[static_cast<size_t>(b) * a.N + j];
      if (node >= 0 && node < a.N && node != j) {
        bool bad = P + node >= a.c.capacity;
        if (!bad) {
          const uint32_t from = page_entry(a.c, b, P + node), dest = page_entry(a.c, b, P + j);
          bad = from >= a.c.num_pages || dest >= a.c.num_pages;
          if (!bad) {
            v[u] = *reinterpret_cast<const uint4*>(chunk_at(pool, row_chunk(a.c, from, P + node, g) + col));
            to[u] = row_chunk(a.c, dest, P + j, g) + col;
            moved |= 1u << u;
          }
        }
        if (bad) report(a.c, b, TALON_STATUS_BAD_PAGE);
      }
    }
  }
  float w = 0.f;
  float* const row = a.weights != nullptr ? a.weights + static_cast<size_t>(b) * a.stride_b + static_cast<size_t>(g) * a.stride_h : nullptr;
  bool w_moves = false;
  if (row != nullptr && blockIdx.x == 0 && tid < count) {
    const int node = a.path[static_cast<size_t>(b) * a.N + tid];
    w_moves = node >= 0 && node < a.N && node != tid && P + node < a.weight_rows && P + tid < a.weight_rows;
    if (w_moves) w = row[P + node];
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (all have arrived before one is written over)
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kPer; ++u)
    if (moved >> u & 1u) *reinterpret_cast<uint4*>(chunk_at(pool, to[u])) = v[u];
  if (w_moves) row[P + tid] = w;
}

// ---- which rows stay: per (sequence, KV head) the first n_sink, the last n_recent and, of those between, the ones of largest
// weight up to the budget; ties go to the lowest row.
// One workgroup of 1024 threads.  Rows that stay whatever they weigh get the largest key and rows past the end the least, so that
// the budget-th largest key decides.  It is found digit by digit (11, 11 and 10 bits of the order-preserving integer image, counts
// in LDS), then the rows are taken in order by ballots and a sum over the wavefronts.  Up to 16384 rows lie in registers, 16
// a thread (4 where no sequence has more than 4096); longer ones are read again from the caches for every digit.
// Bound: the steps that follow each other (three digits with three barriers each); 6.8 us at 4096 rows, 13.6 us at 16 x 8 x 16384,
// where a thread's rows that follow each other and one prefix sum per thread took 15 and 29.
constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;

// (a weight that is no number is the least of all)
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : sortable_u32(w); }

// Sum of the earlier wavefronts' counts; total: of all.  (s_wave is not written again before a barrier.)
__device__ __forceinline__ uint32_t earlier_waves(uint32_t count, uint32_t* s_wave, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  if (lane == 0) s_wave[wave] = count;
  __syncthreads();
  const int incl = wave_inclusive_scan_i32(lane < kSelectWaves ? static_cast<int>(s_wave[lane]) : 0);
  *total = static_cast<uint32_t>(__builtin_amdgcn_readlane(incl, 63));
  return wave == 0 ? 0u : static_cast<uint32_t>(__builtin_amdgcn_readlane(incl, wave - 1));
}

// Lanes below this one whose bit is set.
__device__ __forceinline__ uint32_t mask_rank(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0u));
}

template <int R>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int BLOCK = kSelectThreads * R;
  __shared__ uint32_t s_count[3][2048];
  __shared__ uint32_t s_wave[2][kSelectWaves];
  __shared__ uint32_t s_found[3];
  const int b = blockIdx.y, g = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  int len = a.len[b];
  for (int i = tid; i < 3 * 2048; i += kSelectThreads) (&s_count[0][0])[i] = 0u;
  len = len < 0 ? 0 : (len < a.max_len ? len : a.max_len);
  if (len > a.src.capacity && g == 0 && tid == 0) report(a.src, b, TALON_STATUS_BAD_PAGE);   // rows beyond the page table
  len = len < a.src.capacity ? len : a.src.capacity;
  const float* const w = a.weights + static_cast<size_t>(b) * a.stride_b + static_cast<size_t>(g) * a.stride_h;
  float* const w_out = a.new_weights != nullptr ? a.new_weights + static_cast<size_t>(b) * a.new_stride_b + static_cast<size_t>(g) * a.new_stride_h : nullptr;
  int32_t* const kept = a.kept + (static_cast<size_t>(b) * a.Hkv + g) * a.budget;
  const int stays = len < a.budget ? len : a.budget;
  if (g == 0 && tid == 0) a.new_len[b] = stays;
  for (int m = stays + tid; m < a.budget; m += kSelectThreads) kept[m] = -1;
  if (stays == len) {   // nothing is dropped
    for (int m = tid; m < len; m += kSelectThreads) {
      kept[m] = m;
      if (w_out != nullptr && w_out != w) w_out[m] = w[m];
    }
    return;
  }
  const int blocks = (len + BLOCK - 1) / BLOCK;
  float x[R];
  uint32_t key[R];
  const int at_lane = wave * (64 * R) + lane;   // a wavefront has 64 * R rows that follow each other
  auto load = [&](int block) {
    const int first = block * BLOCK + at_lane;
#pragma unroll
    for (int e = 0; e < R; ++e) {
      const int row = first + 64 * e;
      x[e] = w[row < len ? row : len - 1];
    }
#pragma unroll
    for (int e = 0; e < R; ++e) {
      const int row = first + 64 * e;
      key[e] = row >= len ? 0u : (row < a.n_sink || row >= len - a.n_recent ? ~0u : weight_key(x[e]));
    }
  };
  if (blocks == 1) load(0);
  uint32_t need = static_cast<uint32_t>(stays), found = 0, ties = 0;   // found: digits of the last key to stay that are known
  __syncthreads();
#pragma unroll
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : (digit == 1 ? 10 : 0);
    const int bits = digit == 2 ? 10 : 11;
    uint32_t* const counts = s_count[digit];
    for (int block = 0; block < blocks; ++block) {
      if (blocks > 1) load(block);
#pragma unroll
      for (int e = 0; e < R; ++e) {
        if (digit > 0 && key[e] >> (shift + bits) != found) continue;
        const uint32_t bin = key[e] >> shift & ((1u << bits) - 1u);
        // (rows that all fall into one bin, as zeros do, are counted at once)
        const uint32_t common = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(bin)));
        const unsigned long long here = __ballot(1);
        if (__ballot(bin == common) == here) {
          if (lane == __ffsll(static_cast<long long>(here)) - 1) atomicAdd(&counts[common], static_cast<uint32_t>(__popcll(here)));
        } else {
          atomicAdd(&counts[bin], 1u);
        }
      }
    }
    __syncthreads();
    // the bin, from the largest down, in which the need-th lies: two bins a thread, thread 0 has the largest
    const uint32_t lo_bin = 2046u - 2u * tid;
    const uint2 c = *reinterpret_cast<const uint2*>(&counts[lo_bin]);
    const uint32_t incl = static_cast<uint32_t>(wave_inclusive_scan_i32(static_cast<int>(c.x + c.y)));
    uint32_t all;
    const uint32_t before = earlier_waves(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(incl), 63)), s_wave[digit & 1], &all) + incl - c.x - c.y;
    if (before < need && need <= before + c.x + c.y) {
      const bool upper = need <= before + c.y;
      s_found[0] = lo_bin + (upper ? 1u : 0u);
      s_found[1] = need - before - (upper ? 0u : c.y);
      s_found[2] = upper ? c.y : c.x;
    }
    __syncthreads();
    found = found << bits | static_cast<uint32_t>(uniform(static_cast<int>(s_found[0])));
    need = static_cast<uint32_t>(uniform(static_cast<int>(s_found[1])));
    ties = static_cast<uint32_t>(uniform(static_cast<int>(s_found[2])));
  }
  // rows above `found` stay, and of those equal to it the first `need`
  uint32_t taken = 0, equal = 0;
  for (int block = 0; block < blocks; ++block) {
    if (blocks > 1) load(block);
    unsigned long long stay[R];
    uint32_t count = 0, total;
    if (ties == need) {
#pragma unroll
      for (int e = 0; e < R; ++e) stay[e] = __ballot(key[e] >= found);
    } else {
      uint32_t same = 0;
#pragma unroll
      for (int e = 0; e < R; ++e) same += static_cast<uint32_t>(__popcll(__ballot(key[e] == found)));
      uint32_t rank = equal + earlier_waves(same, s_wave[1], &total);
      equal += total;
#pragma unroll
      for (int e = 0; e < R; ++e) {
        const unsigned long long eq = __ballot(key[e] == found);
        stay[e] = __ballot(key[e] > found || (key[e] == found && rank + mask_rank(eq) < need));
        rank += static_cast<uint32_t>(__popcll(eq));
      }
    }
#pragma unroll
    for (int e = 0; e < R; ++e) count += static_cast<uint32_t>(__popcll(stay[e]));
    uint32_t at = taken + earlier_waves(count, s_wave[0], &total);
    taken += total;
    // (weights in place: a row only moves towards the front, and this block's are read)
#pragma unroll
    for (int e = 0; e < R; ++e) {
      const uint32_t to = at + mask_rank(stay[e]);
      if ((stay[e] >> lane & 1ull) && to < static_cast<uint32_t>(stays)) {
        kept[to] = block * BLOCK + at_lane + 64 * e;
        if (w_out != nullptr) w_out[to] = x[e];
      }
      at += static_cast<uint32_t>(__popcll(stay[e]));
    }
    if (blocks > 1) __syncthreads();
  }
}

// ---- rows move: kept[m] of the source's pages to row m of the destination's.
// In place a workgroup has one (sequence, KV head) and 2^lanes_log chunks of 8 values of the rows of K or of V and goes through the
// rows in order, a block of them read before it is written (a row only moves towards the front, so nothing is read behind its
// write).  Into other pages there is no order, and the rows are spread over as many workgroups as there are blocks.  A thread finds one
// row's places for all, while the block before moves.
// Bound: the bytes; 16 sequences, 4096 of up to 16384 rows each (8 heads of 128) into other pages 107 to 118 us (5 TB/s).  One
// sequence in place has too few workgroups for that: 1024 of 4096 rows 6.5 us, 30000 of 65536 183 us (203 where every lane finds its
// rows itself and between the blocks).
constexpr int kMoveThreads = 1024;
constexpr int kMoveChunks = 8;   // of 16 bytes per thread and block
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, int lanes_log) {
  constexpr uint32_t kStays = ~0u;
  __shared__ uint2 s_row[2][kMoveThreads];   // where a block's rows lie and where they go (first chunks), or kStays
  const int tid = threadIdx.x;
  const int per = kMoveThreads >> lanes_log;                       // rows of a chunk of the block
  const int step = per * kMoveChunks;                              // rows of a block: at most one per thread
  const int groups = (a.Dh / 8 + (1 << lanes_log) - 1) >> lanes_log;
  const int unit = blockIdx.x;                                     // K or V, a group of chunks
  const bool is_v = unit >= groups;
  const int col = ((unit - (is_v ? groups : 0)) << lanes_log) + (tid & ((1 << lanes_log) - 1));
  const int b = blockIdx.z / a.Hkv, g = blockIdx.z - b * a.Hkv;
  int len = a.len[b];
  len = len < 0 ? 0 : (len < a.max_len ? len : a.max_len);
  len = len < a.src.capacity ? len : a.src.capacity;
  const int stays = len < a.budget ? len : a.budget;
  if (a.in_place && stays == len) return;
  const int room = stays < a.dst.capacity ? stays : a.dst.capacity;
  if (room < stays && tid == 0) report(a.dst, b, TALON_STATUS_BAD_PAGE);
  const int32_t* const kept = a.kept + (static_cast<size_t>(b) * a.Hkv + g) * a.budget;
  const uint16_t* const from = static_cast<const uint16_t*>(is_v ? a.src.v : a.src.k);
  uint16_t* const to = static_cast<uint16_t*>(is_v ? a.dst.v : a.dst.k);
  const int stride = static_cast<int>(gridDim.y) * step;
  int m0 = static_cast<int>(blockIdx.y) * step;
  if (m0 >= room) return;

  // This thread's row of the block that begins at `first`, in two round trips to memory and then to LDS.
  int row = 0, m = 0;
  uint32_t e_from = 0, e_to = 0;
  bool mine = false;
  auto load_row = [&](int first) {
    m = first + tid;
    mine = tid < step && m < room;
    if (mine) row = kept[m];
  };
  auto load_pages = [&]() {
    if (mine) {
      e_from = page_entry(a.src, b, row);
      e_to = page_entry(a.dst, b, m);
    }
  };
  auto place = [&](int st) {
    uint2 at = make_uint2(kStays, kStays);
    if (mine && !(a.in_place && row == m)) {
      if (e_from < a.src.num_pages && e_to < a.dst.num_pages) at = make_uint2(row_chunk(a.src, e_from, row, g), row_chunk(a.dst, e_to, m, g));
      else report(e_from < a.src.num_pages ? a.dst : a.src, b, TALON_STATUS_BAD_PAGE);
    }
    s_row[st][tid] = at;
  };
  load_row(m0);
  load_pages();
  place(0);
  __syncthreads();
  for (int st = 0; m0 < room; m0 += stride, st ^= 1) {
    const bool more = m0 + stride < room;
    if (more) load_row(m0 + stride);
    u32x4 v[kMoveChunks];
    uint32_t dest[kMoveChunks];
#pragma unroll
    for (int u = 0; u < kMoveChunks; ++u) {
      const uint2 at = s_row[st][(tid >> lanes_log) + per * u];
      v[u] = u32x4{0, 0, 0, 0};
      dest[u] = kStays;
      if (at.y != kStays && col * 8 < a.Dh) {
        v[u] = *reinterpret_cast<const u32x4*>(chunk_at(from, at.x + col));
        dest[u] = at.y + col;
      }
    }
    if (more) load_pages();
    // (all rows of the block have arrived before one is written over)
#pragma unroll
    for (int u = 0; u < kMoveChunks; ++u) asm volatile("" : "+v"(v[u]));
    if (a.in_place) __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveChunks; ++u)
      if (dest[u] != kStays) *reinterpret_cast<u32x4*>(chunk_at(to, dest[u])) = v[u];
    if (more) {
      place(st ^ 1);
      __syncthreads();
    }
  }
}

}  // namespace

hipError_t launch_rotary_store(const RotaryArgs& args, int dtype, hipStream_t s) {
  RotaryArgs a = args;
  a.units = (a.pairs + 7) / 8 + (a.Dh - 2 * a.pairs + 15) / 16;
  // (x / units as a product: exact for x * units < 2^32, and x < 65792 heads * 65 units)
  a.inv_units = a.units == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + a.units - 1) / a.units);
  const dim3 grid(a.N, a.B);
  const size_t lds = static_cast<size_t>(a.pairs) * sizeof(float2);
  if (dtype == TALON_DTYPE_F16) hipLaunchKernelGGL(rotary_store_kernel<true>, grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL(rotary_store_kernel<false>, grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_compact(const CompactArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(paged_compact_kernel, dim3(2 * ((a.Dh + 63) / 64), a.Hkv, a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_evict(const EvictArgs& a, hipStream_t s) {
  if (a.max_len <= 4 * kSelectThreads) hipLaunchKernelGGL(evict_select_kernel<4>, dim3(a.Hkv, a.B), dim3(kSelectThreads), 0, s, a);
  else hipLaunchKernelGGL(evict_select_kernel<16>, dim3(a.Hkv, a.B), dim3(kSelectThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int most = a.budget < a.max_len ? a.budget : a.max_len;
  if (most == 0) return hipSuccess;
  // Chunks of a row that a workgroup moves: 128 values or what the head has (2 KiB that are read together and whole lines).  In place,
  // where a workgroup has all rows, 64 values if that leaves fewer workgroups than compute units: 4 sequences, 2048 of 8192 rows 25.8 us
  // against 28.5, one sequence, 30000 of 65536 233 against 321; with 16 sequences 128 values are better, 4096 of 16384 rows 129 us against 136.
  int lanes_log = a.Dh > 64 ? 4 : 3;
  if (a.in_place && lanes_log == 4 && 2ll * a.B * a.Hkv * ((a.Dh + 127) / 128) < 256) lanes_log = 3;
  const int step = (kMoveThreads >> lanes_log) * kMoveChunks;
  const int groups = (a.Dh / 8 + (1 << lanes_log) - 1) >> lanes_log;
  const int blocks = a.in_place ? 1 : (most + step - 1) / step < 65535 ? (most + step - 1) / step : 65535;
  hipLaunchKernelGGL(evict_move_kernel, dim3(2 * groups, blocks, a.B * a.Hkv), dim3(kMoveThreads), 0, s, a, lanes_log);
  return hipGetLastError();
}

}  // namespace talon
