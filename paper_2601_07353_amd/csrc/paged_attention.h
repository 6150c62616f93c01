// Attention of new tokens over a paged cache (App. B's tree attention where the cache is kept in pages), included by one
// source per storage type and head width.
//
//   x_ij = scale q_i . k_j,   capped: cap tanh(x / cap),   biased: - slope_h |p_i - p_j|,   -inf where i does not see j
//   out_i = sum_j softmax_j(x_ij) v_j,   lse_i = log sum_j exp(x_ij)
//
// One pass over the rows of K and V: running maximum, denominator and output (fp32).  The rows of the new tokens lie in the
// cache like all others, so there is one kind of key tile.
//
// Tiling.  The G query heads of a KV head and the new tokens make one row dimension (row = token * G + head).  A workgroup of
// NW = 4 or 8 wavefronts takes 32 * NW of these rows, 32 a wavefront, and streams 64-row tiles of K and V through LDS (two
// stages each, global to LDS without registers).  Both products are formed transposed (a query is a lane):
//   S^T[key][query] = K . Q^T,   O^T[dh][query] += V^T . P^T
// so that the accumulators of S^T are the operand P^T of the second product as they stand, and the statistics of a row are
// scalars of a lane.  While the matrix pipe forms the scores of tile t + 1 the vector pipe takes the exponentials of tile t.
// Bound: those two, which share a SIMD's issue slots; the step's barrier and the wait for its loads.  Two chunks of 2048 tokens at
// 8192 rows, 32/8 heads of 128, 661 us (936 TFLOP/s; 795 us capped, 735 with distances, 913 with both); one at 4096 rows, 16/4
// heads of 256 (one wavefront per SIMD), 308 us (558 TFLOP/s; 486 us with the tiles one after the other).
//
// Work.  Every (sequence, KV head, row tile) needs a number of key tiles that the host does not know (lengths are on the
// device).  All of them, end to end in that order, are one line of W tiles, cut into equal shares of ceil(W / workgroups), at
// least `least`: whatever the lengths are, no workgroup has more than a tile more than another.  (In front of a
// row tile's tiles the line has `extra` units of nothing, for what a workgroup does besides: queries, first loads, outputs.)  A share ends inside a row
// tile as a rule: what it has of it goes to a slot (output not yet divided, maximum, denominator; fp32), and a second kernel
// joins the slots of a row tile in the order of the shares.  A row tile that lies in one share is written at once.
// A share's first incomplete piece lies in slot 2 * share, a last one that is not also its first in 2 * share + 1; cut[share]
// says what the merge behind the share's end has to do: {sequence * Hkv + KV head, first row, rows, last share | (slot & 1) << 30},
// rows = 0 where nothing begins to be cut there.  Where every row tile has a few key tiles at most, nothing is cut: a share is
// a row tile, and there is no second launch.  Where there is little work, a share is one of the even pieces of a row tile.
//
// Values of V that are no finite numbers must not reach a row that does not see them (0 * NaN), so a tile that some row of the
// workgroup does not see whole is looked through for them first; where there are any they are set to zero and the rows that
// do see them become NaN.
#pragma once

#include <type_traits>

#include "paged_device.h"

namespace talon {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool F16>
struct Storage {
  using x8 = std::conditional_t<F16, f16x8, bf16x8>;
  using x4 = std::conditional_t<F16, f16x4, bf16x4>;
  using x1 = std::conditional_t<F16, _Float16, __bf16>;
  static constexpr uint32_t kExponents = F16 ? 0x7C007C00u : 0x7F807F80u;   // of two values
  static __device__ __forceinline__ floatx16 mfma(x8 a, x8 b, floatx16 c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // bit 0: the lower of the two values is no finite number, bit 1: the upper one
  static __device__ __forceinline__ uint32_t not_finite(uint32_t two) {
    const uint32_t e = two & kExponents;
    return ((e & 0xFFFFu) == (kExponents & 0xFFFFu) ? 1u : 0u) | ((e >> 16) == (kExponents >> 16) ? 2u : 0u);
  }
};

constexpr int kTileRows = 64;
constexpr int kMaskWords = 4;   // a mask of up to 256 new tokens is kept in LDS

// 16 bytes per lane from global memory to LDS, lane l at lds_base + 16 * l.  In assembly, because the compiler waits for all
// outstanding loads of its builtin before any LDS read; the waits are tile_landed()'s.
__device__ __forceinline__ void global_to_lds(const uint16_t* src, const uint16_t* lds_base) {
  const uint32_t lds_addr = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
      (__attribute__((address_space(3))) void*)(lds_base)));
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(src), "s"(lds_addr) : "memory", "m0");
}

// LDS image of a tile: rows of DH values without padding, the 16-byte chunks of a row permuted (differently for K, read as
// 16-byte fragments of 16 rows, and V, read by the transposing load) so that no two lanes of a read share a bank.
template <int DH>
struct PagedSmem {
  static constexpr int CPR = DH / 8;
  static constexpr int T_ELEMS = kTileRows * DH;
  static constexpr int POS_BYTES = 8 * (kTileRows + 32) * 4;       // positions of a tile's rows and of its queries, per wavefront
  static constexpr int MASK_BYTES = 256 * kMaskWords * 8;          // mask words of the queries
  static constexpr int BYTES = 4 * T_ELEMS * 2 + POS_BYTES + MASK_BYTES + 16;   // two stages of K, two of V; the rows of V that are not finite
  __device__ static int kswz(int row) { return DH >= 128 ? (row & 15) : ((row >> 1) & 7); }
  __device__ static int vswz(int row) { return DH >= 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); }
};

// Key tiles [*first, *first + result) of row tile rt of a sequence.
// ALL: of all rows, whatever sees them.
template <int TILE, int ROW_TILE, bool ALL = false>
__device__ __forceinline__ int tiles_of(const ScoreArgs& sc, int P, int n, uint32_t inv_g, int rt, int* first) {
  if constexpr (ALL) {
    *first = 0;
    return (P + n + TILE - 1) / TILE;
  }
  int last = div_g((rt + 1) * ROW_TILE - 1, inv_g);
  last = last < n - 1 ? last : n - 1;
  const int end = sc.mask != nullptr ? P + n : P + last + 1;
  int begin = 0;
  if (sc.window > 0) {
    const int lowest = P + (sc.offset != nullptr || sc.mask != nullptr ? 0 : div_g(rt * ROW_TILE, inv_g));
    begin = lowest - sc.window + 1;
    begin = begin < 0 ? 0 : begin;
  }
  *first = begin / TILE;
  return (end + TILE - 1) / TILE - begin / TILE;
}

// Rows beyond the page tables, reported by the workgroup of the last share, which has the least to do, if anything.  The kernels of few
// rows do it in find_share behind the lengths (in front of it: 0.3 us of one token's 10), that of many rows in front of it (behind the
// lengths: 2 % of 16 trees of 256 nodes at 16384 rows, through the loop's registers); beside the lengths that every workgroup looks at, it
// took 0.3 to 0.6 us of all calls over short prefixes, in instructions that are not in the cache yet.
__device__ __forceinline__ void report_table_ends(const PagedAttnArgs& a) {
  if (__builtin_expect(blockIdx.x == gridDim.x - 1, 0)) {
    const ScoreArgs& sc = a.sc;
#pragma unroll 1
    for (int b = static_cast<int>(threadIdx.x); b < a.B; b += static_cast<int>(blockDim.x))
      report_table_end(a.c, b, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N);
  }
}

// A workgroup's share of the line of key tiles: [x, x_end), which begins with tile `at` of row tile rt of (b, g).  Or a piece of one
// row tile, `take` tiles from `at` on, the last one of which has share `last`.
struct Share {
  int share, tiles;          // its number, tiles of a share
  int x, x_end;
  int b, g, rt, at, P, n;
  int take, last;            // of a piece (take > 0)
};

// Every wavefront works this out from the lengths, lane l for sequences l, l + 64, ...  (Loops, not unrolled copies: a workgroup
// comes here with a cold instruction cache.)  False: nothing to do.
template <int TILE, int ROW_TILE, bool ALL = false>
__device__ __forceinline__ bool find_share(const PagedAttnArgs& a, int lane, Share* w) {
  const ScoreArgs& sc = a.sc;
  const bool split = a.split != 0;
  // Workgroup ids are dealt round-robin to the 8 XCDs: neighbouring shares, which read the same rows of K and V where a sequence
  // has several row tiles, go to one XCD and its L2.  (The grid is a multiple of 8.)
  const int share = static_cast<int>(blockIdx.x & 7u) * (static_cast<int>(gridDim.x) >> 3) + static_cast<int>(blockIdx.x >> 3);
  int sum = 0, pieces = 0, P = 0, n = 0;   // of this lane's sequence: its tiles, its pieces of at most `least` tiles
  auto pieces_of = [&](int tiles) { return (tiles + a.least - 1) / a.least; };
  auto look = [&](int bb) {
    sum = pieces = P = n = 0;
    if (bb < a.B) {
      clamped_lengths(a.c, sc.prefix_len[bb], sc.n_new[bb], sc.max_prefix_len, sc.N, &P, &n);
      const int row_tiles = ALL ? (P + n > 0 ? 1 : 0) : (n * a.G + ROW_TILE - 1) / ROW_TILE;
      if (!split) sum = row_tiles;
      else {
        int first;
#pragma unroll 1
        for (int r = 0; r < row_tiles; ++r) {
          const int tiles = tiles_of<TILE, ROW_TILE, ALL>(sc, P, n, a.inv_g, r, &first);
          sum += tiles + a.extra;
          pieces += pieces_of(tiles);
        }
      }
      sum *= a.Hkv;
      pieces *= a.Hkv;
    }
  };
  int total_l = 0, pieces_l = 0;
#pragma unroll 1
  for (int bb = lane; bb - lane < a.B; bb += 64) {
    look(bb);
    total_l += sum;
    pieces_l += pieces;
  }
  if constexpr (ROW_TILE == 32) report_table_ends(a);
  int total = uniform(wave_sum_i32(total_l));   // of tiles and what row tiles cost besides them
  int tiles = (total + a.slots - 1) / a.slots;
  // Little work: pieces of single row tiles, no share with two of them (and their two prologues)
  bool alone = false;
  if (split && tiles <= a.least) {
    const int all = uniform(wave_sum_i32(pieces_l));
    alone = all <= a.slots;
    if (alone) total = all;
  }
  tiles = alone ? 1 : (tiles < a.least ? a.least : tiles);
  const long long x0 = static_cast<long long>(share) * tiles;
  if (a.cut != nullptr && threadIdx.x == 0 && share < a.slots) a.cut[share] = make_int4(0, 0, 0, 0);
  if (x0 >= total) return false;
  const int x = static_cast<int>(x0);
  int before = 0, b = 0, at = 0, mine = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (a.B > 64) look(b0 + lane);   // (else this lane's sequence is the one it has looked at)
    const int units = alone ? pieces : sum;
    const int incl = wave_inclusive_scan_i32(units);
    const int begin = before + incl - units;
    const unsigned long long in = __ballot(x >= begin && x < begin + units);
    if (in != 0ull) {
      const int l = __ffsll(static_cast<long long>(in)) - 1;
      b = b0 + l;
      at = x - __builtin_amdgcn_readlane(begin, l);
      mine = __builtin_amdgcn_readlane(units, l);
      P = __builtin_amdgcn_readlane(P, l);
      n = __builtin_amdgcn_readlane(n, l);
      break;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  b = uniform(b); at = uniform(at); P = uniform(P); n = uniform(n);
  const int per_head = uniform(mine) / a.Hkv;
  const int g = at / per_head;
  at -= g * per_head;
  int rt = 0;
  w->take = 0;
  w->last = 0;
  if (split) {
#pragma unroll 1
    for (int first;; ++rt) {
      const int t = tiles_of<TILE, ROW_TILE, ALL>(sc, P, n, a.inv_g, rt, &first);
      const int k = alone ? pieces_of(t) : t + a.extra;
      if (at < k) {
        if (alone) {   // piece `at` of k even ones
          w->last = share + k - 1 - at;
          const int begin = static_cast<int>(static_cast<long long>(t) * at / k);
          w->take = static_cast<int>(static_cast<long long>(t) * (at + 1) / k) - begin;
          at = begin;
        }
        break;
      }
      at -= k;
    }
  } else {
    rt = at;
    at = 0;
  }
  w->share = share; w->tiles = tiles; w->x = x; w->x_end = total - x < tiles ? total : x + tiles;
  w->b = b; w->g = g; w->rt = rt; w->at = at; w->P = P; w->n = n;
  return true;
}

// What a share has of a row tile of `tiles` tiles, from unit `at` of it on.
struct Piece {
  int from, to;    // its tiles
  int units;       // its length on the line
  int last;        // share of the row tile's last tile
};
__device__ __forceinline__ Piece next_piece(const PagedAttnArgs& a, const Share& w, int tiles, int at, int x) {
  if (!a.split) return {0, tiles, 1, 0};
  if (w.take > 0) return {at, at + w.take, w.x_end - x, w.last};
  const int rest = tiles + a.extra - at;
  const int units = rest < w.x_end - x ? rest : w.x_end - x;
  const int from = at - a.extra, to = at + units - a.extra;
  return {from < 0 ? 0 : from, to < 0 ? 0 : to, units, (x - at + a.extra + tiles - 1) / w.tiles};
}

// FAR: the cap is above kNearCap.
template <bool F16, int DH, int NW, bool CAP, bool BIAS, bool FAR>
__global__ __launch_bounds__(64 * NW, DH == 256 ? 1 : (NW == 4 ? 2 : 1)) void paged_attention_kernel(PagedAttnArgs a) {
  constexpr bool MOD = CAP || BIAS;   // scores are brought to base-2 units before the softmax
  using ST = Storage<F16>;
  using x8 = typename ST::x8;
  using x4 = typename ST::x4;
  using SM = PagedSmem<DH>;
  constexpr int kWgThreads = 64 * NW;
  constexpr int DSTEPS = DH / 16;
  constexpr int DB = DH / 32;
  constexpr int CPR = DH / 8;
  constexpr int kRowTile = 32 * NW;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31;
  const int h = lane >> 5;
  const ScoreArgs& sc = a.sc;
  const int G = a.G;

  report_table_ends(a);
  Share w;
  if (!find_share<kTileRows, kRowTile>(a, lane, &w)) return;
  int b = w.b, g = w.g, rt = w.rt, at = w.at, x = w.x, P = w.P, n = w.n;
  const int x_end = w.x_end, share = w.share;

  const uint16_t* const k_pool = static_cast<const uint16_t*>(a.c.k);
  const uint16_t* const v_pool = static_cast<const uint16_t*>(a.c.v);
  int* const s_pos = reinterpret_cast<int*>(smem + 4 * SM::T_ELEMS) + wave * (kTileRows + 32);
  uint64_t* const s_mask = reinterpret_cast<uint64_t*>(reinterpret_cast<char*>(smem + 4 * SM::T_ELEMS) + SM::POS_BYTES);
  uint32_t* const s_bad = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(s_mask) + SM::MASK_BYTES);
  auto stage_k = [&](int st) { return smem + st * SM::T_ELEMS; };
  auto stage_v = [&](int st) { return smem + (2 + st) * SM::T_ELEMS; };

  // Tile loads.  With eight wavefronts the last four issue them: a compute unit's address path takes a tile pair's 32 KB in
  // about 512 cycles whoever issues them, and a wavefront waits at its loads for its turn.
  constexpr int ROWS_PER_LOAD = 64 / CPR;
  constexpr int LW = NW == 8 ? 4 : NW;
  constexpr int LOADS = kTileRows / ROWS_PER_LOAD / LW;
  constexpr int ROWS_WAVE = kTileRows / LW;
  const int lwave = wave - (NW - LW);
  const bool loader = lwave >= 0;
  // The lane index anew: what is worked out from it is not kept in registers (or spilled) across the loop by the compiler, which
  // takes this for another value each time.  Around the loads and the rare paths; the fragment reads keep their addresses.
  auto lane_again = [&]() {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
  };

  bool first_piece = true;
  while (x < x_end) {
    // ---- the piece: key tiles [t_begin, t_end) of (b, g, rt)
    int first_tile;
    const int tiles = tiles_of<kTileRows, kRowTile>(sc, P, n, a.inv_g, rt, &first_tile);
    const Piece pc = next_piece(a, w, tiles, at, x);
    if (pc.from == pc.to) break;   // the share ends with what the row tile costs besides its tiles
    const int t_begin = first_tile + pc.from;
    const int t_end = first_tile + pc.to;
    const bool whole = pc.to - pc.from == tiles;
    const int rows = n * G;
    const int row0 = rt * kRowTile;
    const int wrow0 = row0 + wave * 32;
    const int tk0 = div_g(row0, a.inv_g);
    int tk1 = div_g(row0 + kRowTile - 1, a.inv_g);
    tk1 = tk1 < n - 1 ? tk1 : n - 1;
    const int kend = sc.mask != nullptr ? P + n : P + tk1 + 1;   // rows of the cache that the tile looks at
    const bool works = wrow0 < rows;                              // this wavefront has queries

    // ---- this lane's query
    const int rho = wrow0 + l32;
    const bool valid = rho < rows;
    const int token = valid ? div_g(rho, a.inv_g) : tk0;
    const int head = g * G + (valid ? rho - token * G : 0);
    int p_own = P + token;
    float slope2 = 0.f;
    auto token_of = [&](int ln) {
      const int rho_ = wrow0 + (ln & 31);
      return rho_ < rows ? div_g(rho_, a.inv_g) : tk0;
    };

    // ---- which tiles every row of the workgroup sees whole: those inside [seen_from, seen_to)
    const bool positions = sc.window > 0 || BIAS;
    const bool mask_here = sc.mask != nullptr && sc.words <= kMaskWords;
    int seen_to = sc.mask != nullptr || (positions && sc.offset != nullptr) ? P : P + tk0 + 1;
    int seen_from = 0;
    if (sc.window > 0) {
      int most = tk1;
      if (sc.offset != nullptr) {
        most = 0;
        for (int i = tk0 + lane; i <= tk1; i += 64) { const int o = offset_of(sc, b, i); most = most > o ? most : o; }
        most = __builtin_amdgcn_readfirstlane(wave_max_i32(most));
      }
      seen_from = P + most - sc.window + 1;
    }

    float m_run = kNoScore, l_run = 0.f;
    floatx16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.f;

    // ---- addresses of a tile's rows.  A loading wavefront takes ROWS_WAVE rows of a tile, ROWS_PER_LOAD an instruction.  Lane l
    // finds row l % ROWS_WAVE: its page entry, read a step ahead, and where it lies; the lanes of a load then take their rows' places
    // from it.  (Every lane on its own, as many entries and products as loads, cost 0.1 us more a tile; scalar addresses with the
    // entries held a lane each 0.15.)  A row past the end reads the last row instead; its score is hidden.
    uint32_t entry = 0, k_row[LOADS], v_row[LOADS];
    auto key_of = [&](int t, int ln) {
      const int key = t * kTileRows + lwave * ROWS_WAVE + (ln & (ROWS_WAVE - 1));
      return key < kend ? key : kend - 1;
    };
    auto load_entries = [&](int t) {
      if (!loader) return;
      entry = page_entry(a.c, b, key_of(t, lane_again()));
    };
    // (waited for here, in front of the tile loads: where it was first used the wait would count those too)
    auto entries_landed = [&]() { asm volatile("" : "+v"(entry)); };
    auto rows_of = [&](int t, uint32_t (&to)[LOADS]) {
      const int ln = lane_again();
      if (__ballot(entry >= a.c.num_pages) != 0ull && ln == 0) report(a.c, b, TALON_STATUS_BAD_PAGE);
      const int row = static_cast<int>(row_chunk(a.c, entry, key_of(t, ln), g));
#pragma unroll
      for (int i = 0; i < LOADS; ++i) to[i] = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute((i * ROWS_PER_LOAD + ln / CPR) * 4, row));
    };
    auto load_tile = [&](const uint16_t* pool, uint16_t* to, const uint32_t (&rows_)[LOADS], bool is_k) {
      const int lrow = lane / CPR, cslot = lane % CPR;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int u = (lwave * LOADS + i) * ROWS_PER_LOAD;
        const uint32_t chunk = static_cast<uint32_t>(cslot ^ (is_k ? SM::kswz(u + lrow) : SM::vswz(u + lrow)));
        global_to_lds(chunk_at(pool, rows_[i] + chunk), to + u * DH);
      }
    };
    auto tile_landed = [&]() {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    };

    x8 bq[DSTEPS];
    auto qk = [&](const uint16_t* sK, floatx16 (&s)[2], int ln) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
        const int krow_i = 32 * kb + (ln & 31);
        const uint16_t* krow = sK + krow_i * DH;
        const int ksw = SM::kswz(krow_i);
#pragma unroll
        for (int ds = 0; ds < DSTEPS; ++ds) {
          const x8 ak = __builtin_bit_cast(x8, *reinterpret_cast<const uint4*>(krow + ((2 * ds + (ln >> 5)) ^ ksw) * 8));
          s[kb] = ST::mfma(ak, bq[ds], s[kb]);
        }
      }
      // (fragments are read four matrix instructions ahead)
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int g_ = 0; g_ < 2 * DSTEPS - 4; ++g_) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };

    auto seen_by = [&](int i, int key0) {   // rows of a tile that token i may see, but for the window
      if (mask_here) return seen_rows(sc, i, P, key0, kend, s_mask + (i - tk0) * sc.words);
      return seen_rows(sc, b, i, P, key0, kend);
    };
    // Scores are in base-2 units with MOD, else still to be multiplied by scale * log2(e).
    // Register r of s[kb] is row 32 * kb + 8 * (r / 4) + 4 * h + r % 4 of the tile.
    auto base2_scores = [&](floatx16 (&s)[2]) {
      if constexpr (FAR) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = sc.cap_log2e * tanh_of(s[kb][r] * sc.cap_in);
      } else if constexpr (CAP) {
        // cap * tanh(x) = cap * (1 - 2 / (1 + e^(2x)))
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(s[kb][r] * sc.cap_in);
            s[kb][r] = __builtin_fmaf(-2.f * sc.cap_log2e, __builtin_amdgcn_rcpf(1.f + e), sc.cap_log2e);
          }
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] *= sc.scale_log2e;
      }
    };
    // ... of a tile that all rows see whole, which lies in front of every query: the bias is slope * (p_i - key)
    auto whole_scores = [&](int t, floatx16 (&s)[2]) {
      base2_scores(s);
      if constexpr (BIAS) {
        const float bias0 = slope2 * static_cast<float>(p_own - t * kTileRows - 4 * h);
#pragma unroll
        for (int q8 = 0; q8 < 8; ++q8) {   // (eight constants instead of 32, which the compiler keeps in registers)
          const float bias = __builtin_fmaf(slope2, static_cast<float>(8 * q8), -bias0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[q8 / 4][4 * (q8 % 4) + e] += __builtin_fmaf(slope2, static_cast<float>(e), bias);
        }
      }
    };
    // ... of any tile: the bias, and -inf where a row is not seen
    auto hide_rows = [&](int t, floatx16 (&s)[2]) {
      const int key0 = t * kTileRows;
      const int ln = lane_again();
      const int h_ = ln >> 5;
      const unsigned long long bits = seen_by(token_of(ln), key0);
      int p_i = 0;
      if (positions) {
        p_i = s_pos[kTileRows + (ln & 31)];
        const int key = key0 + ln;
        int pos = key;
        if (key >= P && key < kend) pos = P + offset_of(sc, b, key - P);
        __builtin_amdgcn_wave_barrier();
        s_pos[ln] = pos;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      const int window = sc.window > 0 ? sc.window : 0x7FFFFFFF;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t w = static_cast<uint32_t>(bits >> (32 * kb)) >> (4 * h_);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          int4 pos = make_int4(0, 0, 0, 0);
          if (positions) pos = *reinterpret_cast<const int4*>(s_pos + 32 * kb + 8 * q4 + 4 * h_);
          const int ps[4] = {pos.x, pos.y, pos.z, pos.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * q4 + e;
            bool seen = (w >> (8 * q4 + e)) & 1u;
            if (positions) {
              const int apart = p_i - ps[e];
              seen = seen && apart < window;
              if constexpr (BIAS) s[kb][r] = __builtin_fmaf(-slope2, fabsf(static_cast<float>(apart)), s[kb][r]);
            }
            s[kb][r] = seen ? s[kb][r] : kNoScore;
          }
        }
      }
    };
    // Rows of tile t that this lane's query sees, as bits (again; for the rare tile with values that are not finite).
    auto seen_bits = [&](int t) {
      const int ln = lane_again();
      unsigned long long bits = seen_by(token_of(ln), t * kTileRows);
      if (sc.window > 0) {
        const int p_i = s_pos[kTileRows + (ln & 31)];
        for (int k = 0; k < kTileRows; ++k) {
          const int key = t * kTileRows + k;
          const int pos = key < P || key >= kend ? key : P + offset_of(sc, b, key - P);
          if (p_i - pos >= sc.window) bits &= ~(1ull << k);
        }
      }
      return bits;
    };

    // V of a tile that not every row sees: are all values finite?  (Entered and left by all wavefronts together.)
    auto clean_v = [&](int t, int st) {
      uint4* const v = reinterpret_cast<uint4*>(stage_v(st));
      uint32_t any = 0;
      const int tid = wave * 64 + lane_again();
#pragma unroll
      for (int c = 0; c < SM::T_ELEMS / 8 / kWgThreads; ++c) {
        const uint4 u = v[c * kWgThreads + tid];
        any |= ST::not_finite(u.x) | ST::not_finite(u.y) | ST::not_finite(u.z) | ST::not_finite(u.w);
      }
      if (!__syncthreads_or(any != 0u)) return;
      if (tid < 2) s_bad[tid] = 0u;
      __syncthreads();
      for (int c = 0; c < SM::T_ELEMS / 8 / kWgThreads; ++c) {
        const int chunk = c * kWgThreads + tid;
        uint4 u = v[chunk];
        uint32_t* const w = reinterpret_cast<uint32_t*>(&u);
        uint32_t found = 0;
        for (int e = 0; e < 4; ++e) {
          const uint32_t bad = ST::not_finite(w[e]);
          found |= bad;
          if (bad & 1u) w[e] &= 0xFFFF0000u;
          if (bad & 2u) w[e] &= 0x0000FFFFu;
        }
        if (found) {
          v[chunk] = u;
          const int row = chunk / CPR;
          atomicOr(&s_bad[row >> 5], 1u << (row & 31));
        }
      }
      __syncthreads();
      const unsigned long long bad = s_bad[0] | (static_cast<unsigned long long>(s_bad[1]) << 32);
      if (seen_bits(t) & bad) l_run = __builtin_nanf("");
    };

    // What a step does with a tile's finished scores, in parts: running maximum (returns what the output was scaled by) ...
    auto new_maximum = [&](const floatx16 (&s)[2], float* m_safe) {
      float mx = kNoScore;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
      const int mi = __float_as_int(mx);
      const auto sw = __builtin_amdgcn_permlane32_swap(mi, mi, false, false);
      mx = fmaxf(__int_as_float(static_cast<int>(sw[0])), __int_as_float(static_cast<int>(sw[1])));
      const float m_new = fmaxf(m_run, MOD ? mx : mx * sc.scale_log2e);
      *m_safe = m_new == kNoScore ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - *m_safe);
      m_run = m_new;
      if (__ballot(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      }
      return alpha;
    };
    // ... probabilities (rounded to the storage type for the matrix product; the denominator sums them unrounded) ...
    auto probabilities = [&](const floatx16 (&s)[2], float m_safe, float alpha, x8 (&pb)[2][2]) {
      float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int sp = 0; sp < 2; ++sp) {
          x8 pk;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = s[kb][8 * sp + e];
            const float p = __builtin_amdgcn_exp2f(MOD ? v - m_safe : __builtin_fmaf(v, sc.scale_log2e, -m_safe));
            if (e & 1) sum1 += p; else sum0 += p;
            pk[e] = static_cast<typename ST::x1>(p);
          }
          pb[kb][sp] = pk;
        }
      }
      l_run = l_run * alpha + (sum0 + sum1);
    };
    // ... and O^T += V^T . P^T
    auto add_values = [&](const uint16_t* sV, const x8 (&pb)[2][2], int ln) {
      const int i16 = ln & 15;
      const int dhblk = (ln >> 4) & 1;
      const int vrow_l = 4 * (ln >> 5) + (i16 >> 2);
      const int vsw = SM::vswz(vrow_l);
      const int vch = 2 * dhblk + ((i16 & 3) >> 1);
      const int vsub = (i16 & 1) * 4;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int sp = 0; sp < 2; ++sp) {
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const uint16_t* vp = sV + (32 * kb + 16 * sp + vrow_l) * DH + ((4 * db + vch) ^ vsw) * 8 + vsub;
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vp));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vp + 8 * DH));
            const short8v both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            o[db] = ST::mfma(__builtin_bit_cast(x8, both), pb[kb][sp], o[db]);
          }
        }
      }
      // (the two reads of a fragment run two matrix instructions ahead)
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int g_ = 0; g_ < 4 * DB - 2; ++g_) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
    };
    // Loads of a step: V(t + 1), K(t + 2) to the stage that K(t) has left, and the page entries of tile t + 3.
    auto next_loads = [&](int t, int stage) {
      if (!loader) return;
      entries_landed();
      if (t + 2 < t_end) rows_of(t + 2, k_row);
      if (t + 1 < t_end) load_tile(v_pool, stage_v(stage ^ 1), v_row, false);
      if (t + 2 < t_end) load_tile(k_pool, stage_k(stage), k_row, true);
      if (t + 3 < t_end) load_entries(t + 3);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) v_row[j] = k_row[j];
    };

    // Two kinds of steps over one scheme of loads: when the step of tile t begins, K(t), V(t) and K(t + 1) are in LDS, those of
    // even tiles (counted from the first one of the run of whole tiles) in stage 0.
    // A tile that all rows see whole, and whose next is one too: its scores are in s; those of tile t + 1 are formed while its
    // exponentials are taken.  All other tiles (the last of the run, those of a sequence's end, a window's first) go one thing
    // after the other: see the loop below.
    auto step = [&](int t, int ln, auto stage, floatx16 (&s)[2], floatx16 (&s_nxt)[2]) {
      constexpr int kStage = decltype(stage)::value;
      next_loads(t, kStage);
      if (works) {
        x8 pb[2][2];
        float m_safe;
        const float alpha = new_maximum(s, &m_safe);
        qk(stage_k(kStage ^ 1), s_nxt, ln);
        probabilities(s, m_safe, alpha, pb);
        // (Never taken.  It ends a block: the compiler then lets the exponentials run among the matrix instructions of the second
        // product, whose schedule it would otherwise lose among those of the first.  Two chunks of 2048 tokens at 8192 rows: 541 us
        // without, 512 with it.)
        if (t_end < 0) asm volatile("s_nop 0");
        if constexpr (MOD) whole_scores(t + 1, s_nxt);   // (among the matrix instructions of the second product)
        add_values(stage_v(kStage), pb, ln);
      }
      tile_landed();
    };
    // What is left of a tile whose scores are there.
    auto finish_step = [&](int t, int stage, const floatx16 (&s)[2]) {
      next_loads(t, stage);
      if (works) {
        x8 pb[2][2];
        float m_safe;
        const float alpha = new_maximum(s, &m_safe);
        probabilities(s, m_safe, alpha, pb);
        add_values(stage_v(stage), pb, lane_again());
      }
      tile_landed();
    };
    // ---- the tiles of the piece that all rows see whole: [whole_from, whole_to)
    int whole_from = (seen_from + kTileRows - 1) / kTileRows, whole_to = seen_to / kTileRows;
    if (seen_from <= 0) whole_from = 0;
    whole_from = whole_from < t_begin ? t_begin : whole_from;
    whole_to = whole_to < t_end ? whole_to : t_end;
    if (whole_from >= whole_to) whole_from = whole_to = t_end;   // none
    auto stage_of = [&](int t) { return (t - whole_from) & 1; };

    // ---- prologue.  Two round trips to memory: everything that needs no other load (queries, page entries, positions, slopes, mask
    // words), then the first tiles.
    {
      u32x4 qv[DSTEPS];
      const uint16_t* qp = a.q.p + static_cast<int64_t>(b) * a.q.sb + static_cast<int64_t>(token) * a.q.st + static_cast<int64_t>(head) * a.q.sh + 8 * h;
      if (loader) load_entries(t_begin);
      uint32_t second = 0;
      if (loader && t_begin + 1 < t_end) second = page_entry(a.c, b, key_of(t_begin + 1, lane_again()));
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) {
        qv[ds] = u32x4{0, 0, 0, 0};
        if (valid) qv[ds] = *reinterpret_cast<const u32x4*>(qp + 16 * ds);
      }
      int off = token;
      if (sc.offset != nullptr) off = sc.offset[static_cast<size_t>(b) * sc.N + token];
      if constexpr (BIAS) slope2 = sc.slopes[head] * kLog2eF;
      if (mask_here) {
        for (int i = tid; i < (tk1 - tk0 + 1) * sc.words; i += kWgThreads)
          s_mask[i] = sc.mask[(static_cast<size_t>(b) * sc.N + tk0) * sc.words + i];
      }
      if (loader) {
        asm volatile("" : "+v"(entry), "+v"(second));
        rows_of(t_begin, v_row);
        load_tile(k_pool, stage_k(stage_of(t_begin)), v_row, true);
        load_tile(v_pool, stage_v(stage_of(t_begin)), v_row, false);
        if (t_begin + 1 < t_end) {
          entry = second;
          rows_of(t_begin + 1, v_row);
          load_tile(k_pool, stage_k(stage_of(t_begin + 1)), v_row, true);
        }
        if (t_begin + 2 < t_end) load_entries(t_begin + 2);
      }
      p_own = P + (off < 0 ? 0 : (off < kMostOffset ? off : kMostOffset));
      if (h == 0) s_pos[kTileRows + l32] = p_own;   // (read by this wavefront alone)
      // the compiler's waits for these loads stand here, not inside the loop
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ds += 4) asm volatile("" : "+v"(qv[ds]), "+v"(qv[ds + 1]), "+v"(qv[ds + 2]), "+v"(qv[ds + 3]));
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) bq[ds] = __builtin_bit_cast(x8, qv[ds]);
    }
    tile_landed();
    for (int t = t_begin; t < t_end; ++t) {
      floatx16 s_a[2];
      const bool whole_run = t == whole_from;
      if (!whole_run) clean_v(t, stage_of(t));
      if (works) {
        qk(stage_k(stage_of(t)), s_a, lane_again());
        if (whole_run) {
          if constexpr (MOD) whole_scores(t, s_a);
        } else {
          if constexpr (MOD) base2_scores(s_a);
          hide_rows(t, s_a);
        }
      }
      __syncthreads();   // K(t) is used up
      if (whole_run) {
        const int ln = lane_again();
        constexpr std::integral_constant<int, 0> even{};
        constexpr std::integral_constant<int, 1> odd{};
        floatx16 s_b[2];
        for (; t + 2 < whole_to; t += 2) {   // (in pairs, so that the two sets of scores swap roles without a copy)
          step(t, ln, even, s_a, s_b);
          step(t + 1, ln, odd, s_b, s_a);
        }
      }
      finish_step(t, stage_of(t), s_a);
    }

    // ---- what became of the rows
    float l_tot;
    {
      const int li = __float_as_int(l_run);
      const auto sw = __builtin_amdgcn_permlane32_swap(li, li, false, false);
      l_tot = __int_as_float(static_cast<int>(sw[0])) + __int_as_float(static_cast<int>(sw[1]));
    }
    // (worked out again from a lane index that the compiler cannot trace back: it would keep the addresses across the loop)
    int l32_e = l32;
    asm volatile("" : "+v"(l32_e));
    const int rho_e = wrow0 + l32_e;
    if (rho_e < rows) {
      if (whole) {
        const int token_e = div_g(rho_e, a.inv_g);
        const int head_e = g * G + rho_e - token_e * G;
        const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;   // a row that sees nothing
        uint16_t* op = a.out.p + static_cast<int64_t>(b) * a.out.sb + static_cast<int64_t>(token_e) * a.out.st + static_cast<int64_t>(head_e) * a.out.sh;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = static_cast<typename ST::x1>(o[db][4 * q4 + e] * inv);
            *reinterpret_cast<x4*>(op + 32 * db + 8 * q4 + 4 * h) = v;
          }
        if (a.lse != nullptr && h == 0)
          a.lse[(static_cast<size_t>(b) * sc.N + token_e) * (a.Hkv * G) + head_e] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2F;
      } else {
        const int slot = 2 * share + (first_piece ? 0 : 1);
        const int r = rho_e - row0;
        float* po = a.part_o + (static_cast<size_t>(slot) * (DH / 8) * a.rows_slot + r) * 8 + 4 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            float4 v = make_float4(o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
            *reinterpret_cast<float4*>(po + static_cast<size_t>(4 * db + q4) * a.rows_slot * 8) = v;
          }
        if (h == 0) {
          a.part_m[static_cast<size_t>(slot) * a.rows_slot + r] = m_run;
          a.part_l[static_cast<size_t>(slot) * a.rows_slot + r] = l_tot;
        }
      }
    }
    // the row tile goes on behind this share, and begins in it: the merge at this share's end joins it
    if (pc.from == 0 && pc.to < tiles && tid == 0) {
      const int count = rows - row0 < kRowTile ? rows - row0 : kRowTile;
      a.cut[share] = make_int4(b * a.Hkv + g, row0, count, pc.last | (first_piece ? 0 : 1 << 30));
    }

    // ---- on to the next row tile
    x += pc.units;
    at = 0;
    first_piece = false;
    if (x < x_end) {
      ++rt;
      if (rt * kRowTile >= rows) {
        rt = 0;
        if (++g == a.Hkv) {
          g = 0;
          do {   // (x < x_end: there is another sequence with new tokens)
            ++b;
            clamped_lengths(a.c, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N, &P, &n);
          } while (n == 0);
        }
      }
      __syncthreads();   // (s_bad and the stages are free)
    }
  }
}

// Joins the pieces of a row tile that begins in share blockIdx.y and ends in another one.
//   out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s
// One thread per (row, 4 values); pieces are read in the order in which they lie (thread = (slab, row, half)) and the rows
// turned through LDS.
// Bound: the bytes of the pieces; 9 us for 4 trees of 128 nodes (41 MB), 16 us for two chunks of 2048 tokens.
template <bool F16, int DH>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(PagedAttnArgs a) {
  using ST = Storage<F16>;
  using x4 = typename ST::x4;
  constexpr int QPR = DH / 4;
  constexpr int RPW = 256 / QPR;
  __shared__ x4 s_out[RPW][QPR];
  const int share = blockIdx.y;
  const int4 cut = a.cut[share];
  if (static_cast<int>(blockIdx.x) * RPW >= cut.z) return;
  const int last = cut.w & 0x3FFFFFFF;
  const int t = threadIdx.x;
  const int h = t & 1;
  const int r = (t >> 1) % RPW;
  const int slab = t / (2 * RPW);
  const int c = 2 * slab + h;
  int row = blockIdx.x * RPW + r;
  const bool valid = row < cut.z;
  row = valid ? row : cut.z - 1;
  float M = kNoScore, den = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const int pieces = last - share + 1;
  for (int s0 = 0; s0 < pieces; s0 += 8) {
    float ms[8], ls[8];
    float4 vs[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      ms[u] = kNoScore;
      ls[u] = 0.f;
      vs[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s0 + u < pieces) {
        const int slot = 2 * (share + s0 + u) + (s0 + u == 0 ? cut.w >> 30 : 0);
        const size_t at = static_cast<size_t>(slot) * a.rows_slot;
        ms[u] = a.part_m[at + row];
        ls[u] = a.part_l[at + row];
        vs[u] = *reinterpret_cast<const float4*>(a.part_o + (at * (DH / 8) + static_cast<size_t>(slab) * a.rows_slot + row) * 8 + 4 * h);
      }
    }
    float Mb = M;
#pragma unroll
    for (int u = 0; u < 8; ++u) Mb = fmaxf(Mb, ms[u]);
    const float safe = Mb == kNoScore ? 0.f : Mb;   // (a piece that saw nothing has no weight; one with a NaN keeps it)
    const float keep = __builtin_amdgcn_exp2f(M - safe);
    M = Mb;
    den *= keep;
    acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = __builtin_amdgcn_exp2f(ms[u] - safe);
      den = __builtin_fmaf(w, ls[u], den);
      acc.x = __builtin_fmaf(w, vs[u].x, acc.x); acc.y = __builtin_fmaf(w, vs[u].y, acc.y);
      acc.z = __builtin_fmaf(w, vs[u].z, acc.z); acc.w = __builtin_fmaf(w, vs[u].w, acc.w);
    }
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  x4 v;
  v[0] = static_cast<typename ST::x1>(acc.x * inv);
  v[1] = static_cast<typename ST::x1>(acc.y * inv);
  v[2] = static_cast<typename ST::x1>(acc.z * inv);
  v[3] = static_cast<typename ST::x1>(acc.w * inv);
  s_out[r][c] = v;
  const int b = cut.x / a.Hkv;
  const int g = cut.x - b * a.Hkv;
  if (a.lse != nullptr && c == 0 && valid) {
    const int rho = cut.y + row;
    const int token = div_g(rho, a.inv_g);
    a.lse[(static_cast<size_t>(b) * a.sc.N + token) * (a.Hkv * a.G) + g * a.G + rho - token * a.G] = (M + __builtin_amdgcn_logf(den)) * kLn2F;
  }
  __syncthreads();
  const int r2 = t / QPR;
  const int c2 = t - r2 * QPR;
  const int row2 = blockIdx.x * RPW + r2;
  if (row2 < cut.z) {
    const int rho = cut.y + row2;
    const int token = div_g(rho, a.inv_g);
    uint16_t* op = a.out.p + static_cast<int64_t>(b) * a.out.sb + static_cast<int64_t>(token) * a.out.st +
                   static_cast<int64_t>(g * a.G + rho - token * a.G) * a.out.sh;
    *reinterpret_cast<x4*>(op + 4 * c2) = s_out[r2][c2];
  }
}

template <bool F16, int DH>
hipError_t launch_paged_join(const PagedAttnArgs& a, hipStream_t s) {
  constexpr int RPW = 256 / (DH / 4);
  hipLaunchKernelGGL((paged_attention_join_kernel<F16, DH>), dim3((a.rows_slot + RPW - 1) / RPW, a.slots), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <bool F16, int DH, int NW, bool CAP, bool BIAS, bool FAR = false>
hipError_t launch_paged_one(const PagedAttnArgs& a, hipStream_t s) {
  auto kern = paged_attention_kernel<F16, DH, NW, CAP, BIAS, FAR>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     PagedSmem<DH>::BYTES);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, dim3((a.slots + 7) / 8 * 8), dim3(64 * NW), PagedSmem<DH>::BYTES, s, a);
  hipError_t e = hipGetLastError();
  return e != hipSuccess || a.cut == nullptr ? e : launch_paged_join<F16, DH>(a, s);
}

template <bool F16, int DH, int NW, bool FAR>
hipError_t launch_paged_waves(const PagedAttnArgs& a, hipStream_t s) {
  if constexpr (FAR) {
    return a.sc.slopes != nullptr ? launch_paged_one<F16, DH, NW, true, true, true>(a, s) : launch_paged_one<F16, DH, NW, true, false, true>(a, s);
  } else {
    if (a.sc.cap_log2e > 0.f)
      return a.sc.slopes != nullptr ? launch_paged_one<F16, DH, NW, true, true>(a, s) : launch_paged_one<F16, DH, NW, true, false>(a, s);
    return a.sc.slopes != nullptr ? launch_paged_one<F16, DH, NW, false, true>(a, s) : launch_paged_one<F16, DH, NW, false, false>(a, s);
  }
}

template <bool F16, int DH, bool FAR = false>
hipError_t launch_paged(const PagedAttnArgs& a, int waves, hipStream_t s) {
  if constexpr (DH != 256) {   // (heads of 256 leave no registers for two wavefronts on a SIMD)
    if (waves == 8) return launch_paged_waves<F16, DH, 8, FAR>(a, s);
  }
  return launch_paged_waves<F16, DH, 4, FAR>(a, s);
}

}  // namespace

}  // namespace talon
