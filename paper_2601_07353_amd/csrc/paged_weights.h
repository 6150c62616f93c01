// Attention weight that the rows of a paged cache receive from the new tokens (what an eviction goes by), included by one source
// per storage type:
//
//   out[b][g][j] = decay * prior[b][g][j] + sum over new tokens i and heads h of group g of exp(x_ihj - lse_ih)
//
// with the scores x and the denominators lse of the attention call.  The denominators are known, so one product is enough and
// nothing is rounded to 16 bits on the way: the probabilities are summed as they come out of the exponential, in fp32.
//
// Both kernels form S[query][key] = Q . K^T with a key per lane and the queries in registers, so that a lane adds up its own
// key and only the two halves of a wavefront (16 queries of 32 each) are added across lanes.  No two workgroups write one value:
// there are no atomics, and the order of the additions is fixed.
#pragma once

#include "paged_attention.h"

namespace talon {

namespace {

// Whether new token i sees row `key` (at position `pos`), but for the window.
__device__ __forceinline__ bool sees_row(const ScoreArgs& s, int b, int i, int P, int key) {
  if (key < P) return true;
  if (s.mask == nullptr) return key - P <= i;
  const int d = key - P;
  return (s.mask[(static_cast<size_t>(b) * s.N + i) * s.words + (d >> 6)] >> (d & 63)) & 1u;
}

constexpr int kNobody = -1;   // token of a row that counts nothing: behind the last query, or of a token whose lse is +inf

constexpr int kQueryTile = 128;

// A query's entry in the tables of a tile: lse (base 2), token, position, slope (base 2).
struct QueryTables {
  float lse[kQueryTile];
  int token[kQueryTile];
  int pos[kQueryTile];
  float slope[kQueryTile];
};

// Sum over the 16 queries of this half in a 32 x 32 block of products: register r is query 8 * (r / 4) + 4 * h + r % 4.  `whole`: each
// of them sees each key of the block; `everyone`: each of the `count` queries that there are counts.  (One that does not may have any
// score, a NaN too: x = score - inf is not relied on.)
template <bool CAP, bool BIAS>
__device__ __forceinline__ float block_sum(const PagedAttnArgs& a, floatx16 s, const QueryTables& t, int q0, int h, bool whole, bool everyone, int b, int P, int key,
                                           int pos, bool real, int count) {
  const ScoreArgs& sc = a.sc;
  if constexpr (CAP) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = sc.cap_log2e * tanh_of(s[r] * sc.cap_in);
  }
  float x[16];
#pragma unroll
  for (int q4 = 0; q4 < 4; ++q4) {
    const int at = q0 + 8 * q4 + 4 * h;
    const float4 l4 = *reinterpret_cast<const float4*>(&t.lse[at]);
    const float ls[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * q4 + e] = CAP ? s[4 * q4 + e] - ls[e] : __builtin_fmaf(s[4 * q4 + e], sc.scale_log2e, -ls[e]);
    if constexpr (BIAS) {
      const int4 p4 = *reinterpret_cast<const int4*>(&t.pos[at]);
      const float4 f4 = *reinterpret_cast<const float4*>(&t.slope[at]);
      const int ps[4] = {p4.x, p4.y, p4.z, p4.w};
      const float fs[4] = {f4.x, f4.y, f4.z, f4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * q4 + e] = __builtin_fmaf(-fs[e], fabsf(static_cast<float>(ps[e] - pos)), x[4 * q4 + e]);
    }
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if (whole && everyone && count == 32) {   // uniform; nothing else in the way of the exponentials
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[r % 4] += __builtin_amdgcn_exp2f(x[r]);
  } else if (whole && everyone) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r / 4) < count) sum[r % 4] += 8 * (r / 4) + 4 * h + r % 4 < count ? __builtin_amdgcn_exp2f(x[r]) : 0.f;
  } else if (whole) {
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      if (8 * q4 >= count) continue;
      const int4 t4 = *reinterpret_cast<const int4*>(&t.token[q0 + 8 * q4 + 4 * h]);
      const int ts[4] = {t4.x, t4.y, t4.z, t4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += ts[e] != kNobody ? __builtin_amdgcn_exp2f(x[4 * q4 + e]) : 0.f;
    }
  } else {
    const int window = sc.window > 0 ? sc.window : 0x7FFFFFFF;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int at = q0 + 8 * q4 + 4 * h;
      const int4 t4 = *reinterpret_cast<const int4*>(&t.token[at]);
      const int4 p4 = *reinterpret_cast<const int4*>(&t.pos[at]);
      const int ts[4] = {t4.x, t4.y, t4.z, t4.w}, ps[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool seen = real && ts[e] != kNobody && ps[e] - pos < window && sees_row(sc, b, ts[e], P, key);
        sum[e] += seen ? __builtin_amdgcn_exp2f(x[4 * q4 + e]) : 0.f;
      }
    }
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__device__ __forceinline__ float both_halves(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(static_cast<int>(sw[0])) + __int_as_float(static_cast<int>(sw[1]));
}

// ---- many queries: a workgroup of eight wavefronts owns 64 rows of the cache and streams the queries that may see them through LDS,
// 128 (token, head) rows a tile, two stages.  A wavefront has 32 of the rows, whose keys stay in its registers, and 32 queries of
// every tile; the four that share rows add theirs in LDS at the end.  Bound: the exponentials (a quarter of the vector rate) and
// the matrix product, which hardly run at the same time.  The time of a workgroup is short against the call's, so that the last
// ones cost little: 512 tokens at 8192 rows 71 us, against 77 with four wavefronts and tiles of 64 rows and 82 with four wavefronts
// on 128 rows.

template <int DH>
struct WeighSmem {
  static constexpr int STAGE = kQueryTile * DH;
  static constexpr int BYTES = 2 * STAGE * 2 + 2 * static_cast<int>(sizeof(QueryTables)) + 3 * kWeighRows * 4;
};

template <bool F16, int DH, bool CAP, bool BIAS>
__global__ __launch_bounds__(kWeighThreads, DH == 256 ? 2 : 4) void paged_weights_kernel(PagedWeightArgs wa) {
  using ST = Storage<F16>;
  using x8 = typename ST::x8;
  using SM = PagedSmem<DH>;
  const PagedAttnArgs& a = wa.a;
  constexpr int CPR = DH / 8;
  constexpr int DSTEPS = DH / 16;
  constexpr int QT = kQueryTile;
  constexpr int ROWS_PER_LOAD = 64 / CPR;
  constexpr int LOADS = QT / 8 / ROWS_PER_LOAD;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  QueryTables* const s_t = reinterpret_cast<QueryTables*>(smem + 2 * WeighSmem<DH>::STAGE);
  float* const s_part = reinterpret_cast<float*>(s_t + 2);
  const ScoreArgs& sc = a.sc;
  const int b = blockIdx.z, g = blockIdx.y;
  int P, n;
  clamped_lengths(a.c, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N, &P, &n);
  if (blockIdx.x == 0 && g == 0 && threadIdx.x == 0) report_table_end(a.c, b, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N);
  const int len = P + n;
  const int key0 = static_cast<int>(blockIdx.x) * kWeighRows;
  if (key0 >= len) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int G = a.G;

  // ---- this lane's key (a row past the end reads the last one; it gets nothing)
  const int key = key0 + 32 * (wave & 1) + l32;
  const int q0 = 32 * (wave >> 1);   // its queries of a tile
  const bool real = key < len;
  int pos = key;
  x8 bk[DSTEPS];
  {
    const int row = real ? key : len - 1;
    const uint32_t entry = page_entry(a.c, b, row);
    if (real && key >= P) pos = P + offset_of(sc, b, key - P);
    if (__ballot(entry >= a.c.num_pages) != 0ull && lane == 0) report(a.c, b, TALON_STATUS_BAD_PAGE);
    const uint16_t* kp = chunk_at(static_cast<const uint16_t*>(a.c.k), row_chunk(a.c, entry, row, g) + h);
    u32x4 kv[DSTEPS];
#pragma unroll
    for (int ds = 0; ds < DSTEPS; ++ds) kv[ds] = *reinterpret_cast<const u32x4*>(kp + 16 * ds);
    // (the compiler's wait for these loads stands here: inside the loop it would count the queries' loads too)
#pragma unroll
    for (int ds = 0; ds < DSTEPS; ds += 4) asm volatile("" : "+v"(kv[ds]), "+v"(kv[ds + 1]), "+v"(kv[ds + 2]), "+v"(kv[ds + 3]));
#pragma unroll
    for (int ds = 0; ds < DSTEPS; ++ds) bk[ds] = __builtin_bit_cast(x8, kv[ds]);
  }

  // ---- the queries that may see a row of this workgroup: tokens [i_from, i_to)
  const int last_key = key0 + kWeighRows < len ? key0 + kWeighRows - 1 : len - 1;
  const int i_from = sc.mask == nullptr && key0 > P ? key0 - P : 0;
  int i_to = n;
  if (sc.window > 0 && sc.offset == nullptr) {   // P + i - last_key < window
    const long long most = static_cast<long long>(last_key) - P + sc.window;
    i_to = most < i_to ? (most < 0 ? 0 : static_cast<int>(most)) : i_to;
  }
  const int r_end = i_to * G;
  const int rows = n * G;
  // rows of the workgroup are seen by every query from token seen_from on, up to (and without) token seen_to
  const int seen_from = last_key < P ? 0 : (sc.mask != nullptr ? 0x7FFFFFFF : last_key - P);
  const bool near = sc.window == 0 || (sc.offset == nullptr && static_cast<long long>(P) + n - key0 <= sc.window);

  const uint16_t* const qb = a.q.p + static_cast<int64_t>(b) * a.q.sb + static_cast<int64_t>(g) * G * a.q.sh;
  const uint32_t token_chunks = static_cast<uint32_t>(a.q.st / 8), head_chunks = static_cast<uint32_t>(a.q.sh / 8);
  float lse_next = 0.f, slope_next = 0.f;
  int token_next = kNobody, off_next = 0;   // (as loaded: used when the next tile has landed)
  auto load_queries = [&](int r0, int st) {
    // (a lane finds one of this wavefront's 16 rows, the lanes of a load take their rows' places from it: integer products are slow)
    int rho_l = r0 + wave * 16 + (lane & 15);
    rho_l = rho_l < rows ? rho_l : rows - 1;
    const int token_l = div_g(rho_l, a.inv_g);
    const int place = static_cast<int>(static_cast<uint32_t>(token_l) * token_chunks + static_cast<uint32_t>(rho_l - token_l * G) * head_chunks);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = (wave * LOADS + i) * ROWS_PER_LOAD;
      const uint32_t chunk = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute((i * ROWS_PER_LOAD + lane / CPR) * 4, place));
      global_to_lds(chunk_at(qb, chunk + ((lane % CPR) ^ SM::kswz(u + lane / CPR))), smem + st * WeighSmem<DH>::STAGE + u * DH);
    }
    if (tid < QT) {
      const int rho = r0 + tid;
      token_next = kNobody;
      lse_next = __builtin_huge_valf();   // weight 0
      if (rho < r_end) {
        token_next = div_g(rho, a.inv_g);
        const int head = g * G + rho - token_next * G;
        lse_next = a.lse[(static_cast<size_t>(b) * sc.N + token_next) * (a.Hkv * G) + head];
        off_next = token_next;
        if (sc.offset != nullptr) off_next = sc.offset[static_cast<size_t>(b) * sc.N + token_next];
        if constexpr (BIAS) slope_next = sc.slopes[head];
      }
    }
  };
  auto store_tables = [&](int st) {
    if (tid < QT) {
      s_t[st].lse[tid] = lse_next * kLog2eF;
      s_t[st].token[tid] = lse_next == __builtin_huge_valf() ? kNobody : token_next;
      s_t[st].pos[tid] = P + (off_next < 0 ? 0 : (off_next < kMostOffset ? off_next : kMostOffset));
      if constexpr (BIAS) s_t[st].slope[tid] = slope_next * kLog2eF;
    }
  };
  auto landed = [&]() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  // sums of a tile, of sixteen tiles, and of those: what rounding adds up to stays small over thousands of queries
  float acc = 0.f, sum = 0.f;
  int r0 = i_from * G;
  if (r0 < r_end) {
    load_queries(r0, 0);
    store_tables(0);
  }
  landed();
#pragma unroll 1
  for (int st = 0, count = 1; r0 < r_end; r0 += QT, st ^= 1, ++count) {
    const bool more = r0 + QT < r_end;
    if (more) load_queries(r0 + QT, st ^ 1);
    const bool whole = near && r0 + QT <= r_end && div_g(r0, a.inv_g) >= seen_from;
    floatx16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
    const int row = q0 + l32;
    const int swz = SM::kswz(row);
    const bool everyone = __ballot(s_t[st].token[row] == kNobody) == 0ull;
#pragma unroll
    for (int ds = 0; ds < DSTEPS; ++ds) {
      const x8 aq = __builtin_bit_cast(x8, *reinterpret_cast<const uint4*>(smem + st * WeighSmem<DH>::STAGE + row * DH + ((2 * ds + h) ^ swz) * 8));
      s = ST::mfma(aq, bk[ds], s);
    }
    acc += block_sum<CAP, BIAS>(a, s, s_t[st], q0, h, whole, everyone, b, P, key, pos, real, 32);
    if ((count & 15) == 0) {
      sum += acc;
      acc = 0.f;
    }
    if (more) store_tables(st ^ 1);
    landed();
  }
  float total = both_halves(sum + acc);
  if (q0 != 0 && h == 0) s_part[32 * (wave - 2) + l32] = total;
  __syncthreads();
  if (q0 == 0 && h == 0 && real) {
#pragma unroll
    for (int v = 0; v < 3; ++v) total += s_part[32 * (2 * v + wave) + l32];
    const size_t at = static_cast<size_t>(b) * wa.stride_b + static_cast<size_t>(g) * wa.stride_h + key;
    wa.out[at] = total + (wa.prior != nullptr && key < P ? wa.decay * wa.prior[at] : 0.f);
  }
}

// ---- few queries (at most 32 (token, head) rows of a KV head): they stay in registers and K streams through LDS, 32 rows a tile and
// wavefront, two stages each, in the shares of paged_attention.h (nothing is cut that would have to be joined, and no wavefront waits
// for another).  Bound: the bytes of K; 8 tokens at 16384 rows of 8 heads of 128 61 to 63 us (4.4 TB/s), 64 at 8192 228 us (4.7 TB/s).
// One workgroup per compute unit, also for heads of 64: 8 at 16384 31 us, 37 with two.
template <int DH>
struct WeighFewSmem {
  static constexpr int NW = DH == 256 ? 4 : 8;
  static constexpr int STAGE = 32 * DH;
  static constexpr int BYTES = NW * 2 * STAGE * 2 + NW * 2 * 64 * 4 + static_cast<int>(sizeof(QueryTables)) * NW;
};

template <bool F16, int DH, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * WeighFewSmem<DH>::NW, DH == 256 ? 1 : 2) void paged_weights_few_kernel(PagedWeightArgs wa) {
  using ST = Storage<F16>;
  using x8 = typename ST::x8;
  using SM = PagedSmem<DH>;
  using WS = WeighFewSmem<DH>;
  const PagedAttnArgs& a = wa.a;
  constexpr int NW = WS::NW;
  constexpr int CPR = DH / 8;
  constexpr int DSTEPS = DH / 16;
  constexpr int ROWS_PER_LOAD = 64 / CPR;
  constexpr int LOADS = 32 / ROWS_PER_LOAD;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  const ScoreArgs& sc = a.sc;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int G = a.G;
  Share w;
  if (!find_share<32, 32, true>(a, lane, &w)) return;
  int b = w.b, g = w.g, at = w.at, x = w.x, P = w.P, n = w.n;
  uint16_t* const s_k = smem + wave * 2 * WS::STAGE;
  float* const s_prior = reinterpret_cast<float*>(smem + NW * 2 * WS::STAGE) + wave * 2 * 64;
  QueryTables& s_t = *(reinterpret_cast<QueryTables*>(reinterpret_cast<float*>(smem + NW * 2 * WS::STAGE) + NW * 2 * 64) + wave);
  const uint16_t* const k_pool = static_cast<const uint16_t*>(a.c.k);

  while (x < w.x_end) {
    const int len = P + n;
    const int tiles = (len + 31) / 32;   // (all rows have a weight, also those that a window hides)
    const Piece pc = next_piece(a, w, tiles, at, x);
    if (pc.from == pc.to) break;
    const int take = pc.to - pc.from;
    const int t_begin = pc.from + take * wave / NW, t_end = n == 0 ? t_begin : pc.from + take * (wave + 1) / NW;
    const int rows = n * G;
    const float* const prior = wa.prior != nullptr ? wa.prior + static_cast<size_t>(b) * wa.stride_b + static_cast<size_t>(g) * wa.stride_h : nullptr;
    float* const out = wa.out + static_cast<size_t>(b) * wa.stride_b + static_cast<size_t>(g) * wa.stride_h;

    if (n == 0) {   // without new tokens the weights only decay
      for (int key = pc.from * 32 + tid; key < pc.to * 32 && key < len; key += 64 * NW) out[key] = prior != nullptr ? wa.decay * prior[key] : 0.f;
    }
    uint32_t pages = 0;
    int pages_at = -1;
    auto load_tile = [&](int t, int st) {
      const int at64 = (t * 32) >> a.c.page_shift >> 6;
      if (at64 != pages_at) {
        pages_at = at64;
        int i = at64 * 64 + lane;
        i = i < a.c.max_pages ? i : a.c.max_pages - 1;
        pages = static_cast<uint32_t>(a.c.table[static_cast<size_t>(b) * a.c.max_pages + i]);
        asm volatile("" : "+v"(pages));   // waited for here
      }
      int row = t * 32 + l32;
      row = row < len ? row : len - 1;
      const uint32_t entry = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(((row >> a.c.page_shift) & 63) * 4, static_cast<int>(pages)));
      if (__ballot(entry >= a.c.num_pages) != 0ull && lane == 0) report(a.c, b, TALON_STATUS_BAD_PAGE);
      const int chunk = static_cast<int>(row_chunk(a.c, entry, row, g));
      uint32_t from[LOADS];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) from[i] = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute((i * ROWS_PER_LOAD + lane / CPR) * 4, chunk));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int u = i * ROWS_PER_LOAD;
        global_to_lds(chunk_at(k_pool, from[i] + ((lane % CPR) ^ SM::kswz(u + lane / CPR))), s_k + st * WS::STAGE + u * DH);
      }
      if (prior != nullptr && P > 0) {
        int key = t * 32 + l32;
        key = key < P ? key : P - 1;
        const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(s_prior + st * 64)));
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(prior + key), "s"(lds) : "memory", "m0");
      }
    };

    // ---- the queries, their denominators and places
    x8 aq[DSTEPS];
    bool everyone;
    {
      const bool valid = l32 < rows;
      const int token = valid ? div_g(l32, a.inv_g) : 0;
      const int head = g * G + (valid ? l32 - token * G : 0);
      const uint16_t* qp = a.q.p + static_cast<int64_t>(b) * a.q.sb + static_cast<int64_t>(token) * a.q.st + static_cast<int64_t>(head) * a.q.sh + 8 * h;
      u32x4 qv[DSTEPS];
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) {
        qv[ds] = u32x4{0, 0, 0, 0};
        if (valid) qv[ds] = *reinterpret_cast<const u32x4*>(qp + 16 * ds);
      }
      float lse = __builtin_huge_valf();
      if (h == 0) {
        if (valid) lse = a.lse[(static_cast<size_t>(b) * sc.N + token) * (a.Hkv * G) + head];
        s_t.lse[l32] = lse * kLog2eF;
        s_t.token[l32] = lse == __builtin_huge_valf() ? kNobody : token;
        s_t.pos[l32] = P + offset_of(sc, b, token);
        if constexpr (BIAS) s_t.slope[l32] = valid ? sc.slopes[head] * kLog2eF : 0.f;
      }
      // (the compiler's wait for these loads stands here: inside the loop it would count the tile loads too)
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ds += 4) asm volatile("" : "+v"(qv[ds]), "+v"(qv[ds + 1]), "+v"(qv[ds + 2]), "+v"(qv[ds + 3]));
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) aq[ds] = __builtin_bit_cast(x8, qv[ds]);
      everyone = __ballot(h == 0 && valid && lse == __builtin_huge_valf()) == 0ull;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const bool loads_prior = prior != nullptr && P > 0;
    const bool positions = sc.window > 0 || BIAS;
    if (t_begin < t_end) load_tile(t_begin, 0);
    if (t_begin + 1 < t_end) load_tile(t_begin + 1, 1);
#pragma unroll 1
    for (int t = t_begin, st = 0; t < t_end; ++t, st ^= 1) {
      if (t + 1 < t_end) {   // the loads of the next tile may be on their way
        if (loads_prior) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS + 1) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      const int key = t * 32 + l32;
      const bool real = key < len;
      int pos = key;
      if (positions && real && key >= P) pos = P + offset_of(sc, b, key - P);
      floatx16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
      const uint16_t* krow = s_k + st * WS::STAGE + l32 * DH;
      const int swz = SM::kswz(l32);
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) {
        const x8 bk = __builtin_bit_cast(x8, *reinterpret_cast<const uint4*>(krow + ((2 * ds + h) ^ swz) * 8));
        s = ST::mfma(aq[ds], bk, s);
      }
      const float before = loads_prior ? s_prior[st * 64 + l32] : 0.f;
      // every query sees the tile whole where it lies in the prefix and nothing hides it (rows without a query have weight 0)
      const bool whole = (t + 1) * 32 <= P && sc.window == 0;
      const float total = both_halves(block_sum<CAP, BIAS>(a, s, s_t, 0, h, whole, everyone, b, P, key, pos, real, rows));
      if (h == 0 && real) out[key] = total + (key < P ? wa.decay * before : 0.f);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the stage is free
      if (t + 2 < t_end) load_tile(t + 2, st);
    }

    // ---- on to the next KV head or sequence
    x += pc.units;
    at = 0;
    if (x < w.x_end && ++g == a.Hkv) {
      g = 0;
      do {
        ++b;
        clamped_lengths(a.c, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N, &P, &n);
      } while (P + n == 0);
    }
  }
}

template <bool F16, int DH, bool CAP, bool BIAS>
hipError_t launch_weights_one(const PagedWeightArgs& wa, bool few, hipStream_t s) {
  if (few) {
    auto kern = paged_weights_few_kernel<F16, DH, CAP, BIAS>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                       WeighFewSmem<DH>::BYTES);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((wa.a.slots + 7) / 8 * 8), dim3(64 * WeighFewSmem<DH>::NW), WeighFewSmem<DH>::BYTES, s, wa);
  } else {
    const int most = wa.a.sc.max_prefix_len + wa.a.sc.N < wa.a.c.capacity ? wa.a.sc.max_prefix_len + wa.a.sc.N : wa.a.c.capacity;
    auto kern = paged_weights_kernel<F16, DH, CAP, BIAS>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                       WeighSmem<DH>::BYTES);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((most + kWeighRows - 1) / kWeighRows, wa.a.Hkv, wa.a.B), dim3(kWeighThreads), WeighSmem<DH>::BYTES, s, wa);
  }
  return hipGetLastError();
}

template <bool F16, int DH>
hipError_t launch_weights_dh(const PagedWeightArgs& wa, bool few, hipStream_t s) {
  const bool cap = wa.a.sc.cap_log2e > 0.f, bias = wa.a.sc.slopes != nullptr;
  if (cap) return bias ? launch_weights_one<F16, DH, true, true>(wa, few, s) : launch_weights_one<F16, DH, true, false>(wa, few, s);
  return bias ? launch_weights_one<F16, DH, false, true>(wa, few, s) : launch_weights_one<F16, DH, false, false>(wa, few, s);
}

template <bool F16>
hipError_t launch_weights(const PagedWeightArgs& wa, int Dh, bool few, hipStream_t s) {
  switch (Dh) {
    case 64: return launch_weights_dh<F16, 64>(wa, few, s);
    case 128: return launch_weights_dh<F16, 128>(wa, few, s);
    default: return launch_weights_dh<F16, 256>(wa, few, s);
  }
}

}  // namespace

}  // namespace talon
