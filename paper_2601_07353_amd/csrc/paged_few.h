// Attention over a paged cache for few rows: at most 32 (token, head) rows of a KV head, as in decoding (one token of a group of
// heads, a few drafted ones).  Mathematics, scores, shares of key tiles and their join are those of paged_attention.h.
//
// Bound: the bytes of K and V.  One matrix instruction covers all rows, so the wavefronts of a workgroup share the keys instead:
// each has a run of 32-row tiles of its own, its own stage of K and V in LDS and waits for its own loads alone, with no barrier
// before the end of the piece; there the wavefronts' outputs are joined in LDS.  A wavefront loads K(t + 1) when the scores of
// tile t are formed and V(t + 1) when its values are added, so half of its stage is always on its way: 64 KB of a compute unit
// in eight wavefronts, more than the latency of the memory takes at its full rate.
// One workgroup per compute unit: 64 tokens at 8192 rows of 8 heads of 128 244 us (5.5 TB/s), of 64 203 us (5.3 TB/s; 252 with two
// workgroups, whose registers do not suffice).
#pragma once

#include "paged_attention.h"

namespace talon {

namespace {

constexpr int kFewTile = 32;

template <int DH>
struct FewSmem {
  static constexpr int NW = DH == 256 ? 4 : 8;
  static constexpr int STAGE = 2 * kFewTile * DH;                 // values: K, then V, of one wavefront
  static constexpr int POS_BYTES = NW * (kFewTile + 32) * 4;      // positions of a tile's rows and of the queries
  static constexpr int STAT_BYTES = 2 * NW * 32 * 4;              // maxima and denominators
  static constexpr int BYTES = NW * STAGE * 2 + POS_BYTES + STAT_BYTES;
};

template <int N>
__device__ __forceinline__ void wait_loads() {   // until at most N loads are on their way
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

template <bool F16, int DH, bool CAP, bool BIAS, bool FAR>
__global__ __launch_bounds__(64 * FewSmem<DH>::NW, DH == 256 ? 1 : 2) void paged_few_kernel(PagedAttnArgs a) {
  using ST = Storage<F16>;
  using x8 = typename ST::x8;
  using x4 = typename ST::x4;
  using SM = PagedSmem<DH>;
  using FS = FewSmem<DH>;
  constexpr bool MOD = CAP || BIAS;
  constexpr int NW = FS::NW;
  constexpr int DSTEPS = DH / 16;
  constexpr int DB = DH / 32;
  constexpr int CPR = DH / 8;
  constexpr int ROWS_PER_LOAD = 64 / CPR;
  constexpr int LOADS = kFewTile / ROWS_PER_LOAD;   // per tensor and tile
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31;
  const int h = lane >> 5;
  const ScoreArgs& sc = a.sc;
  const int G = a.G;
  Share w;
  if (!find_share<kFewTile, 32>(a, lane, &w)) return;
  int b = w.b, g = w.g, at = w.at, x = w.x, P = w.P, n = w.n;

  uint16_t* const sK = smem + wave * FS::STAGE;
  uint16_t* const sV = sK + kFewTile * DH;
  int* const s_pos = reinterpret_cast<int*>(smem + NW * FS::STAGE) + wave * (kFewTile + 32);
  float* const s_max = reinterpret_cast<float*>(reinterpret_cast<char*>(smem + NW * FS::STAGE) + FS::POS_BYTES);
  float* const s_den = s_max + NW * 32;
  const uint16_t* const k_pool = static_cast<const uint16_t*>(a.c.k);
  const uint16_t* const v_pool = static_cast<const uint16_t*>(a.c.v);
  const int lrow = lane / CPR, cslot = lane % CPR;

  bool first_piece = true;
  while (x < w.x_end) {
    int first_tile;
    const int tiles = tiles_of<kFewTile, 32>(sc, P, n, a.inv_g, 0, &first_tile);
    const Piece pc = next_piece(a, w, tiles, at, x);
    if (pc.from == pc.to) break;   // the share ends with what the row tile costs besides its tiles
    const int take = pc.to - pc.from;
    const int rows = n * G;
    const int kend = P + n;
    // this wavefront's tiles
    const int t_begin = first_tile + pc.from + take * wave / NW;
    const int t_end = first_tile + pc.from + take * (wave + 1) / NW;

    // ---- page entries of its first rows (a lane each, 64 pages), this lane's query
    uint32_t pages = 0;
    int pages_at = -1;
    auto load_pages = [&](int t) {
      const int at64 = (t * kFewTile) >> a.c.page_shift >> 6;
      if (at64 == pages_at) return;
      pages_at = at64;
      int i = at64 * 64 + lane;
      i = i < a.c.max_pages ? i : a.c.max_pages - 1;
      pages = static_cast<uint32_t>(a.c.table[static_cast<size_t>(b) * a.c.max_pages + i]);
    };
    const bool valid = l32 < rows;
    const int token = valid ? div_g(l32, a.inv_g) : 0;
    const int head = g * G + (valid ? l32 - token * G : 0);
    x8 bq[DSTEPS];
    const int p_own = P + offset_of(sc, b, token);
    float slope2 = 0.f;
    if constexpr (BIAS) slope2 = sc.slopes[head] * kLog2eF;
    {
      const uint16_t* qp = a.q.p + static_cast<int64_t>(b) * a.q.sb + static_cast<int64_t>(token) * a.q.st + static_cast<int64_t>(head) * a.q.sh + 8 * h;
      u32x4 qv[DSTEPS];
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) {
        qv[ds] = u32x4{0, 0, 0, 0};
        if (valid) qv[ds] = *reinterpret_cast<const u32x4*>(qp + 16 * ds);
      }
      load_pages(first_tile + pc.from + take * wave / NW);
      // (the compiler's wait for these loads stands here: inside the loop it would count the tile loads too)
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ds += 4) asm volatile("" : "+v"(qv[ds]), "+v"(qv[ds + 1]), "+v"(qv[ds + 2]), "+v"(qv[ds + 3]));
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) bq[ds] = __builtin_bit_cast(x8, qv[ds]);
    }
    const bool positions = sc.window > 0 || BIAS;
    int seen_to = sc.mask != nullptr || (positions && sc.offset != nullptr) ? P : P + 1;   // rows that every query sees: [seen_from, seen_to)
    int seen_from = 0;
    if (sc.window > 0) {
      int most = n - 1;
      if (sc.offset != nullptr) most = uniform(wave_max_i32(lane < n ? offset_of(sc, b, lane) : 0));
      seen_from = P + most - sc.window + 1;
    }

    uint32_t row_at[LOADS];
    auto rows_of = [&](int t) {
      load_pages(t);
      asm volatile("" : "+v"(pages));   // (waited for here where it was read anew)
      int key = t * kFewTile + l32;
      key = key < kend ? key : kend - 1;
      const uint32_t entry = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(((key >> a.c.page_shift) & 63) * 4, static_cast<int>(pages)));
      if (__ballot(entry >= a.c.num_pages) != 0ull && lane == 0) report(a.c, b, TALON_STATUS_BAD_PAGE);
      const int row = static_cast<int>(row_chunk(a.c, entry, key, g));
#pragma unroll
      for (int i = 0; i < LOADS; ++i) row_at[i] = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute((i * ROWS_PER_LOAD + lrow) * 4, row));
    };
    auto load_k = [&]() {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        global_to_lds(chunk_at(k_pool, row_at[i] + (cslot ^ SM::kswz(i * ROWS_PER_LOAD + lrow))), sK + i * ROWS_PER_LOAD * DH);
    };
    auto load_v = [&]() {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        global_to_lds(chunk_at(v_pool, row_at[i] + (cslot ^ SM::vswz(i * ROWS_PER_LOAD + lrow))), sV + i * ROWS_PER_LOAD * DH);
    };
    auto reads_done = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

    float m_run = kNoScore, l_run = 0.f;
    floatx16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = 0.f;

    // Rows of tile t that this lane's query sees, as bits; the positions of the tile's rows in s_pos.
    auto seen_bits = [&](int t) {
      const uint32_t bits = static_cast<uint32_t>(seen_rows(sc, b, token, P, t * kFewTile, kend));
      if (positions && lane < kFewTile) {
        const int key = t * kFewTile + lane;
        s_pos[lane] = key >= P && key < kend ? P + offset_of(sc, b, key - P) : key;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      return bits;
    };

    if (t_begin < t_end) {
      rows_of(t_begin);
      load_k();
      load_v();
    }
#pragma unroll 1
    for (int t = t_begin; t < t_end; ++t) {
      const bool more = t + 1 < t_end;
      const bool in_part = (t + 1) * kFewTile > seen_to || t * kFewTile < seen_from;
      wait_loads<LOADS>();          // K(t)
      floatx16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
      {
        const uint16_t* krow = sK + l32 * DH;
        const int ksw = SM::kswz(l32);
#pragma unroll
        for (int ds = 0; ds < DSTEPS; ++ds) {
          const x8 ak = __builtin_bit_cast(x8, *reinterpret_cast<const uint4*>(krow + ((2 * ds + h) ^ ksw) * 8));
          s = ST::mfma(ak, bq[ds], s);
        }
      }
      reads_done();
      if (more) {
        rows_of(t + 1);
        reads_done();
        load_k();
      }
      if constexpr (FAR) {   // (see paged_attention.h)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = sc.cap_log2e * tanh_of(s[r] * sc.cap_in);
      } else if constexpr (CAP) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(s[r] * sc.cap_in);
          s[r] = __builtin_fmaf(-2.f * sc.cap_log2e, __builtin_amdgcn_rcpf(1.f + e), sc.cap_log2e);
        }
      } else if constexpr (BIAS) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= sc.scale_log2e;
      }
      uint32_t bits = ~0u;
      if (!in_part) {
        if constexpr (BIAS) {
          const float bias0 = slope2 * static_cast<float>(p_own - t * kFewTile - 4 * h);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const float bias = __builtin_fmaf(slope2, static_cast<float>(8 * q4), -bias0);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * q4 + e] += __builtin_fmaf(slope2, static_cast<float>(e), bias);
          }
        }
      } else {
        bits = seen_bits(t);
        const int window = sc.window > 0 ? sc.window : 0x7FFFFFFF;
        const uint32_t mine = bits >> (4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          bool seen = (mine >> (8 * (r / 4) + r % 4)) & 1u;
          if (positions) {
            const int apart = p_own - s_pos[8 * (r / 4) + 4 * h + r % 4];
            seen = seen && apart < window;
            if constexpr (BIAS) s[r] = __builtin_fmaf(-slope2, fabsf(static_cast<float>(apart)), s[r]);
          }
          s[r] = seen ? s[r] : kNoScore;
        }
      }
      // ---- softmax
      float mx = kNoScore;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      {
        const int mi = __float_as_int(mx);
        const auto sw = __builtin_amdgcn_permlane32_swap(mi, mi, false, false);
        mx = fmaxf(__int_as_float(static_cast<int>(sw[0])), __int_as_float(static_cast<int>(sw[1])));
      }
      const float m_new = fmaxf(m_run, MOD ? mx : mx * sc.scale_log2e);
      const float m_safe = m_new == kNoScore ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_safe);
      m_run = m_new;
      if (__ballot(alpha != 1.f) != 0ull) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      }
      x8 pb[2];
      float sum = 0.f;
#pragma unroll
      for (int sp = 0; sp < 2; ++sp)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = s[8 * sp + e];
          const float p = __builtin_amdgcn_exp2f(MOD ? v - m_safe : __builtin_fmaf(v, sc.scale_log2e, -m_safe));
          sum += p;
          pb[sp][e] = static_cast<typename ST::x1>(p);
        }
      l_run = l_run * alpha + sum;
      if (more) wait_loads<LOADS>(); else wait_loads<0>();   // V(t)
      if (in_part) {   // values that are no finite numbers must not reach a row that does not see them
        uint32_t bad_rows = 0;
        uint4* const v = reinterpret_cast<uint4*>(sV);
#pragma unroll 1
        for (int c = 0; c < LOADS; ++c) {
          uint4 u = v[c * 64 + lane];
          uint32_t* const word = reinterpret_cast<uint32_t*>(&u);
          uint32_t found = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bad = ST::not_finite(word[e]);
            found |= bad;
            if (bad & 1u) word[e] &= 0xFFFF0000u;
            if (bad & 2u) word[e] &= 0x0000FFFFu;
          }
          if (found) v[c * 64 + lane] = u;
          unsigned long long lanes = __ballot(found != 0u);
          while (lanes != 0ull) {
            const int l = __ffsll(static_cast<long long>(lanes)) - 1;
            lanes &= lanes - 1ull;
            bad_rows |= 1u << (c * ROWS_PER_LOAD + l / CPR);
          }
        }
        if (bad_rows != 0u) {
          uint32_t seen = bits & bad_rows;
          if (sc.window > 0)
            for (int k = 0; k < kFewTile; ++k)
              if (p_own - s_pos[k] >= sc.window) seen &= ~(1u << k);
          if (seen != 0u) l_run = __builtin_nanf("");
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      // ---- O^T += V^T . P^T
      {
        const int i16 = lane & 15;
        const int dhblk = (lane >> 4) & 1;
        const int vrow_l = 4 * h + (i16 >> 2);
        const int vsw = SM::vswz(vrow_l);
        const int vch = 2 * dhblk + ((i16 & 3) >> 1);
        const int vsub = (i16 & 1) * 4;
#pragma unroll
        for (int sp = 0; sp < 2; ++sp)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const uint16_t* vp = sV + (16 * sp + vrow_l) * DH + ((4 * db + vch) ^ vsw) * 8 + vsub;
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vp));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(vp + 8 * DH));
            o[db] = ST::mfma(__builtin_bit_cast(x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), pb[sp], o[db]);
          }
      }
      reads_done();
      if (more) load_v();
    }

    // ---- the wavefronts' outputs joined: chunk c (4 values) of row r at chunk c ^ (r % 16) of the row, so that the rows of a store
    // fall on different banks
    {
      const int li = __float_as_int(l_run);
      const auto sw = __builtin_amdgcn_permlane32_swap(li, li, false, false);
      const float l_tot = __int_as_float(static_cast<int>(sw[0])) + __int_as_float(static_cast<int>(sw[1]));
      float* const own = reinterpret_cast<float*>(sK);
      if (valid) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<float4*>(own + l32 * DH + ((8 * db + 2 * q4 + h) ^ (l32 & 15)) * 4) =
                make_float4(o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
        if (h == 0) {
          s_max[wave * 32 + l32] = m_run;
          s_den[wave * 32 + l32] = l_tot;
        }
      }
    }
    __syncthreads();
    const bool whole = take == tiles;
    for (int u = tid; u < rows * (DH / 4); u += 64 * NW) {
      const int r = u / (DH / 4), c = u - r * (DH / 4);
      float M = kNoScore;
#pragma unroll
      for (int v = 0; v < NW; ++v) M = fmaxf(M, s_max[v * 32 + r]);
      const float safe = M == kNoScore ? 0.f : M;
      float den = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float f = __builtin_amdgcn_exp2f(s_max[v * 32 + r] - safe);
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem + v * FS::STAGE) + r * DH + (c ^ (r & 15)) * 4);
        den = __builtin_fmaf(f, s_den[v * 32 + r], den);
        acc.x = __builtin_fmaf(f, y.x, acc.x); acc.y = __builtin_fmaf(f, y.y, acc.y);
        acc.z = __builtin_fmaf(f, y.z, acc.z); acc.w = __builtin_fmaf(f, y.w, acc.w);
      }
      if (whole) {
        const int token_e = div_g(r, a.inv_g);
        const int head_e = g * G + r - token_e * G;
        const float inv = den == 0.f ? 0.f : 1.f / den;   // a row that sees nothing
        x4 v;
        v[0] = static_cast<typename ST::x1>(acc.x * inv);
        v[1] = static_cast<typename ST::x1>(acc.y * inv);
        v[2] = static_cast<typename ST::x1>(acc.z * inv);
        v[3] = static_cast<typename ST::x1>(acc.w * inv);
        *reinterpret_cast<x4*>(a.out.p + static_cast<int64_t>(b) * a.out.sb + static_cast<int64_t>(token_e) * a.out.st + static_cast<int64_t>(head_e) * a.out.sh + 4 * c) = v;
        if (a.lse != nullptr && c == 0)
          a.lse[(static_cast<size_t>(b) * sc.N + token_e) * (a.Hkv * G) + head_e] = (M + __builtin_amdgcn_logf(den)) * kLn2F;
      } else {
        const size_t slot = static_cast<size_t>(2 * w.share + (first_piece ? 0 : 1));
        *reinterpret_cast<float4*>(a.part_o + ((slot * (DH / 8) + (c >> 1)) * a.rows_slot + r) * 8 + 4 * (c & 1)) = acc;
        if (c == 0) {
          a.part_m[slot * a.rows_slot + r] = M;
          a.part_l[slot * a.rows_slot + r] = den;
        }
      }
    }
    if (pc.from == 0 && pc.to < tiles && tid == 0) a.cut[w.share] = make_int4(b * a.Hkv + g, 0, rows, pc.last | (first_piece ? 0 : 1 << 30));

    // ---- on to the next KV head or sequence
    x += pc.units;
    at = 0;
    first_piece = false;
    if (x < w.x_end) {
      if (++g == a.Hkv) {
        g = 0;
        do {   // (x < x_end: there is another sequence with new tokens)
          ++b;
          clamped_lengths(a.c, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N, &P, &n);
        } while (n == 0);
      }
      __syncthreads();   // the stages are free
    }
  }
}

template <bool F16, int DH, bool CAP, bool BIAS, bool FAR = false>
hipError_t launch_few_one(const PagedAttnArgs& a, hipStream_t s) {
  auto kern = paged_few_kernel<F16, DH, CAP, BIAS, FAR>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     FewSmem<DH>::BYTES);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, dim3((a.slots + 7) / 8 * 8), dim3(64 * FewSmem<DH>::NW), FewSmem<DH>::BYTES, s, a);
  hipError_t e = hipGetLastError();
  return e != hipSuccess || a.cut == nullptr ? e : launch_paged_join<F16, DH>(a, s);
}

template <bool F16, int DH, bool FAR = false>
hipError_t launch_few(const PagedAttnArgs& a, hipStream_t s) {
  if constexpr (FAR) {
    return a.sc.slopes != nullptr ? launch_few_one<F16, DH, true, true, true>(a, s) : launch_few_one<F16, DH, true, false, true>(a, s);
  } else {
    if (a.sc.cap_log2e > 0.f) return a.sc.slopes != nullptr ? launch_few_one<F16, DH, true, true>(a, s) : launch_few_one<F16, DH, true, false>(a, s);
    return a.sc.slopes != nullptr ? launch_few_one<F16, DH, false, true>(a, s) : launch_few_one<F16, DH, false, false>(a, s);
  }
}

}  // namespace

}  // namespace talon
