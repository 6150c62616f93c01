// Attention weight that the rows of a paged cache receive from the new tokens (what an eviction goes by):
//
//   out[b][g][j] = decay * prior[b][g][j] + sum over new tokens i and heads h of group g of exp(x_ihj - lse_ih)
//
// with the scores x and the denominators lse of the attention call.  The denominators are known, so one product is enough and
// nothing is rounded to 16 bits on the way: the probabilities are summed as they come out of the exponential, in fp32.
//
// A workgroup of four wavefronts owns 128 rows of one (sequence, KV head), 32 a wavefront, whose keys stay in registers, and
// streams the queries that may see them, 64 (token, head) rows (32 of heads of 256) at a time, through LDS (two stages).  The product is formed
// transposed, S^T[key][query] = K . Q^T: a lane adds up 16 keys over its queries; the 32 lanes are added at the end.  No two
// workgroups write one value, so there are no atomics and the order of the additions is fixed.  Bound: K's bytes for a few
// queries, the exponentials and the matrix product for many.
#include "paged_device.h"

namespace talon {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kKeysPerWg = 128;

template <bool F16>
__device__ __forceinline__ floatx16 product(uint4 k, uint4 q, floatx16 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, k), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}

// tanh(x) to a few units in the last place, also near 0, where 1 - 2 / (1 + e^(2x)) keeps no more than its absolute accuracy
// (the sums here stay in fp32, so the scores have to be as good): the continued fraction x / (1 + x^2 / (3 + x^2 / (5 + ...)))
// of Lambert, cut behind 13 and written as a quotient; its error is below 2^-24 for |x| <= 2, beyond the other form is exact.
__device__ __forceinline__ float tanh_of(float x) {
  const float u = x * x;
  const float num = __builtin_fmaf(__builtin_fmaf(u + 378.f, u, 17325.f), u, 135135.f);
  const float den = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(28.f, u, 3150.f), u, 62370.f), u, 135135.f);
  const float small = x * (num * __builtin_amdgcn_rcpf(den));
  const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2eF));
  const float large = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + e), 1.f);
  return fabsf(x) <= 2.f ? small : large;
}

template <bool F16, int DH>
__global__ __launch_bounds__(256, DH == 256 ? 2 : 3) void paged_weights_kernel(PagedWeightArgs a) {
  constexpr int CPR = DH / 8;
  constexpr int DSTEPS = DH / 16;
  constexpr int kQueryTile = DH == 256 ? 32 : 64;
  constexpr int CHUNKS = kQueryTile * CPR / 256;   // 16-byte chunks of a query tile per thread
  __shared__ __attribute__((aligned(16))) uint16_t s_q[2][kQueryTile * DH];
  __shared__ float s_lse[2][kQueryTile];
  __shared__ int s_token[2][kQueryTile];
  __shared__ int s_pos[kKeysPerWg];
  const ScoreArgs& sc = a.sc;
  const int b = blockIdx.z, g = blockIdx.y;
  int P, n;
  clamped_lengths(a.c, sc.prefix_len[b], sc.n_new[b], sc.max_prefix_len, sc.N, &P, &n);
  const int len = P + n;
  const int key0 = blockIdx.x * kKeysPerWg;
  if (key0 >= len || n == 0) {   // without new tokens the rows' weights only decay
    if (n == 0 && key0 < len) {
      const int key = key0 + threadIdx.x;
      if (threadIdx.x < kKeysPerWg && key < len) {
        const size_t at = static_cast<size_t>(b) * a.stride_b + static_cast<size_t>(g) * a.stride_h + key;
        a.out[at] = a.prior != nullptr ? a.decay * a.prior[at] : 0.f;
      }
    }
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int G = a.G;
  const bool positions = sc.window > 0 || sc.slopes != nullptr;

  // ---- this lane's key (every row past the end reads the last one; nobody sees it)
  const int kw0 = key0 + 32 * wave;
  uint4 ak[DSTEPS];
  {
    const int key = kw0 + l32 < len ? kw0 + l32 : len - 1;
    const uint32_t entry = page_entry(a.c, b, key);
    if (__ballot(entry >= a.c.num_pages) != 0ull && lane == 0) report(a.c, b, TALON_STATUS_BAD_PAGE);
    const uint16_t* kp = chunk_at(static_cast<const uint16_t*>(a.c.k), row_chunk(a.c, entry, key, g) + h);
#pragma unroll
    for (int ds = 0; ds < DSTEPS; ++ds) ak[ds] = *reinterpret_cast<const uint4*>(kp + 16 * ds);
  }
  if (positions && tid < kKeysPerWg) {
    const int key = key0 + tid;
    s_pos[tid] = key >= P && key < len ? P + offset_of(sc, b, key - P) : key;
  }

  // ---- the queries that may see a row of this workgroup: tokens [i_from, i_to)
  const int last_key = key0 + kKeysPerWg < len ? key0 + kKeysPerWg - 1 : len - 1;
  int i_from = sc.mask == nullptr && key0 > P ? key0 - P : 0;
  int i_to = n;
  if (sc.window > 0 && sc.offset == nullptr) {   // P + i - last_key < window
    const long long most = static_cast<long long>(last_key) - P + sc.window;
    i_to = most < i_to ? (most < 0 ? 0 : static_cast<int>(most)) : i_to;
  }
  const int r_end = i_to * G;
  const int rows = n * G;
  int r0 = i_from * G;
  float acc[16], sum[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = sum[r] = 0.f;

  const uint16_t* const qb = a.q.p + static_cast<int64_t>(b) * a.q.sb + static_cast<int64_t>(g) * G * a.q.sh;
  uint4 qv[CHUNKS];
  float lse_next = 0.f;
  int token_next = 0;
  auto load_queries = [&](int r) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int chunk = c * 256 + tid;
      int rho = r + chunk / CPR;
      rho = rho < rows ? rho : rows - 1;
      const int token = div_g(rho, a.inv_g);
      qv[c] = *reinterpret_cast<const uint4*>(qb + static_cast<int64_t>(token) * a.q.st + static_cast<int64_t>(rho - token * G) * a.q.sh + chunk % CPR * 8);
    }
    if (tid < kQueryTile) {
      const int rho = r + tid;
      token_next = -1;
      if (rho < r_end) {
        token_next = div_g(rho, a.inv_g);
        lse_next = a.lse[(static_cast<size_t>(b) * sc.N + token_next) * (a.Hkv * G) + g * G + rho - token_next * G];
      }
    }
  };
  auto store_queries = [&](int st) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int chunk = c * 256 + tid;
      const int row = chunk / CPR;
      const int swz = DH >= 128 ? (row & 15) : ((row >> 1) & 7);
      *reinterpret_cast<uint4*>(&s_q[st][row * DH + ((chunk % CPR) ^ swz) * 8]) = qv[c];
    }
    if (tid < kQueryTile) {
      s_lse[st][tid] = lse_next * kLog2eF;
      s_token[st][tid] = token_next;
    }
  };
  if (r0 < r_end) {
    load_queries(r0);
    store_queries(0);
  }
  __syncthreads();
  int folded = 0;
  for (int st = 0; r0 < r_end; r0 += kQueryTile, st ^= 1) {
    const bool more = r0 + kQueryTile < r_end;
    if (more) load_queries(r0 + kQueryTile);
#pragma unroll
    for (int qb_ = 0; qb_ < kQueryTile / 32; ++qb_) {
      floatx16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
      const int row = 32 * qb_ + l32;
      const int swz = DH >= 128 ? (row & 15) : ((row >> 1) & 7);
#pragma unroll
      for (int ds = 0; ds < DSTEPS; ++ds) {
        const uint4 q = *reinterpret_cast<const uint4*>(&s_q[st][row * DH + ((2 * ds + h) ^ swz) * 8]);
        s = product<F16>(ak[ds], q, s);
      }
      const float lse2 = s_lse[st][row];
      const int token = s_token[st][row];
      if (sc.cap_log2e > 0.f) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = sc.cap_log2e * tanh_of(s[r] * sc.cap_in);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= sc.scale_log2e;
      }
      const unsigned long long bits = token < 0 ? 0ull : seen_rows(sc, b, token, P, kw0, len);
      const uint32_t w = static_cast<uint32_t>(bits) >> (4 * h);
      if (positions) {
        const int p_i = token < 0 ? 0 : P + offset_of(sc, b, token);
        const float slope2 = sc.slopes != nullptr && token >= 0 ? sc.slopes[g * G + (r0 + row - token * G)] * kLog2eF : 0.f;
        const int window = sc.window > 0 ? sc.window : 0x7FFFFFFF;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = 8 * (r / 4) + r % 4;
          const int apart = p_i - s_pos[32 * wave + k + 4 * h];
          const float x = __builtin_fmaf(-slope2, fabsf(static_cast<float>(apart)), s[r]) - lse2;
          acc[r] += ((w >> k) & 1u) && apart < window ? __builtin_amdgcn_exp2f(x) : 0.f;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = 8 * (r / 4) + r % 4;
          acc[r] += ((w >> k) & 1u) ? __builtin_amdgcn_exp2f(s[r] - lse2) : 0.f;
        }
      }
    }
    if (++folded == 8) {   // sums of sixteen, then the sums of those: what rounding adds up to stays small over thousands of queries
      folded = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) { sum[r] += acc[r]; acc[r] = 0.f; }
    }
    if (more) store_queries(st ^ 1);
    __syncthreads();
  }
  // ---- over the 32 queries of a half
  float mine = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float v = sum[r] + acc[r];
    v += __int_as_float(dpp_i32<kDppXor1>(__float_as_int(v)));
    v += __int_as_float(dpp_i32<kDppXor2>(__float_as_int(v)));
    v += __int_as_float(dpp_i32<kDppHalfMirror>(__float_as_int(v)));
    v += __int_as_float(dpp_i32<kDppMirror>(__float_as_int(v)));
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    v = __int_as_float(static_cast<int>(p[0])) + __int_as_float(static_cast<int>(p[1]));
    mine = l32 == r ? v : mine;
  }
  const int key = kw0 + 8 * (l32 / 4) + l32 % 4 + 4 * h;
  if (l32 < 16 && key < len) {
    const size_t at = static_cast<size_t>(b) * a.stride_b + static_cast<size_t>(g) * a.stride_h + key;
    a.out[at] = mine + (a.prior != nullptr && key < P ? a.decay * a.prior[at] : 0.f);
  }
}

template <bool F16>
hipError_t launch_weights(const PagedWeightArgs& a, int Dh, hipStream_t s) {
  const int most = a.sc.max_prefix_len + a.sc.N < a.c.capacity ? a.sc.max_prefix_len + a.sc.N : a.c.capacity;
  const dim3 grid((most + kKeysPerWg - 1) / kKeysPerWg, a.Hkv, a.B);
  switch (Dh) {
    case 64: hipLaunchKernelGGL((paged_weights_kernel<F16, 64>), grid, dim3(256), 0, s, a); break;
    case 128: hipLaunchKernelGGL((paged_weights_kernel<F16, 128>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((paged_weights_kernel<F16, 256>), grid, dim3(256), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_weights(const PagedWeightArgs& a, int Dh, int dtype, hipStream_t s) {
  return dtype == TALON_DTYPE_F16 ? launch_weights<true>(a, Dh, s) : launch_weights<false>(a, Dh, s);
}

}  // namespace talon
