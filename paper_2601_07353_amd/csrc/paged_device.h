// Device helpers of the calls on a paged cache.
#pragma once

#include "device_utils.h"
#include "paged_internal.h"

namespace talon {

constexpr float kNoScore = -__builtin_huge_valf();
constexpr float kLog2eF = 1.4426950408889634f;
constexpr float kLn2F = 0.6931471805599453f;

// tanh(x) to a few units in the last place, also near 0, where 1 - 2 / (1 + e^(2x)) keeps no more than its absolute accuracy
// (scores of large caps, and the weights, whose sums stay in fp32, need better): the continued fraction x / (1 + x^2 / (3 + x^2 / (5 + ...)))
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

// x / G for 0 <= x < 2^24, G <= 128: exact, since x * (inv_g * G - 2^32) < 2^32.
// (inv_g is 0 for G = 1; without a branch, which would end a block.)
__device__ __forceinline__ int div_g(int x, uint32_t inv_g) {
  return static_cast<int>(__umulhi(static_cast<uint32_t>(x), inv_g)) + (x & -static_cast<int>(inv_g == 0u));
}

// Rows that a sequence has in the cache and rows that are new, whatever the device's numbers say: neither
// points beyond what the call or the page table allows for.
__device__ __forceinline__ void clamped_lengths(const PagedRows& c, int prefix, int fresh, int max_prefix, int N, int* P, int* n) {
  int p = prefix < 0 ? 0 : (prefix > max_prefix ? max_prefix : prefix);
  p = p < c.capacity ? p : c.capacity;
  int m = fresh < 0 ? 0 : (fresh > N ? N : fresh);
  *P = p;
  *n = m < c.capacity - p ? m : c.capacity - p;
}

__device__ __forceinline__ void report(const PagedRows& c, int b, uint32_t bit) { atomicOr(&c.status[b], bit); }

// Rows that lie beyond the page table, which clamped_lengths leaves out: reported by one thread of a call.
__device__ __forceinline__ void report_table_end(const PagedRows& c, int b, int prefix, int fresh, int max_prefix, int N) {
  const int p = prefix < 0 ? 0 : (prefix > max_prefix ? max_prefix : prefix);
  const int m = fresh < 0 ? 0 : (fresh > N ? N : fresh);
  if (p + m > c.capacity) report(c, b, TALON_STATUS_BAD_PAGE);
}

// First chunk of (row's page entry, row, KV head); an entry that names no page of the pool is page 0 (the caller reports it).
__device__ __forceinline__ uint32_t row_chunk(const PagedRows& c, uint32_t entry, int row, int g) {
  const uint32_t page = entry < c.num_pages ? entry : 0u;
  const uint32_t slot = static_cast<uint32_t>(row) & ((1u << c.page_shift) - 1u);
  return page * c.page_chunks + slot * c.token_chunks + static_cast<uint32_t>(g) * c.head_chunks;
}

__device__ __forceinline__ uint32_t page_entry(const PagedRows& c, int b, int row) {
  return static_cast<uint32_t>(c.table[static_cast<size_t>(b) * c.max_pages + (row >> c.page_shift)]);
}

template <class T>
__device__ __forceinline__ T* chunk_at(T* base, uint32_t chunk) { return base + static_cast<size_t>(chunk) * 8; }

// Which of the 64 rows from `row0` on the new token `i` of a sequence may see, by its mask words or causally (not yet by a
// window), as bits; rows from `end` on are never seen.
// `w`: the token's mask words.
template <class W>
__device__ __forceinline__ unsigned long long seen_rows(const ScoreArgs& s, int i, int P, int row0, int end, const W* w) {
  unsigned long long bits;
  const int d = row0 - P;   // new token that row0 is
  if (s.mask == nullptr) {
    const int count = P + i + 1 - row0;
    bits = count >= 64 ? ~0ull : (count <= 0 ? 0ull : (1ull << count) - 1ull);
  } else {
    if (d >= 0) {
      const int at = d >> 6, shift = d & 63;
      bits = at < s.words ? w[at] >> shift : 0ull;
      if (shift != 0 && at + 1 < s.words) bits |= w[at + 1] << (64 - shift);
    } else if (d > -64) {
      bits = (w[0] << -d) | ((1ull << -d) - 1ull);
    } else {
      bits = ~0ull;
    }
  }
  const int left = end - row0;
  if (left < 64) bits &= left <= 0 ? 0ull : (1ull << left) - 1ull;
  return bits;
}

__device__ __forceinline__ unsigned long long seen_rows(const ScoreArgs& s, int b, int i, int P, int row0, int end) {
  return seen_rows(s, i, P, row0, end, s.mask != nullptr ? s.mask + (static_cast<size_t>(b) * s.N + i) * s.words : nullptr);
}

// Position of new token i relative to the prefix.  (Bounded, so that positions stay 32-bit numbers.)
constexpr int kMostOffset = (1 << 30) - 1;
__device__ __forceinline__ int offset_of(const ScoreArgs& s, int b, int i) {
  if (s.offset == nullptr) return i;
  const int o = s.offset[static_cast<size_t>(b) * s.N + i];
  return o < 0 ? 0 : (o < kMostOffset ? o : kMostOffset);
}

}  // namespace talon
