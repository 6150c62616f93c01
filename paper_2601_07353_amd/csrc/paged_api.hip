// C ABI of the calls on a paged cache: argument validation and launches.  Everything that can be checked on the host is
// checked before the first launch, so a failed call enqueues nothing.
#include <math.h>

#include "paged_internal.h"
#include "paged_plan.h"
#include "talon_internal.h"

namespace talon {

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

constexpr int kMostRows = 1 << 30;        // of a sequence: positions are 32-bit numbers
constexpr int kMostHeads = 128;

int invalid(const char* fmt, const char* what) { set_error(fmt, what); return TALON_ERR_INVALID_ARG; }

int check_cache(const talon_paged_cache* c, const char* name, PagedRows* out) {
  if (!c) return invalid("%s is NULL", name);
  if (c->B < 1 || c->B > TALON_B_MAX) { set_error("%s: B=%d outside [1, %d]", name, c->B, TALON_B_MAX); return TALON_ERR_INVALID_ARG; }
  if (c->dtype != TALON_DTYPE_BF16 && c->dtype != TALON_DTYPE_F16) { set_error("%s: dtype %d not supported (bf16 or f16)", name, c->dtype); return TALON_ERR_UNSUPPORTED; }
  if (c->Hkv < 1) { set_error("%s: Hkv=%d must be >= 1", name, c->Hkv); return TALON_ERR_INVALID_ARG; }
  if (c->Hkv > kMostHeads) { set_error("%s: Hkv=%d above %d is not supported", name, c->Hkv, kMostHeads); return TALON_ERR_UNSUPPORTED; }
  if (c->Dh < 8 || c->Dh % 8) { set_error("%s: Dh=%d must be a positive multiple of 8", name, c->Dh); return TALON_ERR_INVALID_ARG; }
  if (c->Dh > 1024) { set_error("%s: Dh=%d above 1024 is not supported", name, c->Dh); return TALON_ERR_UNSUPPORTED; }
  if (c->page_size < 1 || (c->page_size & (c->page_size - 1))) { set_error("%s: page_size=%d must be a power of two", name, c->page_size); return TALON_ERR_INVALID_ARG; }
  if (c->num_pages < 1 || c->max_pages < 1) { set_error("%s: num_pages=%d and max_pages=%d must be >= 1", name, c->num_pages, c->max_pages); return TALON_ERR_INVALID_ARG; }
  const long long capacity = static_cast<long long>(c->max_pages) * c->page_size;
  if (capacity > kMostRows) { set_error("%s: %lld rows per sequence, at most %d are supported", name, capacity, kMostRows); return TALON_ERR_UNSUPPORTED; }
  if (!c->k || !c->v || !c->page_table || !c->status) return invalid("%s holds a NULL pointer", name);
  if (!aligned16(c->k) || !aligned16(c->v)) return invalid("%s: K/V pools must be 16-byte aligned", name);
  if (!aligned4(c->page_table) || !aligned4(c->status)) return invalid("%s: page_table or status is misaligned", name);
  const int64_t strides[3] = {c->stride_page, c->stride_token, c->stride_head};
  const int sizes[3] = {c->num_pages, c->page_size, c->Hkv};
  int64_t chunks[3];
  long double last = 0.0L;
  for (int i = 0; i < 3; ++i) {
    const int64_t st = sizes[i] > 1 ? strides[i] : 0;
    if (sizes[i] > 1 && (st < c->Dh || st % 8)) return invalid("%s: strides must be >= Dh and multiples of 8 elements", name);
    chunks[i] = st / 8;
    last += static_cast<long double>(chunks[i]) * (sizes[i] - 1);
  }
  if (last + c->Dh / 8 > 4294967295.0L) { set_error("%s: a pool of more than 64 GiB per tensor is not supported", name); return TALON_ERR_UNSUPPORTED; }
  if (out) {
    out->k = c->k; out->v = c->v; out->table = c->page_table; out->status = c->status;
    out->max_pages = c->max_pages; out->num_pages = static_cast<uint32_t>(c->num_pages);
    out->page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
    out->capacity = static_cast<int>(capacity);
    out->page_chunks = static_cast<uint32_t>(chunks[0]); out->token_chunks = static_cast<uint32_t>(chunks[1]); out->head_chunks = static_cast<uint32_t>(chunks[2]);
  }
  return TALON_OK;
}

int check_view(const talon_view* v, const char* name, int B, int N, int H, int Dh, bool written, RowsView* out) {
  if (!v || !v->data) return invalid("%s is NULL", name);
  if (!aligned16(v->data)) return invalid("%s is not 16-byte aligned", name);
  const int64_t strides[3] = {v->stride_b, v->stride_t, v->stride_h};
  const int sizes[3] = {B, N, H};
  for (int i = 0; i < 3; ++i) {
    if (sizes[i] == 1) continue;
    if (strides[i] % 8 || strides[i] < (written ? Dh : 0)) return invalid(written ? "%s: strides must be >= Dh and multiples of 8 elements"
                                                                                   : "%s: strides must be >= 0 and multiples of 8 elements", name);
  }
  out->p = static_cast<uint16_t*>(v->data);
  out->sb = B == 1 ? 0 : v->stride_b; out->st = N == 1 ? 0 : v->stride_t; out->sh = H == 1 ? 0 : v->stride_h;
  return TALON_OK;
}

int check_new(int N, const int32_t* n_new, const int32_t* prefix_len) {
  if (N < 1 || N > 65536) { set_error("N=%d outside [1, 65536]", N); return TALON_ERR_INVALID_ARG; }
  if (!n_new || !prefix_len) { set_error("n_new / prefix_len is NULL"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(n_new) || !aligned4(prefix_len)) { set_error("n_new / prefix_len is misaligned"); return TALON_ERR_INVALID_ARG; }
  return TALON_OK;
}

int check_heads(int N, int Hq, int Hkv, int Dh) {
  if (Hq < 1) { set_error("Hq=%d must be >= 1", Hq); return TALON_ERR_INVALID_ARG; }
  if (Dh != 64 && Dh != 128 && Dh != 256) { set_error("Dh=%d not supported (64, 128 or 256)", Dh); return TALON_ERR_UNSUPPORTED; }
  if (Hq % Hkv) { set_error("Hq=%d is not a multiple of Hkv=%d", Hq, Hkv); return TALON_ERR_UNSUPPORTED; }
  if (Hq / Hkv > 128) { set_error("Hq/Hkv=%d above 128 is not supported", Hq / Hkv); return TALON_ERR_UNSUPPORTED; }
  if (static_cast<long long>(N) * (Hq / Hkv) >= 1 << 24) { set_error("N=%d tokens of %d heads per KV head are not supported", N, Hq / Hkv); return TALON_ERR_UNSUPPORTED; }
  return TALON_OK;
}

int check_scores(const talon_scores* s, int N, int Dh, int max_prefix_len, const int32_t* n_new, const int32_t* prefix_len, bool weights, ScoreArgs* out) {
  static const talon_scores plain = {nullptr, nullptr, nullptr, 0.f, 0.f, 0};
  if (!s) s = &plain;
  if (max_prefix_len < 0 || max_prefix_len > kMostRows) { set_error("max_prefix_len=%d outside [0, %d]", max_prefix_len, kMostRows); return TALON_ERR_INVALID_ARG; }
  if (reinterpret_cast<uintptr_t>(s->mask) & 7u) { set_error("mask is misaligned"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(s->offset) || !aligned4(s->slopes)) { set_error("offset / slopes is misaligned"); return TALON_ERR_INVALID_ARG; }
  if (!(s->scale >= 0.f) || isinf(s->scale)) { set_error("scale=%g must be finite and >= 0 (0 selects 1/sqrt(Dh))", static_cast<double>(s->scale)); return TALON_ERR_INVALID_ARG; }
  if (!(s->softcap >= 0.f) || isinf(s->softcap)) { set_error("softcap=%g must be finite and >= 0 (0: none)", static_cast<double>(s->softcap)); return TALON_ERR_INVALID_ARG; }
  if (s->window < 0) { set_error("window=%d must be >= 0 (0: none)", s->window); return TALON_ERR_INVALID_ARG; }
  const double scale = s->scale == 0.f ? 1.0 / sqrt(static_cast<double>(Dh)) : static_cast<double>(s->scale);
  const double log2e = 1.4426950408889634;
  // What the kernels multiply by has to be a number in 32 bits: a score of 0 times infinity is none, and a quotient below the least normal
  // number has lost its digits.
  auto held = [](double x) { return fabs(x) <= 3.4028234e38; };
  if (!held(scale * log2e) || !held(s->softcap * log2e) ||
      (s->softcap > 0.f && (!held(2.0 * scale * log2e / s->softcap) || scale / s->softcap < 1.1754944e-38))) {
    set_error("scale=%g with softcap=%g: the products with log2(e) and the quotient must be normal 32-bit numbers", scale, static_cast<double>(s->softcap));
    return TALON_ERR_INVALID_ARG;
  }
  out->n_new = n_new; out->prefix_len = prefix_len; out->mask = s->mask; out->offset = s->offset; out->slopes = s->slopes;
  out->N = N; out->words = (N + 63) / 64; out->max_prefix_len = max_prefix_len; out->window = s->window;
  out->scale_log2e = static_cast<float>(scale * log2e);
  out->cap_log2e = static_cast<float>(s->softcap * log2e);
  out->cap_in = s->softcap > 0.f ? static_cast<float>(weights || s->softcap > kNearCap ? scale / s->softcap : 2.0 * scale * log2e / s->softcap) : 0.f;
  return TALON_OK;
}

uint32_t inverse_of(int G) { return G == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + G - 1) / G); }

}  // namespace

}  // namespace talon

using namespace talon;

extern "C" {

int talon_rotary_store(const talon_paged_cache* cache, const talon_view* q, const talon_view* k, const talon_view* v,
                       const talon_view* q_out, int32_t N, int32_t Hq, const int32_t* n_new, const int32_t* prefix_len,
                       const int32_t* pos, int32_t axes, const int32_t* pos_base, const float* inv_freq, int32_t pairs,
                       const int32_t* pair_axis, int32_t interleaved, void* stream) {
  RotaryArgs a = {};
  int rc = check_cache(cache, "cache", &a.c);
  if (rc) return rc;
  if ((rc = check_new(N, n_new, prefix_len))) return rc;
  if (Hq < 1 || Hq > 65536) { set_error("Hq=%d outside [1, 65536]", Hq); return TALON_ERR_INVALID_ARG; }
  const int B = cache->B, Hkv = cache->Hkv, Dh = cache->Dh;
  if ((rc = check_view(q, "q", B, N, Hq, Dh, false, &a.q))) return rc;
  if ((rc = check_view(k, "k", B, N, Hkv, Dh, false, &a.k))) return rc;
  if ((rc = check_view(v, "v", B, N, Hkv, Dh, false, &a.v))) return rc;
  if ((rc = check_view(q_out, "q_out", B, N, Hq, Dh, true, &a.q_out))) return rc;
  if (a.q.p == a.q_out.p && (a.q.sb != a.q_out.sb || a.q.st != a.q_out.st || a.q.sh != a.q_out.sh)) { set_error("q in place needs q's strides"); return TALON_ERR_INVALID_ARG; }
  if (pairs < 0 || pairs > Dh / 2) { set_error("pairs=%d outside [0, Dh/2=%d]", pairs, Dh / 2); return TALON_ERR_INVALID_ARG; }
  if (axes < 1 || axes > 8) { set_error("axes=%d outside [1, 8]", axes); return TALON_ERR_INVALID_ARG; }
  if (pairs > 0 && (!pos || !inv_freq)) { set_error("pos / inv_freq is NULL"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(pos) || !aligned4(inv_freq) || !aligned4(pos_base) || !aligned4(pair_axis)) { set_error("pos, pos_base, inv_freq or pair_axis is misaligned"); return TALON_ERR_INVALID_ARG; }
  a.n_new = n_new; a.prefix_len = prefix_len; a.pos = pos; a.base = pos_base; a.axis = pair_axis; a.inv_freq = inv_freq;
  a.B = B; a.N = N; a.Hq = Hq; a.Hkv = Hkv; a.Dh = Dh; a.pairs = pairs; a.axes = axes; a.interleaved = interleaved != 0;
  return check_hip(launch_rotary_store(a, cache->dtype, static_cast<hipStream_t>(stream)), "rotary store launch");
}

size_t talon_paged_attention_workspace_bytes(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t max_prefix_len) {
  if (B < 1 || B > TALON_B_MAX) { set_error("B=%d outside [1, %d]", B, TALON_B_MAX); return 0; }
  if (N < 1 || N > 65536) { set_error("N=%d outside [1, 65536]", N); return 0; }
  if (Hkv < 1 || Hkv > kMostHeads) { set_error("Hkv=%d outside [1, %d]", Hkv, kMostHeads); return 0; }
  if (check_heads(N, Hq, Hkv, Dh)) return 0;
  if (max_prefix_len < 0 || max_prefix_len > kMostRows) { set_error("max_prefix_len=%d outside [0, %d]", max_prefix_len, kMostRows); return 0; }
  const PagedPlan p = paged_plan(B, N, Hq, Hkv, Dh, max_prefix_len);
  if (p.tiles >= 1ll << 30) { set_error("%lld key tiles are more than one call takes", p.tiles); return 0; }
  return p.room;
}

int talon_paged_attention(const talon_paged_cache* cache, const talon_view* q, int32_t N, int32_t Hq, const int32_t* n_new,
                          const int32_t* prefix_len, int32_t max_prefix_len, const talon_scores* scores, const talon_view* out,
                          float* out_lse, void* workspace, size_t workspace_bytes, void* stream) {
  PagedAttnArgs a = {};
  int rc = check_cache(cache, "cache", &a.c);
  if (rc) return rc;
  const int B = cache->B, Hkv = cache->Hkv, Dh = cache->Dh;
  if ((rc = check_new(N, n_new, prefix_len))) return rc;
  if ((rc = check_heads(N, Hq, Hkv, Dh))) return rc;
  if ((rc = check_scores(scores, N, Dh, max_prefix_len, n_new, prefix_len, false, &a.sc))) return rc;
  if ((rc = check_view(q, "q", B, N, Hq, Dh, false, &a.q))) return rc;
  if ((rc = check_view(out, "out", B, N, Hq, Dh, true, &a.out))) return rc;
  if (!aligned4(out_lse)) { set_error("out_lse is misaligned"); return TALON_ERR_INVALID_ARG; }
  const int prefix = max_prefix_len < a.c.capacity ? max_prefix_len : a.c.capacity;
  const PagedPlan p = paged_plan(B, N, Hq, Hkv, Dh, prefix);
  if (p.tiles >= 1ll << 30) { set_error("%lld key tiles are more than one call takes", p.tiles); return TALON_ERR_UNSUPPORTED; }
  a.lse = out_lse;
  a.B = B; a.Hkv = Hkv; a.G = Hq / Hkv; a.inv_g = inverse_of(a.G);
  a.slots = p.slots; a.least = p.least; a.extra = p.extra; a.rows_slot = p.rows_slot;
  a.split = p.split;
  if (p.split) {
    if (!workspace || !aligned16(workspace)) { set_error("workspace is NULL or not 16-byte aligned"); return TALON_ERR_INVALID_ARG; }
    if (workspace_bytes < p.bytes) { set_error("workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, p.bytes); return TALON_ERR_WORKSPACE; }
    char* w = static_cast<char*>(workspace);
    a.part_o = reinterpret_cast<float*>(w);
    a.part_m = reinterpret_cast<float*>(w + p.off_m);
    a.part_l = reinterpret_cast<float*>(w + p.off_l);
    a.cut = reinterpret_cast<int4*>(w + p.off_cut);
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f16 = cache->dtype == TALON_DTYPE_F16;
  hipError_t e;
  if (scores && scores->softcap > kNearCap) e = f16 ? launch_paged_attention_f16_far(a, Dh, p.waves, s) : launch_paged_attention_bf16_far(a, Dh, p.waves, s);
  else if (Dh == 64) e = f16 ? launch_paged_attention_f16_64(a, p.waves, s) : launch_paged_attention_bf16_64(a, p.waves, s);
  else if (Dh == 128) e = f16 ? launch_paged_attention_f16_128(a, p.waves, s) : launch_paged_attention_bf16_128(a, p.waves, s);
  else e = f16 ? launch_paged_attention_f16_256(a, p.waves, s) : launch_paged_attention_bf16_256(a, p.waves, s);
  return check_hip(e, "paged attention launch");
}

int talon_paged_weights(const talon_paged_cache* cache, const talon_view* q, int32_t N, int32_t Hq, const int32_t* n_new,
                        const int32_t* prefix_len, int32_t max_prefix_len, const talon_scores* scores, const float* lse,
                        float decay, const float* prior, float* weights, int64_t stride_b, int64_t stride_h, void* stream) {
  PagedWeightArgs wa = {};
  PagedAttnArgs& a = wa.a;
  int rc = check_cache(cache, "cache", &a.c);
  if (rc) return rc;
  const int B = cache->B, Hkv = cache->Hkv, Dh = cache->Dh;
  if ((rc = check_new(N, n_new, prefix_len))) return rc;
  if ((rc = check_heads(N, Hq, Hkv, Dh))) return rc;
  if ((rc = check_scores(scores, N, Dh, max_prefix_len, n_new, prefix_len, true, &a.sc))) return rc;
  if ((rc = check_view(q, "q", B, N, Hq, Dh, false, &a.q))) return rc;
  if (!lse || !weights) { set_error("lse / weights is NULL"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(lse) || !aligned4(weights) || !aligned4(prior)) { set_error("lse, weights or prior is misaligned"); return TALON_ERR_INVALID_ARG; }
  if (!(fabsf(decay) <= 1.f)) { set_error("decay=%g outside [-1, 1]", static_cast<double>(decay)); return TALON_ERR_INVALID_ARG; }
  const long long most = static_cast<long long>(max_prefix_len) + N < a.c.capacity ? static_cast<long long>(max_prefix_len) + N : a.c.capacity;
  if ((Hkv > 1 && stride_h < most) || (B > 1 && stride_b < most) || stride_h < 0 || stride_b < 0) {
    set_error("weights: strides %lld, %lld do not hold %lld rows", (long long)stride_b, (long long)stride_h, most);
    return TALON_ERR_INVALID_ARG;
  }
  const long long far = (N > 1 ? a.q.st / 8 * (N - 1) : 0) + a.q.sh / 8 * (Hq / Hkv - 1);
  if (far >= 1ll << 32) { set_error("q: a sequence's tokens lie more than 64 GiB apart"); return TALON_ERR_UNSUPPORTED; }
  a.lse = const_cast<float*>(lse);
  a.B = B; a.Hkv = Hkv; a.G = Hq / Hkv; a.inv_g = inverse_of(a.G);
  wa.prior = prior; wa.out = weights; wa.stride_b = stride_b; wa.stride_h = stride_h; wa.decay = decay;
  const bool few = static_cast<long long>(N) * a.G <= 32;
  if (!few && (most + kWeighRows - 1) / kWeighRows * kWeighThreads >= 1ll << 32) {   // (the threads of a grid's dimension)
    set_error("%lld rows for more than 32 queries of a KV head are not supported", most);
    return TALON_ERR_UNSUPPORTED;
  }
  const WeighPlan p = weigh_plan(B, Hkv, Dh, static_cast<int>(most));
  if (p.tiles >= 1ll << 30) { set_error("%lld key tiles are more than one call takes", p.tiles); return TALON_ERR_UNSUPPORTED; }
  a.split = 1; a.slots = p.slots; a.least = p.least; a.extra = p.extra;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return check_hip(cache->dtype == TALON_DTYPE_F16 ? launch_paged_weights_f16(wa, Dh, few, s) : launch_paged_weights_bf16(wa, Dh, few, s),
                   "paged weights launch");
}

int talon_paged_evict(const talon_paged_cache* cache, const talon_paged_cache* dst, const int32_t* len, int32_t max_len,
                      const float* weights, int64_t stride_b, int64_t stride_h, int32_t budget, int32_t n_sink,
                      int32_t n_recent, int32_t* kept, int32_t* new_len, float* new_weights, int64_t new_stride_b,
                      int64_t new_stride_h, void* stream) {
  EvictArgs a = {};
  int rc = check_cache(cache, "cache", &a.src);
  if (rc) return rc;
  if (!dst) dst = cache;
  if ((rc = check_cache(dst, "dst", &a.dst))) return rc;
  if (dst->B != cache->B || dst->Hkv != cache->Hkv || dst->Dh != cache->Dh || dst->dtype != cache->dtype) {
    set_error("dst must have the cache's B, Hkv, Dh and dtype");
    return TALON_ERR_INVALID_ARG;
  }
  if (!len || !weights || !kept || !new_len) { set_error("talon_paged_evict: NULL pointer argument"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(len) || !aligned4(weights) || !aligned4(kept) || !aligned4(new_len) || !aligned4(new_weights)) { set_error("talon_paged_evict: misaligned pointer"); return TALON_ERR_INVALID_ARG; }
  if (new_len == len) { set_error("new_len must not be len"); return TALON_ERR_INVALID_ARG; }
  if (max_len < 0 || max_len > kMostRows) { set_error("max_len=%d outside [0, %d]", max_len, kMostRows); return TALON_ERR_INVALID_ARG; }
  if (budget < 1 || budget > kMostRows) { set_error("budget=%d outside [1, %d]", budget, kMostRows); return TALON_ERR_INVALID_ARG; }
  if (n_sink < 0 || n_recent < 0 || static_cast<long long>(n_sink) + n_recent > budget) {
    set_error("n_sink=%d and n_recent=%d must be >= 0 and fit the budget of %d", n_sink, n_recent, budget);
    return TALON_ERR_INVALID_ARG;
  }
  const int most = max_len < a.src.capacity ? max_len : a.src.capacity;
  const int stays = budget < most ? budget : most;
  if (stays > a.dst.capacity) { set_error("dst holds %d rows per sequence, %d may stay", a.dst.capacity, stays); return TALON_ERR_INVALID_ARG; }
  const int B = cache->B, Hkv = cache->Hkv;
  if ((Hkv > 1 && stride_h < most) || (B > 1 && stride_b < most) || stride_h < 0 || stride_b < 0 ||
      (new_weights && ((Hkv > 1 && new_stride_h < stays) || (B > 1 && new_stride_b < stays) || new_stride_h < 0 || new_stride_b < 0))) {
    set_error("weights: a stride does not hold the rows");
    return TALON_ERR_INVALID_ARG;
  }
  if (new_weights == weights && ((B > 1 && new_stride_b != stride_b) || (Hkv > 1 && new_stride_h != stride_h))) { set_error("weights in place need one set of strides"); return TALON_ERR_INVALID_ARG; }
  a.len = len; a.new_len = new_len; a.weights = weights; a.new_weights = new_weights;
  a.stride_b = stride_b; a.stride_h = stride_h; a.new_stride_b = new_stride_b; a.new_stride_h = new_stride_h;
  a.kept = kept; a.B = B; a.Hkv = Hkv; a.Dh = cache->Dh; a.budget = budget; a.n_sink = n_sink; a.n_recent = n_recent; a.max_len = max_len;
  a.in_place = dst->page_table == cache->page_table && dst->k == cache->k && dst->v == cache->v;
  if (a.in_place && (dst->page_size != cache->page_size || dst->max_pages != cache->max_pages || dst->num_pages != cache->num_pages ||
                     a.dst.page_chunks != a.src.page_chunks || a.dst.token_chunks != a.src.token_chunks || a.dst.head_chunks != a.src.head_chunks)) {
    set_error("dst in place must be the same cache");
    return TALON_ERR_INVALID_ARG;
  }
  return check_hip(launch_paged_evict(a, static_cast<hipStream_t>(stream)), "paged evict launch");
}

int talon_paged_compact(const talon_paged_cache* cache, int32_t N, const int32_t* path, const int32_t* accept_len,
                        const int32_t* prefix_len, int32_t* new_prefix_len, float* weights, int32_t weight_rows,
                        int64_t stride_b, int64_t stride_h, void* stream) {
  CompactArgs a = {};
  int rc = check_cache(cache, "cache", &a.c);
  if (rc) return rc;
  if (N < 1 || N > TALON_N_MAX) { set_error("N=%d outside [1, %d]", N, TALON_N_MAX); return TALON_ERR_INVALID_ARG; }
  if (!path || !accept_len || !prefix_len || !new_prefix_len) { set_error("talon_paged_compact: NULL pointer argument"); return TALON_ERR_INVALID_ARG; }
  if (!aligned4(path) || !aligned4(accept_len) || !aligned4(prefix_len) || !aligned4(new_prefix_len) || !aligned4(weights)) { set_error("talon_paged_compact: misaligned pointer"); return TALON_ERR_INVALID_ARG; }
  if (new_prefix_len == prefix_len) { set_error("new_prefix_len must not be prefix_len"); return TALON_ERR_INVALID_ARG; }
  if (weights && (weight_rows < 0 || (cache->Hkv > 1 && stride_h < weight_rows) || (cache->B > 1 && stride_b < weight_rows) || stride_h < 0 || stride_b < 0)) {
    set_error("weights: strides %lld, %lld do not hold %d rows", (long long)stride_b, (long long)stride_h, weight_rows);
    return TALON_ERR_INVALID_ARG;
  }
  a.path = path; a.accept_len = accept_len; a.prefix_len = prefix_len; a.new_prefix_len = new_prefix_len;
  a.weights = weights; a.weight_rows = weight_rows; a.stride_b = stride_b; a.stride_h = stride_h;
  a.B = cache->B; a.N = N; a.Hkv = cache->Hkv; a.Dh = cache->Dh;
  return check_hip(launch_paged_compact(a, static_cast<hipStream_t>(stream)), "paged compact launch");
}

}  // extern "C"
