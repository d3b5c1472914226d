// extern "C" entry points of the last part of include/qblora.h (rotary positions, paged cache plan, attention): host-side
// argument checks and dispatch.  No device memory is allocated here.
#include <cmath>

#include "serving.cuh"

namespace qb {
namespace {

bool heads_ok(const qblora_heads* h, HeadsView* v) {
  if (!h || !h->data || h->heads < 1 || h->token_stride < 0 || h->head_stride < 0) return false;
  if (h->dtype != QBLORA_F32 && h->dtype != QBLORA_BF16) return false;
  if (reinterpret_cast<uintptr_t>(h->data) % (h->dtype == QBLORA_F32 ? 4 : 2)) return false;
  *v = {h->data, h->token_stride, h->head_stride, h->heads, h->dtype};
  return true;
}

// y may be x itself, not x's memory in another type or order: elements are written while others of x are still to be read
bool in_place_ok(const HeadsView& x, const HeadsView& y, int64_t tokens) {
  return x.data != y.data || (x.dtype == y.dtype && (x.ts == y.ts || tokens == 1) && (x.hs == y.hs || x.heads == 1));
}

bool cache_ok(const qblora_kv_cache* c, CacheView* v) {
  if (!c || !c->k || !c->v) return false;
  if (reinterpret_cast<uintptr_t>(c->k) % 2 || reinterpret_cast<uintptr_t>(c->v) % 2) return false;
  if (c->n_pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return false;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return false;
  if ((int64_t)c->n_pages * c->page_size >= (int64_t)1 << 31) return false;
  *v = {static_cast<__nv_bfloat16*>(c->k), static_cast<__nv_bfloat16*>(c->v), c->page_stride, c->token_stride,
        c->head_stride, c->n_pages, c->page_size, c->kv_heads};
  return true;
}

bool rope_ok(const qblora_rope_cfg* c, int inverse, RopeView* v) {
  if (!c || !c->turns || reinterpret_cast<uintptr_t>(c->turns) % 8) return false;
  if (c->head_dim < 2 || c->rotary_dim < 2 || c->rotary_dim % 2 || c->rotary_dim > c->head_dim) return false;
  if (c->layout != QBLORA_ROPE_HALF && c->layout != QBLORA_ROPE_PAIRS) return false;
  if (!std::isfinite(c->amplitude)) return false;
  *v = {c->head_dim, c->rotary_dim, c->layout, c->amplitude, inverse ? -1.0f : 1.0f, c->turns};
  return true;
}

// Requests with more rows (new tokens x query heads per key head) than this go to the tcgen05 kernel.  A second row tile of
// paged_warp.cu reads the keys and values again, while 128 rows cost the tcgen05 kernel what 17 do; but its set-up is longer and
// the two kernels of a call whose requests straddle the border run one after the other.  Measured, 32 requests of 2000 to 4000 keys,
// 8 key heads: 12 rows 83 us there; 24 rows 131 us there, 102 here; 40 rows 104 here.  16 requests of 12 to 28 rows: 49 us
// with all of them there, 61 us with those above 16 rows here.  So a call whose requests all have 17 to 32 rows would be better off
// with a border of 16; the host, which does not know the lengths, cannot tell it from one that straddles the border.
constexpr int kNarrowRows = 32;

bool int_ptr_ok(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// An array of n int32 values of a call; p may be NULL.
struct IntSpan { const int32_t* p; int64_t n; };
bool overlap(const IntSpan& a, const IntSpan& b) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a0 < b0 + (uintptr_t)b.n * 4 && b0 < a0 + (uintptr_t)a.n * 4;
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" {

int qblora_rope_table(int32_t rotary_dim, double base, int32_t scale, double factor, int64_t trained_len, double slow,
                      double fast, uint64_t* turns) {
  if (!turns || rotary_dim < 2 || rotary_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return QBLORA_ERR_INVALID_ARG;
  if (scale < QBLORA_ROPE_SCALE_NONE || scale > QBLORA_ROPE_SCALE_BANDED) return QBLORA_ERR_INVALID_ARG;
  if (scale != QBLORA_ROPE_SCALE_NONE && !(factor > 0.0 && std::isfinite(factor))) return QBLORA_ERR_INVALID_ARG;
  if (scale == QBLORA_ROPE_SCALE_BANDED && !(trained_len > 0 && slow < fast)) return QBLORA_ERR_INVALID_ARG;
  if (scale == QBLORA_ROPE_SCALE_BASE) {
    if (rotary_dim == 2) return QBLORA_ERR_INVALID_ARG;   // the exponent d / (d - 2) has no value
    base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    if (!(base > 1.0)) return QBLORA_ERR_INVALID_ARG;
  }
  const double two_pi = 6.283185307179586476925;
  for (int j = 0; j < rotary_dim / 2; ++j) {
    double f = std::pow(base, -2.0 * j / rotary_dim) / two_pi;
    if (scale == QBLORA_ROPE_SCALE_LINEAR) f /= factor;
    if (scale == QBLORA_ROPE_SCALE_BANDED) {
      double w = ((double)trained_len * f - slow) / (fast - slow);
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      f = f * w + f / factor * (1.0 - w);
    }
    f -= std::floor(f);                                    // whole turns per position (factor < 1) change nothing
    turns[j] = static_cast<uint64_t>(std::ldexp(f, 64));   // f < 1: below 2^64
  }
  return QBLORA_OK;
}

int qblora_rope(const qblora_rope_cfg* cfg, int inverse, const int32_t* positions, int64_t tokens, const qblora_heads* x,
                const qblora_heads* y, const qblora_heads* x2, const qblora_heads* y2, void* stream) {
  RopeCall c{};
  if (!rope_ok(cfg, inverse, &c.cfg) || !int_ptr_ok(positions) || tokens < 1) return QBLORA_ERR_INVALID_ARG;
  if (!heads_ok(x, &c.q) || !heads_ok(y, &c.q_out) || x->heads != y->heads) return QBLORA_ERR_INVALID_ARG;
  if ((x2 == nullptr) != (y2 == nullptr)) return QBLORA_ERR_INVALID_ARG;
  if (x2) {
    if (!heads_ok(x2, &c.k) || !heads_ok(y2, &c.k_out) || x2->heads != y2->heads) return QBLORA_ERR_INVALID_ARG;
    if (x2->dtype != x->dtype || y2->dtype != y->dtype) return QBLORA_ERR_INVALID_ARG;
    if (!in_place_ok(c.k, c.k_out, tokens) || x2->data == y->data || x->data == y2->data || y->data == y2->data) return QBLORA_ERR_INVALID_ARG;
  }
  if (!in_place_ok(c.q, c.q_out, tokens)) return QBLORA_ERR_INVALID_ARG;
  c.positions = positions; c.T = tokens;
  return launch_rope(c, static_cast<cudaStream_t>(stream));
}

int qblora_rope_append(const qblora_rope_cfg* cfg, const int32_t* positions, const int32_t* slots, int64_t tokens,
                       const qblora_heads* q, const qblora_heads* k, const qblora_heads* v, const qblora_heads* q_out,
                       const qblora_kv_cache* cache, void* stream) {
  RopeCall c{};
  if (!rope_ok(cfg, 0, &c.cfg) || !int_ptr_ok(positions) || !int_ptr_ok(slots) || tokens < 1) return QBLORA_ERR_INVALID_ARG;
  if (!heads_ok(q, &c.q) || !heads_ok(k, &c.k) || !heads_ok(v, &c.v) || !heads_ok(q_out, &c.q_out)) return QBLORA_ERR_INVALID_ARG;
  if (!cache_ok(cache, &c.cache)) return QBLORA_ERR_INVALID_ARG;
  if (q->heads != q_out->heads || q_out->dtype != QBLORA_BF16 || k->dtype != q->dtype || v->dtype != q->dtype) return QBLORA_ERR_INVALID_ARG;
  if (k->heads != cache->kv_heads || v->heads != cache->kv_heads || cfg->head_dim != cache->head_dim) return QBLORA_ERR_INVALID_ARG;
  if (!in_place_ok(c.q, c.q_out, tokens) || q_out->data == k->data || q_out->data == v->data) return QBLORA_ERR_INVALID_ARG;
  c.positions = positions; c.slots = slots; c.T = tokens;
  return launch_rope(c, static_cast<cudaStream_t>(stream));
}

int qblora_kv_plan(const int32_t* ctx_len, const int32_t* new_len, const int32_t* release, int32_t n_requests,
                   int32_t* block_table, int32_t width, int32_t* free_pages, int32_t capacity, const int32_t* free_count,
                   int32_t* free_count_out, int32_t page_size, int32_t tokens, int32_t* cu_new, int32_t* kv_len,
                   int32_t* positions, int32_t* slots, int32_t* admitted, void* stream) {
  if (!int_ptr_ok(ctx_len) || !int_ptr_ok(new_len) || !int_ptr_ok(block_table) || !int_ptr_ok(free_pages)) return QBLORA_ERR_INVALID_ARG;
  if (!int_ptr_ok(free_count) || !int_ptr_ok(free_count_out) || free_count == free_count_out) return QBLORA_ERR_INVALID_ARG;
  if (!int_ptr_ok(cu_new) || !int_ptr_ok(kv_len) || !int_ptr_ok(positions) || !int_ptr_ok(slots) || !int_ptr_ok(admitted)) return QBLORA_ERR_INVALID_ARG;
  if (release && !int_ptr_ok(release)) return QBLORA_ERR_INVALID_ARG;
  if (n_requests < 1 || width < 1 || capacity < 1 || page_size < 1 || tokens < 1) return QBLORA_ERR_INVALID_ARG;
  if ((int64_t)capacity * page_size >= (int64_t)1 << 31 || (int64_t)width * page_size >= (int64_t)1 << 31) return QBLORA_ERR_INVALID_ARG;
  if (n_requests > kPlanMaxRequests) return QBLORA_ERR_UNSUPPORTED;
  // Every CTA reads the lengths for itself, whenever it runs: nothing that is written may lie in what is read, or in another output.
  const IntSpan arrays[] = {{block_table, (int64_t)n_requests * width}, {free_pages, capacity}, {free_count_out, 1}, {cu_new, n_requests + 1},
                            {kv_len, n_requests}, {positions, tokens}, {slots, tokens}, {admitted, n_requests},      // written
                            {ctx_len, n_requests}, {new_len, n_requests}, {release, n_requests}, {free_count, 1}};   // read only
  for (int i = 0; i < 8; ++i)
    for (int j = i + 1; j < 12; ++j)
      if (overlap(arrays[i], arrays[j])) return QBLORA_ERR_INVALID_ARG;
  PlanCall c{ctx_len, new_len, release, n_requests, block_table, width, free_pages, capacity, free_count, free_count_out,
             page_size, tokens, cu_new, kv_len, positions, slots, admitted};
  return launch_kv_plan(c, static_cast<cudaStream_t>(stream));
}

size_t qblora_attention_workspace_bytes(const qblora_kv_cache* cache, int32_t q_heads, int64_t tokens) {
  if (!cache || cache->kv_heads < 1 || q_heads < 1 || q_heads % cache->kv_heads || tokens < 1) return 0;
  if (cache->head_dim < 1 || cache->head_dim > 256) return 0;
  return kAttnResetBytes + paged_attention_scratch_bytes(cache->head_dim) + tc_attention_scratch_bytes(cache->head_dim);
}

int qblora_paged_attention(const qblora_kv_cache* cache, const int32_t* block_table, int32_t width, const int32_t* cu_new,
                           const int32_t* kv_len, int32_t n_requests, const qblora_heads* q, int64_t tokens, float scale,
                           int causal, int32_t window, const qblora_heads* out, float* lse, void* ws, size_t ws_bytes,
                           void* stream) {
  AttnCall c{};
  HeadsView qv, ov;
  if (!cache_ok(cache, &c.cache) || !heads_ok(q, &qv) || !heads_ok(out, &ov)) return QBLORA_ERR_INVALID_ARG;
  if (!int_ptr_ok(block_table) || !int_ptr_ok(cu_new) || !int_ptr_ok(kv_len) || (lse && !int_ptr_ok(lse))) return QBLORA_ERR_INVALID_ARG;
  if (width < 1 || n_requests < 1 || tokens < 1 || tokens >= (int64_t)1 << 31 || window < 0 || !std::isfinite(scale)) return QBLORA_ERR_INVALID_ARG;
  // key numbers are rounded up to whole tiles (of at most 128 keys) in 32 bits
  if ((int64_t)width * cache->page_size > ((int64_t)1 << 31) - 256) return QBLORA_ERR_INVALID_ARG;
  if (qv.dtype != QBLORA_BF16 || ov.dtype != QBLORA_BF16 || qv.heads != ov.heads || qv.heads % cache->kv_heads) return QBLORA_ERR_INVALID_ARG;
  if (cache->head_dim % 8) return QBLORA_ERR_INVALID_ARG;
  if (!aligned16(q->data) || !aligned16(out->data) || !aligned16(cache->k) || !aligned16(cache->v)) return QBLORA_ERR_INVALID_ARG;
  if (qv.ts % 8 || qv.hs % 8 || ov.ts % 8 || ov.hs % 8 || c.cache.ps % 8 || c.cache.ts % 8 || c.cache.hs % 8) return QBLORA_ERR_INVALID_ARG;
  if (cache->head_dim > 256 || tokens * q->heads >= (int64_t)1 << 31) return QBLORA_ERR_UNSUPPORTED;
  if (!ws || !aligned16(ws) || ws_bytes < qblora_attention_workspace_bytes(cache, q->heads, tokens)) return QBLORA_ERR_WORKSPACE;
  c.table = block_table; c.width = width; c.cu = cu_new; c.kv = kv_len; c.B = n_requests;
  c.q = static_cast<const __nv_bfloat16*>(qv.data); c.q_ts = qv.ts; c.q_hs = qv.hs;
  c.out = static_cast<__nv_bfloat16*>(ov.data); c.o_ts = ov.ts; c.o_hs = ov.hs;
  c.lse = lse; c.T = tokens; c.H = qv.heads; c.G = qv.heads / cache->kv_heads; c.D = cache->head_dim;
  c.scale = scale; c.causal = causal != 0; c.window = window;
  c.status = static_cast<int*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int rc = QBLORA_OK;
  if (!force_general()) {
    int cluster = 0;
    rc = paged_cluster_size(c, &cluster);
    if (rc) return rc;
    if (cluster) {
      // The status word: a kernel before this one may overlap with its beginning, which a memset may not, but costs the host more
      // to enqueue (1 request of 513 keys: 7.1 us and 10.3 us on the device, 14.7 us and 13.6 us for the host).  While a stream
      // is captured the device's time is what counts.
      cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
      QB_CUDA(cudaStreamIsCapturing(st, &capture));
      if (capture == cudaStreamCaptureStatusNone) QB_CUDA(cudaMemsetAsync(ws, 0, kStatusBytes, st));
      else rc = launch_attention_reset(ws, kStatusBytes, st);
      if (rc) return rc;
      return launch_paged_cluster(c, cluster, st);
    }
  }
  rc = launch_attention_reset(ws, kAttnResetBytes, st);
  if (rc) return rc;
  if (force_general()) return launch_simt_attention(c, st);
  char* wide_counters = static_cast<char*>(ws) + kStatusBytes;
  char* counters = wide_counters + kWideCounterBytes;
  char* scratch = counters + kPagedCounterBytes;
  if (!paged_warp_supported(c)) return launch_paged_attention(c, counters, scratch, st);
  const bool wide = tc_attention_supported(c) && tokens * c.G > kNarrowRows;     // there may be requests for the tcgen05 form
  char* wide_scratch = scratch + paged_attention_scratch_bytes(c.D);
  rc = launch_paged_warp(c, wide ? kNarrowRows : 0x7fffffff, counters, scratch, st);
  if (!rc && wide) rc = launch_tc_attention(c, kNarrowRows, wide_counters, wide_scratch, st);
  if (!rc) rc = launch_paged_join(c, counters, scratch, wide_counters, wide_scratch, st);
  return rc;
}

}  // extern "C"
