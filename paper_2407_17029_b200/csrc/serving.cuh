// Shared declarations of the calls between the products of a served layer: rotary positions, the paged cache's plan
// and the attention over it (include/qblora.h, last part).
#pragma once
#include "common.cuh"

namespace qb {

struct HeadsView {
  void* data;
  int64_t ts, hs;   // token and head stride, elements
  int heads, dtype;
};

struct CacheView {
  __nv_bfloat16 *k, *v;
  int64_t ps, ts, hs;   // page, entry and head stride, elements
  int n_pages, page_size, kv_heads;
};

struct RopeView {
  int D, rot, layout;
  float amp, sign;   // sign: +1 forward, -1 inverse
  const uint64_t* turns;
};

// y2 / cache: see qblora_rope and qblora_rope_append.  v.data == nullptr: plain rotation of one or two tensors.
struct RopeCall {
  RopeView cfg;
  const int* positions;
  const int* slots;
  int64_t T;
  HeadsView q, k, v, q_out, k_out;   // heads == 0: not there
  CacheView cache;                   // used when slots != nullptr: k and v go there
};
int launch_rope(const RopeCall& c, cudaStream_t st);

struct PlanCall {
  const int *ctx, *add, *release;
  int B;
  int* table; int width;
  int* stack; int capacity;
  const int* count; int* count_out;
  int page, T;
  int *cu, *kv, *pos, *slots, *admitted;
};
constexpr int kPlanMaxRequests = 8192;
int launch_kv_plan(const PlanCall& c, cudaStream_t st);

struct AttnCall {
  CacheView cache;
  const int* table; int width;
  const int *cu, *kv; int B;
  const __nv_bfloat16* q; int64_t q_ts, q_hs;
  __nv_bfloat16* out; int64_t o_ts, o_hs;
  float* lse;
  int64_t T;
  int H, G, D;          // query heads, query heads per key head, head size
  float scale;
  int causal, window;
  int* status;
};

// Rows and keys of one request, with every length forced into its range (they come from device memory).
struct ReqView { int t0, n, kv; };
__device__ __forceinline__ ReqView attn_request(const AttnCall& c, int b) {
  ReqView r;
  const int T = (int)c.T;
  r.t0 = min(max(__ldg(c.cu + b), 0), T);
  const int t1 = min(max(__ldg(c.cu + b + 1), r.t0), T);
  r.n = t1 - r.t0;
  const long long most = (long long)c.width * c.cache.page_size;
  r.kv = (int)min((long long)max(__ldg(c.kv + b), 0), most);
  return r;
}
// Keys [lo, hi) that the row at position p (may be negative) sees.
__device__ __forceinline__ int attn_hi(const AttnCall& c, int kv, int p) { return c.causal ? max(0, min(kv, p + 1)) : kv; }
__device__ __forceinline__ int attn_lo(const AttnCall& c, int p) { return c.window > 0 && p >= c.window ? p - c.window + 1 : 0; }

// ---- attention: layout of the caller's workspace, after the status word
//   counters that every call zeroes (launch_attention_reset), then the parts of paged_attn.cu or paged_warp.cu, then those of
//   tc_attn.cu
constexpr int kPagedMaxSms = 160, kPagedMaxPerSm = 4;       // resident CTAs of paged_attn.cu
constexpr int kPagedWarps = 8, kPagedLevels = 4;            // warps per SM, and shares per warp, of paged_warp.cu
constexpr int kPagedMaxShares = kPagedMaxSms * kPagedWarps * kPagedLevels;
constexpr int kWideRounds = 3, kWideMaxShares = kPagedMaxSms * kWideRounds;     // of tc_attn.cu
constexpr size_t kWideCounterBytes = 256;
constexpr size_t kPagedCounterBytes = (size_t)(1 + kPagedMaxShares) * 4 / 256 * 256 + 256;
constexpr size_t kAttnResetBytes = kStatusBytes + kWideCounterBytes + kPagedCounterBytes;
int launch_attention_reset(void* ws, size_t bytes, cudaStream_t st);    // zeroes that many, a multiple of 16

// Any head size up to 256, any page size and strides that are multiples of 8 elements (paged_attn.cu).
size_t paged_attention_scratch_bytes(int head_dim);
int launch_paged_attention(const AttnCall& c, char* counters, char* scratch, cudaStream_t st);

// An item that shares cut: `n` parts.  Of paged_warp.cu: part 0 in slot `slot0`, part i in slot 2 (first + i kv_heads).  Of tc_attn.cu,
// one row tile of it: part 0 in slot 2 slot0 + tile, part i in slot 4 (first + i) + tile.
struct JoinCut { int slot0, first, n, t0, r0, rows, h, tile; };
constexpr int kJoinThreads = 256, kJoinShort = 32, kJoinWideShort = 8;
struct JoinCall {
  const uint32_t* counts;     // [3]: items of at most kJoinShort parts; of more; most rows of an item
  const JoinCut* cuts;        // [kPagedMaxShares]: the first from the front, the others from the back
  const float *part_o, *part_ml;
  int rows_per_slot;
  uint32_t div_group;
  const uint32_t* wide_counts;   // [2]: row tiles of at most kJoinWideShort parts; of more
  const JoinCut* wide_cuts;      // [2 kWideMaxShares] likewise
  const float *wide_o, *wide_ml; // [slot][D / 4][128 rows][4], [slot][128][2]
};

// Few rows per key head, head sizes 64 and 128, pages that fit its tiles (paged_warp.cu): requests of at most `narrow_rows` rows
// (new tokens * G).
bool paged_warp_supported(const AttnCall& c);
int launch_paged_warp(const AttnCall& c, int narrow_rows, char* counters, char* scratch, cudaStream_t st);
// Joins the parts that it and tc_attn.cu have left.  A kernel launched between may not end before the kernels in front of it.
int launch_paged_join(const AttnCall& c, char* counters, char* scratch, char* wide_counters, char* wide_scratch, cudaStream_t st);

// The same kernel for calls so small that every item has a cluster of CTAs to itself: one launch, no workspace but the status
// word (zeroed on the stream).  paged_cluster_size gives the CTAs per cluster, 0 where the call is none of these.
int paged_cluster_size(const AttnCall& c, int* size);
int launch_paged_cluster(const AttnCall& c, int size, cudaStream_t st);

// Many rows per key head (tc_attn.cu): requests with more than `narrow_rows` rows.  Launched behind launch_paged_warp, beside whose
// kernels it may start as SMs become free.
constexpr int kWideMaxRequests = 1024;
bool tc_attention_supported(const AttnCall& c);
size_t tc_attention_scratch_bytes(int head_dim);
void tc_attention_join(int head_dim, char* counters, char* scratch, JoinCall* j);     // the wide part of it
int launch_tc_attention(const AttnCall& c, int narrow_rows, char* counters, char* scratch, cudaStream_t st);

// TMA maps (CUtensorMap) of the cache's K and V.
int make_cache_maps(const AttnCall& c, int box_keys, void* tm_k, void* tm_v);

// General path: any head size up to 256, any page size.
int launch_simt_attention(const AttnCall& c, cudaStream_t st);

}  // namespace qb
