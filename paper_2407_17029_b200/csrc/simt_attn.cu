// Attention over the paged cache, general path: CUDA cores, any head size (a multiple of 8 up to 256), any page size and
// strides.  One CTA per (row, query head); its four warps take the row's keys in turn, each with the running maximum and
// sum of a softmax, and are joined in warp order at the end.  A key that the row does not see is never read.
//
// What bounds it: a row re-reads its keys from L2 for every query head and every new row, and each score is a warp-wide
// reduction.  It is the path for what the tensor-core kernels do not take, and what they are checked against.  Measured: 64
// requests decoding over up to 8100 keys, 8 key heads of 4: 3.1 ms (0.35 TB/s); 512 tokens behind 512 keys: 2.3 ms (2.8 TFLOP/s).
#include "serving.cuh"

namespace qb {
namespace {

constexpr int SA_WARPS = 4;
constexpr int SA_MAX_PER_LANE = 8;   // 256 / 32

__global__ void __launch_bounds__(SA_WARPS * 32) simt_attention_kernel(const __grid_constant__ AttnCall c) {
  __shared__ float s_m[SA_WARPS], s_l[SA_WARPS], s_o[SA_WARPS][256];
  const int h = blockIdx.x % c.H;
  const int64_t t = blockIdx.x / c.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the request of row t: the last b with cu[b] <= t whose rows reach past t
  int lo_b = 0, hi_b = c.B;
  while (lo_b < hi_b) {
    const int mid = (lo_b + hi_b) >> 1;
    if ((int64_t)__ldg(c.cu + mid + 1) <= t) lo_b = mid + 1; else hi_b = mid;
  }
  if (lo_b >= c.B) return;
  const ReqView r = attn_request(c, lo_b);
  if (t < r.t0 || t >= r.t0 + r.n) return;
  const int p = r.kv - r.n + (int)(t - r.t0);
  const int hi = attn_hi(c, r.kv, p), lo = min(attn_lo(c, p), hi);
  const int hk = h / c.G;
  const int pairs = c.D >> 1;   // lane holds pairs lane, lane + 32, ...: coalesced 4-byte loads

  float2 q[SA_MAX_PER_LANE / 2], o[SA_MAX_PER_LANE / 2];
  const __nv_bfloat16* qr = c.q + t * c.q_ts + (int64_t)h * c.q_hs;
#pragma unroll
  for (int i = 0; i < SA_MAX_PER_LANE / 2; ++i) {
    const int j = lane + 32 * i;
    q[i] = j < pairs ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(qr + 2 * j)) : make_float2(0.f, 0.f);
    o[i] = make_float2(0.f, 0.f);
  }
  float m = -INFINITY, l = 0.f;
  const int* row = c.table + (int64_t)lo_b * c.width;
  for (int j = lo + warp; j < hi; j += SA_WARPS) {
    const int page = __ldg(row + j / c.cache.page_size);
    if (page < 0 || page >= c.cache.n_pages) {
      if (lane == 0) atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
      continue;
    }
    const int64_t off = (int64_t)page * c.cache.ps + (int64_t)(j % c.cache.page_size) * c.cache.ts + (int64_t)hk * c.cache.hs;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < SA_MAX_PER_LANE / 2; ++i) {
      const int e = lane + 32 * i;
      if (e < pairs) {
        const float2 k = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(c.cache.k + off + 2 * e));
        s = fmaf(q[i].x, k.x, s);
        s = fmaf(q[i].y, k.y, s);
      }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= c.scale;
    const float mn = fmaxf(m, s);
    // before the first finite score both may be -infinity: the weight of such a key is zero
    const float f = mn == -INFINITY ? 0.f : expf(m - mn);
    const float w = mn == -INFINITY ? (s != s ? s : 0.f) : expf(s - mn);
    m = mn;
    l = l * f + w;
#pragma unroll
    for (int i = 0; i < SA_MAX_PER_LANE / 2; ++i) {
      const int e = lane + 32 * i;
      if (e < pairs) {
        const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(c.cache.v + off + 2 * e));
        o[i].x = fmaf(w, v.x, o[i].x * f);
        o[i].y = fmaf(w, v.y, o[i].y * f);
      }
    }
  }
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
  for (int i = 0; i < SA_MAX_PER_LANE / 2; ++i) {
    const int e = lane + 32 * i;
    if (e < pairs) { s_o[warp][2 * e] = o[i].x; s_o[warp][2 * e + 1] = o[i].y; }
  }
  __syncthreads();
  float M = -INFINITY;
  for (int w = 0; w < SA_WARPS; ++w) M = fmaxf(M, s_m[w]);
  float L = 0.f, f[SA_WARPS];
  for (int w = 0; w < SA_WARPS; ++w) {
    f[w] = s_m[w] == -INFINITY ? (s_l[w] != s_l[w] ? s_l[w] : 0.f) : expf(s_m[w] - M);
    L += s_l[w] * f[w];
  }
  __nv_bfloat16* out = c.out + t * c.o_ts + (int64_t)h * c.o_hs;
  for (int d = threadIdx.x; d < c.D; d += SA_WARPS * 32) {
    float a = 0.f;
    for (int w = 0; w < SA_WARPS; ++w) a += f[w] == 0.f ? 0.f : s_o[w][d] * f[w];
    out[d] = __float2bfloat16_rn(L == 0.f ? 0.f : a / L);
  }
  if (c.lse && threadIdx.x == 0) c.lse[t * c.H + h] = L == 0.f ? -INFINITY : M + logf(L);
}

}  // namespace

int launch_simt_attention(const AttnCall& c, cudaStream_t st) {
  if (c.T * c.H >= (int64_t)1 << 31) return QBLORA_ERR_UNSUPPORTED;
  simt_attention_kernel<<<(unsigned)(c.T * c.H), SA_WARPS * 32, 0, st>>>(c);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

}  // namespace qb
