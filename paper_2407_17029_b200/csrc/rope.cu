// Rotary positions (qblora_rope) and their serving form that writes the paged cache (qblora_rope_append).
//
// Pair j of a head at position p is turned by p * f_j turns.  The table holds f_j in units of 2^-64 turns, so the angle
// modulo one turn is the low 64 bits of one integer product; its top 32 bits, read as a signed number, are the angle in
// units of 2^-32 turns, exact at every position (a product in fp32 is off by a hundredth of a radian at position 10^5).
//
// What bounds it: HBM, every element read once and written once, in 16-byte words with several loads in flight per thread.
// Measured: fp32, 8191 rows of 40 + 40 heads of 128, 671 MB: 119.5 us = 5.6 TB/s (a copy: 6.5); bf16, 4095 rows of
// 52 + 52 + 52 heads into a cache, 327 MB: 57.8 us = 5.7 TB/s; one row: 2.4 us in a graph.
// Sizes and alignments of the general form (below): 4095 rows of 32 + 32 heads of 96, 24 of them rotated, 127 us where the
// bytes take 16 (with 32 rotated, the wide form: 20 us): a sine and 64-bit divisions for each pair of each head.
#include "serving.cuh"

namespace qb {
namespace {

__device__ __forceinline__ void rope_angle(const RopeView& r, int pos, int pair, float& co, float& si) {
  const uint64_t phase = (uint64_t)(int64_t)pos * __ldg(r.turns + pair);
  const float half_turns = (float)(int32_t)(phase >> 32) * (1.0f / 2147483648.0f);   // angle / pi, in [-1, 1)
  sincospif(half_turns, &si, &co);
  co *= r.amp;
  si *= r.amp * r.sign;
}

// offset of head 0 of slot's entry, or -1
__device__ __forceinline__ int64_t cache_entry(const CacheView& c, int slot) {
  if (slot < 0) return -1;
  const int page = slot / c.page_size;
  if (page >= c.n_pages) return -1;
  return (int64_t)page * c.ps + (int64_t)(slot - page * c.page_size) * c.ts;
}

__device__ __forceinline__ float ld1(const float* p) { return *p; }
__device__ __forceinline__ float ld1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st1(float* p, float x) { *p = x; }
__device__ __forceinline__ void st1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Eight consecutive values, as loaded (so that several loads can be on their way) and as floats.
template <typename T> struct Eight;
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
template <> struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
__device__ __forceinline__ void st8(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void st8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Where head h of the concatenated list (q heads, k heads, v heads) of row t comes from and goes to.
template <typename TI, typename TO>
struct Place {
  const TI* src;
  TO* dst;        // nullptr: nothing is written
  bool rotate;
};
template <typename TI, typename TO>
__device__ __forceinline__ Place<TI, TO> place(const RopeCall& c, int64_t t, int64_t entry, int h) {
  Place<TI, TO> r;
  r.rotate = true;
  if (h < c.q.heads) {
    r.src = static_cast<const TI*>(c.q.data) + t * c.q.ts + (int64_t)h * c.q.hs;
    r.dst = static_cast<TO*>(c.q_out.data) + t * c.q_out.ts + (int64_t)h * c.q_out.hs;
    return r;
  }
  h -= c.q.heads;
  if (h < c.k.heads) {
    r.src = static_cast<const TI*>(c.k.data) + t * c.k.ts + (int64_t)h * c.k.hs;
    if (c.slots) r.dst = entry < 0 ? nullptr : reinterpret_cast<TO*>(c.cache.k) + entry + (int64_t)h * c.cache.hs;
    else r.dst = static_cast<TO*>(c.k_out.data) + t * c.k_out.ts + (int64_t)h * c.k_out.hs;
    return r;
  }
  h -= c.k.heads;
  r.rotate = false;
  r.src = static_cast<const TI*>(c.v.data) + t * c.v.ts + (int64_t)h * c.v.hs;
  r.dst = entry < 0 ? nullptr : reinterpret_cast<TO*>(c.cache.v) + entry + (int64_t)h * c.cache.hs;
  return r;
}

// Wide form.  A CTA takes `tokens` rows and a range of heads: it puts the sines of its rows into shared memory, each once, and
// its threads then own one chunk of a row each -- 16 elements that hold eight whole pairs (or 16, or the last 8, elements
// behind the rotated part) -- for every `per`-th head.  Loads of 64 bytes in flight per thread and four CTAs per SM carry it
// (64 registers): 5.7 TB/s at 4095 rows of 52 + 52 + 52 heads, against 4.8 TB/s with twice the loads and half the CTAs.
constexpr int RW_THREADS = 256, RW_TOKENS = 4, RW_MAX_PAIRS = 128;

template <typename TI, typename TO, int LAYOUT>
__global__ void __launch_bounds__(RW_THREADS, 4) rope_wide_kernel(const __grid_constant__ RopeCall c, int chunks, int tokens, int heads_per_cta) {
  __shared__ float s_cos[RW_TOKENS * RW_MAX_PAIRS], s_sin[RW_TOKENS * RW_MAX_PAIRS];
  const int tid = threadIdx.x, pairs = c.cfg.rot >> 1;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int n = (int)min((int64_t)tokens, c.T - t0);
  const int n_heads = c.q.heads + c.k.heads + c.v.heads;
  const int h0 = blockIdx.y * heads_per_cta, h1 = min(h0 + heads_per_cta, n_heads);
  if (h0 < c.q.heads + c.k.heads) {
    for (int i = tid; i < n * pairs; i += RW_THREADS) {
      const int tt = i / pairs, pair = i - tt * pairs;
      rope_angle(c.cfg, __ldg(c.positions + t0 + tt), pair, s_cos[tt * RW_MAX_PAIRS + pair], s_sin[tt * RW_MAX_PAIRS + pair]);
    }
  }
  __syncthreads();
  const int chunk = tid % chunks, slot = tid / chunks, per = RW_THREADS / chunks;
  if (slot >= per) return;
  const int rot_chunks = c.cfg.rot >> 4;
  const bool rot = chunk < rot_chunks;
  int e0, e1;      // first elements of the chunk's two halves of eight
  if (rot) {
    if (LAYOUT == QBLORA_ROPE_HALF) { e0 = chunk * 8; e1 = e0 + pairs; }
    else { e0 = chunk * 16; e1 = e0 + 8; }
  } else {
    e0 = c.cfg.rot + (chunk - rot_chunks) * 16;
    e1 = e0 + 8 < c.cfg.D ? e0 + 8 : -1;
  }
  for (int tt = 0; tt < n; ++tt) {
    const int64_t t = t0 + tt;
    const int64_t entry = c.slots ? cache_entry(c.cache, __ldg(c.slots + t)) : -1;
    const float *co = s_cos + tt * RW_MAX_PAIRS + chunk * 8, *si = s_sin + tt * RW_MAX_PAIRS + chunk * 8;
    // UNROLL heads at a time: all their loads go out before the first store (a store may alias a load, so the compiler would not
    // move one in front of the other)
    constexpr int UNROLL = sizeof(TI) == 2 ? 2 : 1;
    for (int hb = h0 + slot; hb < h1; hb += UNROLL * per) {
      Eight<TI> ra[UNROLL], rb[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (hb + u * per >= h1) break;
        const Place<TI, TO> w = place<TI, TO>(c, t, entry, hb + u * per);
        ra[u].load(w.src + e0);
        if (e1 >= 0) rb[u].load(w.src + e1);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (hb + u * per >= h1) break;
        const Place<TI, TO> w = place<TI, TO>(c, t, entry, hb + u * per);
        float a[8], b[8];
        ra[u].get(a);
        if (e1 >= 0) rb[u].get(b);
        if (rot && w.rotate) {
          if (LAYOUT == QBLORA_ROPE_HALF) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = a[i], y = b[i];
              a[i] = x * co[i] - y * si[i];
              b[i] = y * co[i] + x * si[i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = a[2 * i], y = a[2 * i + 1];
              a[2 * i] = x * co[i] - y * si[i];
              a[2 * i + 1] = y * co[i] + x * si[i];
              x = b[2 * i]; y = b[2 * i + 1];
              b[2 * i] = x * co[4 + i] - y * si[4 + i];
              b[2 * i + 1] = y * co[4 + i] + x * si[4 + i];
            }
          }
        }
        if (w.dst) {
          st8(w.dst + e0, a);
          if (e1 >= 0) st8(w.dst + e1, b);
        }
      }
    }
  }
}

// Any strides, alignment and even rotary size: one pair (or one element behind the rotated part) of one head per thread.
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) rope_any_kernel(const __grid_constant__ RopeCall c) {
  const int pairs = c.cfg.rot >> 1, items = pairs + (c.cfg.D - c.cfg.rot);
  const int n_heads = c.q.heads + c.k.heads + c.v.heads;
  const int64_t total = c.T * n_heads * items;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
    const int item = (int)(id % items);
    const int64_t rest = id / items;
    const int h = (int)(rest % n_heads);
    const int64_t t = rest / n_heads;
    const int64_t entry = c.slots ? cache_entry(c.cache, __ldg(c.slots + t)) : -1;
    const Place<TI, TO> w = place<TI, TO>(c, t, entry, h);
    if (!w.dst) continue;
    if (item >= pairs) {
      const int e = c.cfg.rot + item - pairs;
      st1(w.dst + e, ld1(w.src + e));
      continue;
    }
    const int e0 = c.cfg.layout == QBLORA_ROPE_HALF ? item : 2 * item;
    const int e1 = c.cfg.layout == QBLORA_ROPE_HALF ? item + pairs : 2 * item + 1;
    float x = ld1(w.src + e0), y = ld1(w.src + e1);
    if (w.rotate) {
      float co, si;
      rope_angle(c.cfg, __ldg(c.positions + t), item, co, si);
      const float u = x * co - y * si;
      y = y * co + x * si;
      x = u;
    }
    st1(w.dst + e0, x);
    st1(w.dst + e1, y);
  }
}

bool heads_wide(const HeadsView& v) {
  if (v.heads == 0) return true;
  const int per16 = v.dtype == QBLORA_BF16 ? 8 : 4;
  return aligned16(v.data) && v.ts % per16 == 0 && v.hs % per16 == 0;
}

template <typename TI, typename TO>
int launch_typed(const RopeCall& c, cudaStream_t st) {
  const int n_heads = c.q.heads + c.k.heads + c.v.heads;
  bool wide = c.cfg.D % 8 == 0 && c.cfg.rot % 16 == 0 && heads_wide(c.q) && heads_wide(c.k) && heads_wide(c.v) &&
              heads_wide(c.q_out) && heads_wide(c.k_out);
  if (c.slots)
    wide = wide && aligned16(c.cache.k) && aligned16(c.cache.v) && c.cache.ps % 8 == 0 && c.cache.ts % 8 == 0 && c.cache.hs % 8 == 0;
  const int chunks = c.cfg.rot / 16 + (c.cfg.D - c.cfg.rot + 15) / 16;
  if (wide && c.cfg.rot <= 2 * RW_MAX_PAIRS && chunks <= RW_THREADS) {
    const int per = RW_THREADS / chunks;
    // rows per CTA: more share the set-up, as long as the device is full several times over; few rows: heads over CTAs instead
    int tokens = RW_TOKENS, split = 1;
    while (tokens > 1 && c.T < (int64_t)tokens * 148 * 8) tokens >>= 1;
    const int most = (n_heads + per - 1) / per;
    while (split < most && c.T * split < 148 * 2) ++split;
    const int heads_per_cta = (most + split - 1) / split * per;
    const dim3 grid((unsigned)((c.T + tokens - 1) / tokens), (unsigned)((n_heads + heads_per_cta - 1) / heads_per_cta));
    if ((c.T + tokens - 1) / tokens > 0x7fffffff) return QBLORA_ERR_UNSUPPORTED;
    if (c.cfg.layout == QBLORA_ROPE_HALF) rope_wide_kernel<TI, TO, QBLORA_ROPE_HALF><<<grid, RW_THREADS, 0, st>>>(c, chunks, tokens, heads_per_cta);
    else rope_wide_kernel<TI, TO, QBLORA_ROPE_PAIRS><<<grid, RW_THREADS, 0, st>>>(c, chunks, tokens, heads_per_cta);
  } else {
    const int64_t total = c.T * n_heads * (c.cfg.D - c.cfg.rot / 2);
    int64_t blocks = (total + 255) / 256;
    if (blocks > 148 * 16) blocks = 148 * 16;
    rope_any_kernel<TI, TO><<<(unsigned)blocks, 256, 0, st>>>(c);
  }
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

}  // namespace

int launch_rope(const RopeCall& c, cudaStream_t st) {
  const bool in32 = c.q.dtype == QBLORA_F32, out32 = !c.slots && c.q_out.dtype == QBLORA_F32;
  if (in32) return out32 ? launch_typed<float, float>(c, st) : launch_typed<float, __nv_bfloat16>(c, st);
  return out32 ? launch_typed<__nv_bfloat16, float>(c, st) : launch_typed<__nv_bfloat16, __nv_bfloat16>(c, st);
}

}  // namespace qb
