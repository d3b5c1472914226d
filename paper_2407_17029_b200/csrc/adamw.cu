// AdamW over many tensors at once, states in 32 bits or in 8, with the global gradient norm and clipping
// (qblora_adamw_prepare, qblora_adamw_step; the formulas stand in include/qblora.h).
//
// What bounds it: memory with states in 32 bits, 30 bytes an element (p, m, v in and out, g in, the bf16 copy out): 125 M elements in 607
// us, 6.2 TB/s.  With states in 8 bits, 16 to 18 bytes an element, the instructions (640 for a warp's 256 elements, 2.0 to 2.3 a cycle) and,
// behind them, the wait for loads (3.9 of the stalls an issue): 480 us, and 68 for the norm's pass over bf16 gradients (3.7 TB/s); more bytes on
// their way, by more CTAs an SM or asynchronous copies, changed nothing (488 to 653).  At the 80 registers that three CTAs an SM leave, two
// blocks in flight beside a copy of the tensor's table entry in every lane do not fit: adamw_kernel<8> spills 100 bytes of stores and 148 of
// loads a thread, adamw_kernel<0> 112 and 260, adamw_kernel<32> 8 and 12.  The unit of work is a block of 256 consecutive elements of one tensor, one warp's 8 elements per lane: a scale's block lies
// within a warp, so its maximum is five shuffles and no element is read twice.  The tensors are a table in the workspace; a warp takes
// runs of neighbouring blocks and searches the first blocks for their tensor where the last one's does not fit.  Lane l holds elements 4 l
// .. 4 l + 3 and 128 + 4 l .. of the block, so every load and store of a warp is one contiguous run.
//
// One launch without the norm, two with it: the step's count is read by every CTA as it starts and written by the CTA that
// ends last.
#include <cfloat>
#include <cmath>

#include <cuda_fp16.h>

#include "common.cuh"

namespace qb {
namespace {

constexpr int AW_BLOCK = 256, AW_WARPS = 8, AW_THREADS = AW_WARPS * 32;
constexpr int AW_NORM_CTAS = 592;              // most CTAs of the norm kernel: 4 on each of 148 SMs
constexpr int AW_MAX_TENSORS = 65536;

struct AwTensor {
  float* p; const void* g; __nv_bfloat16* copy; void* m; void* v; float* m_scale; float* v_scale;
  long long n;
  uint32_t first;                              // its first block
  int g16, bits8, wide;                        // wide: every pointer allows the vector accesses
  float lr_mult, decay;
};

// The workspace: control words, the norm's parts, the table, the first blocks.
struct AwControl {
  uint32_t norm_ticket, step_ticket;           // CTAs that have come to their end; back to 0 after every call
  float factor;                                // of the gradients; negative: leave the step out
  uint32_t blocks;                             // of all tensors
};
constexpr size_t kAwParts = kStatusBytes;
constexpr size_t kAwTable = kAwParts + AW_NORM_CTAS * 8 + 128;
static_assert(sizeof(AwControl) <= kStatusBytes && kAwTable % 16 == 0, "layout");
size_t aw_first_at(int n) { return kAwTable + align_up((size_t)n * sizeof(AwTensor), 16); }

struct AwView {
  AwControl* ctl; double* parts; const AwTensor* table; const uint32_t* first; int n;
};
AwView aw_view(void* ws, int n) {
  char* w = static_cast<char*>(ws);
  return {reinterpret_cast<AwControl*>(w), reinterpret_cast<double*>(w + kAwParts), reinterpret_cast<const AwTensor*>(w + kAwTable),
          reinterpret_cast<const uint32_t*>(w + aw_first_at(n)), n};
}

struct AwStep {
  AwView w;
  const float* lr; int* steps; float* norm;
  double log_b1, log_b2, max_norm;             // log: -infinity for a beta of 0
  float b1, b2, c1, c2, eps;                   // c = 1 - beta
  uint32_t seed;
  int clipped;                                 // the norm kernel runs in front
};

// ---- the table ---------------------------------------------------------------------------------------------------------
constexpr int AW_TABLE_PART = 32;              // entries per launch: they travel as kernel arguments
struct AwTablePart { AwTensor t[AW_TABLE_PART]; };
__global__ void __launch_bounds__(AW_TABLE_PART) adamw_table_kernel(const __grid_constant__ AwTablePart part, int at, int count, int n,
                                                                    uint32_t blocks, char* ws, size_t first_at) {
  const int i = threadIdx.x;
  AwTensor* table = reinterpret_cast<AwTensor*>(ws + kAwTable);
  uint32_t* first = reinterpret_cast<uint32_t*>(ws + first_at);
  if (i < count) { table[at + i] = part.t[i]; first[at + i] = part.t[i].first; }
  if (at + count == n && i == 0) {
    first[n] = blocks;
    AwControl* c = reinterpret_cast<AwControl*>(ws);
    *c = AwControl{0u, 0u, 1.0f, blocks};
  }
}

// tensor of block b: the last k with first[k] <= b that has blocks.  `k` is a guess: the tensor of the warp's block before.
__device__ __forceinline__ int aw_find(const AwView& w, uint32_t b, int k) {
  if (__ldg(w.first + k) <= b && b < __ldg(w.first + k + 1)) return k;
  int lo = 0, hi = w.n;                        // first[lo] <= b < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(w.first + mid) <= b) lo = mid; else hi = mid;
  }
  return lo;
}

// ---- 256 elements of a warp: lane l holds 4 l + e and 128 + 4 l + e in x[e] and x[4 + e] -------------------------------------
__device__ __forceinline__ int aw_elem(int lane, int i) { return (i >> 2) * 128 + 4 * lane + (i & 3); }

template <bool FULL>
__device__ __forceinline__ void aw_load_f32(const float* a, long long base, int left, int lane, float (&x)[8]) {
  if constexpr (FULL) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 v = *reinterpret_cast<const float4*>(a + base + h * 128 + 4 * lane);
      x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = aw_elem(lane, i) < left ? a[base + aw_elem(lane, i)] : 0.f;
  }
}
template <bool FULL>
__device__ __forceinline__ void aw_store_f32(float* a, long long base, int left, int lane, const float (&x)[8]) {
  if constexpr (FULL) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float4*>(a + base + h * 128 + 4 * lane) = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (aw_elem(lane, i) < left) a[base + aw_elem(lane, i)] = x[i];
  }
}
template <bool FULL>
__device__ __forceinline__ void aw_load_g(const AwTensor& t, long long base, int left, int lane, float (&x)[8]) {
  if (!t.g16) { aw_load_f32<FULL>(static_cast<const float*>(t.g), base, left, lane, x); return; }
  const __nv_bfloat16* a = static_cast<const __nv_bfloat16*>(t.g);
  if constexpr (FULL) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 v = *reinterpret_cast<const uint2*>(a + base + h * 128 + 4 * lane);
      x[4 * h] = __uint_as_float(v.x << 16); x[4 * h + 1] = __uint_as_float(v.x & 0xffff0000u);
      x[4 * h + 2] = __uint_as_float(v.y << 16); x[4 * h + 3] = __uint_as_float(v.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = aw_elem(lane, i) < left ? __bfloat162float(a[base + aw_elem(lane, i)]) : 0.f;
  }
}

// Two fp32 operations in one instruction, each rounded by itself.
__device__ __forceinline__ unsigned long long aw_two(float a, float b) {
  unsigned long long v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ void aw_split(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ unsigned long long aw_mul2(unsigned long long a, unsigned long long b) {
  unsigned long long v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ unsigned long long aw_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ float aw_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float aw_sqrt(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float aw_max(float a, float b) {          // NaN if one is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// ---- 8-bit states --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t aw_mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xA3C59AC3u;
  x = (x ^ (x >> 15)) * 0x5D8E3B97u;
  return x ^ (x >> 16);
}
// eight e4m3 codes -> fp32 (exact) times the scale
__device__ __forceinline__ void aw_from_codes(const uint32_t (&w)[2], float scale, float (&x)[8]) {
  const unsigned long long both = aw_two(scale, scale);
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    uint32_t p;
    asm("{\n .reg .b16 c;\n cvt.u16.u32 c, %1;\n cvt.rn.f16x2.e4m3x2 %0, c;\n}" : "=r"(p) : "r"(w[h >> 1] >> (16 * (h & 1))));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p));
    aw_split(aw_mul2(aw_two(f.x, f.y), both), x[2 * h], x[2 * h + 1]);
  }
}
template <bool FULL>
__device__ __forceinline__ void aw_load_codes(const void* a, long long base, int left, int lane, uint32_t (&w)[2]) {
  const uint8_t* c = static_cast<const uint8_t*>(a);
  w[0] = w[1] = 0u;
  if constexpr (FULL) {
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = *reinterpret_cast<const uint32_t*>(c + base + h * 128 + 4 * lane);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (aw_elem(lane, i) < left) w[i >> 2] |= (uint32_t)c[base + aw_elem(lane, i)] << (8 * (i & 3));
  }
}
// The neighbour of |y| by chance: with y 2^-120, e4m3's exponent is at the lower end of fp32's, where its subnormal numbers are subnormal
// too, and 20 bits of the mantissa are to go.  What the random bits, added to the upper 16 of them, carry out decides.  The code comes
// in the top byte of the result (y's sign is shifted out).  RND: which 16 of the random bits, as a byte permutation that puts them into
// the middle bytes.  The block's largest y may be three units of fp32 above 448 (its factor and the product are rounded): 3 + 16 * 65535
// still carries nothing out.
template <uint32_t RND>
__device__ __forceinline__ uint32_t aw_round(float y, uint32_t rnd) {
  uint32_t low;          // (as assembly: the compiler folds this permutation and the ones that gather the codes into zeros)
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(low) : "r"(rnd), "n"(RND));
  return (__float_as_uint(y) << 4) + low;
}
constexpr uint32_t AW_LOW = 0x4104, AW_HIGH = 0x4324;
// SIGNED: else no x is below zero.
template <bool FULL, uint32_t RND, bool SIGNED>
__device__ __forceinline__ void aw_store_codes(void* a, float* scale, long long base, int left, int lane, const float (&x)[8],
                                               const uint32_t (&rnd)[8]) {
  float most = fabsf(x[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) most = aw_max(most, fabsf(x[i]));
  uint32_t all = __reduce_max_sync(0xffffffffu, __float_as_uint(most) & 0x7fffffffu);    // bits order like the numbers, NaN above all
  const bool odd = all >= 0x7f800000u;         // NaN or infinity: they do not count
  if (odd) {
    all = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t y = __float_as_uint(x[i]) & 0x7fffffffu;
      if (y < 0x7f800000u) all = max(all, y);
    }
    all = __reduce_max_sync(0xffffffffu, all);
  }
  float top = __uint_as_float(all);
  if (top < 0x1p-118f) top = 0.f;
  const float inv = top > 0.f ? __fmul_rn(__frcp_rn(top), 448.0f) : 0.f;
  const unsigned long long inv2 = aw_two(inv, inv), down2 = aw_two(0x1p-120f, 0x1p-120f);
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t z[4];
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      float y0, y1;
      aw_split(aw_mul2(aw_mul2(aw_two(x[4 * h + e], x[4 * h + e + 1]), inv2), down2), y0, y1);
      z[e] = aw_round<RND>(y0, rnd[4 * h + e]);
      z[e + 1] = aw_round<RND>(y1, rnd[4 * h + e + 1]);
    }
    w[h] = __byte_perm(__byte_perm(z[0], z[1], 0x0073), __byte_perm(z[2], z[3], 0x0073), 0x5410);
    if (SIGNED) {
      const float* y = x + 4 * h;
      const uint32_t sign = __byte_perm(__byte_perm(__float_as_uint(y[0]), __float_as_uint(y[1]), 0x0073),
                                        __byte_perm(__float_as_uint(y[2]), __float_as_uint(y[3]), 0x0073), 0x5410);
      w[h] = (w[h] & 0x7f7f7f7fu) | (sign & 0x80808080u);
    }
  }
  if (odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((__float_as_uint(x[i]) & 0x7fffffffu) >= 0x7f800000u) w[i >> 2] |= 0x7fu << (8 * (i & 3));
  }
  uint8_t* c = static_cast<uint8_t*>(a);
  if constexpr (FULL) {
    *reinterpret_cast<uint32_t*>(c + base + 4 * lane) = w[0];
    *reinterpret_cast<uint32_t*>(c + base + 128 + 4 * lane) = w[1];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (aw_elem(lane, i) < left) c[base + aw_elem(lane, i)] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
  if (lane == 0) *scale = top * (1.0f / 448.0f);
}

// ---- the step --------------------------------------------------------------------------------------------------------------
struct AwNow { float factor, lr, up1, up2; uint32_t key; };

// What a block of tensor t is loaded into.
template <int BITS>
struct AwRaw { float g[8], p[8], m[BITS == 8 ? 1 : 8], v[BITS == 8 ? 1 : 8], ms, vs; uint32_t cm[2], cv[2]; };

// FULL: 256 elements, every pointer aligned.
template <int BITS, bool FULL>
__device__ __forceinline__ void aw_fetch(const AwTensor& t, uint32_t b, int lane, AwRaw<BITS>& r) {
  const uint32_t mine = b - t.first;
  const long long base = (long long)mine * AW_BLOCK;
  const int left = FULL ? AW_BLOCK : (int)min((long long)AW_BLOCK, t.n - base);
  aw_load_g<FULL>(t, base, left, lane, r.g);
  aw_load_f32<FULL>(t.p, base, left, lane, r.p);
  if (BITS == 8 || (BITS == 0 && t.bits8)) {
    aw_load_codes<FULL>(t.m, base, left, lane, r.cm);
    aw_load_codes<FULL>(t.v, base, left, lane, r.cv);
    r.ms = t.m_scale[mine];
    r.vs = t.v_scale[mine];
  } else if constexpr (BITS != 8) {
    aw_load_f32<FULL>(static_cast<const float*>(t.m), base, left, lane, r.m);
    aw_load_f32<FULL>(static_cast<const float*>(t.v), base, left, lane, r.v);
  }
}

template <int BITS, bool FULL>
__device__ __forceinline__ void aw_update(const AwStep& s, const AwNow& now, const AwTensor& t, uint32_t b, int lane, const AwRaw<BITS>& r) {
  const uint32_t mine = b - t.first;
  const long long base = (long long)mine * AW_BLOCK;
  const int left = FULL ? AW_BLOCK : (int)min((long long)AW_BLOCK, t.n - base);
  const bool bits8 = BITS == 8 || (BITS == 0 && t.bits8);
  float p[8], m[8], v[8];
  const float (&g)[8] = r.g;
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = r.p[i];
  if (bits8) {
    aw_from_codes(r.cm, r.ms, m);
    aw_from_codes(r.cv, r.vs, v);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const unsigned long long r = aw_two(v[i], v[i + 1]);
      aw_split(aw_mul2(r, r), v[i], v[i + 1]);
    }
  } else if constexpr (BITS != 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { m[i] = r.m[i]; v[i] = r.v[i]; }
  }
  const float rate = now.lr * t.lr_mult;
  float root[8];
  const unsigned long long factor = aw_two(now.factor, now.factor), b1 = aw_two(s.b1, s.b1), b2 = aw_two(s.b2, s.b2), c1 = aw_two(s.c1, s.c1),
                           c2 = aw_two(s.c2, s.c2), up1 = aw_two(now.up1, now.up1), up2 = aw_two(now.up2, now.up2),
                           eps = aw_two(s.eps, s.eps), decay = aw_two(t.decay, t.decay), back = aw_two(-rate, -rate);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    // (packed products, single sums: a packed sum of packed products comes out as one operation of one rounding)
    const unsigned long long x = aw_mul2(aw_two(g[i], g[i + 1]), factor);
    float m0, m1, x0, x1, v0, v1, q0, q1;
    aw_split(aw_mul2(b1, aw_two(m[i], m[i + 1])), m0, m1);
    aw_split(aw_mul2(c1, x), x0, x1);
    aw_split(aw_mul2(b2, aw_two(v[i], v[i + 1])), v0, v1);
    aw_split(aw_mul2(c2, aw_mul2(x, x)), q0, q1);
    m[i] = __fadd_rn(m0, x0);
    m[i + 1] = __fadd_rn(m1, x1);
    v[i] = __fadd_rn(v0, q0);
    v[i + 1] = __fadd_rn(v1, q1);
    const unsigned long long mm = aw_two(m[i], m[i + 1]);
    // held in 8 bits, the root is a result itself; in 32 it only divides
    root[i] = bits8 ? __fsqrt_rn(v[i]) : aw_sqrt(v[i]);
    root[i + 1] = bits8 ? __fsqrt_rn(v[i + 1]) : aw_sqrt(v[i + 1]);
    float d0, d1;                              // 0 or at least 2^-75: no flush to zero
    aw_split(aw_fma2(aw_two(root[i], root[i + 1]), up2, eps), d0, d1);
    const unsigned long long pp = aw_two(p[i], p[i + 1]);
    const unsigned long long up = aw_mul2(aw_mul2(mm, up1), aw_two(aw_rcp(d0), aw_rcp(d1)));
    aw_split(aw_fma2(back, aw_fma2(decay, pp, up), pp), p[i], p[i + 1]);
  }
  aw_store_f32<FULL>(t.p, base, left, lane, p);
  if (t.copy) {
    if constexpr (FULL) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(p[4 * h], p[4 * h + 1]), c = __floats2bfloat162_rn(p[4 * h + 2], p[4 * h + 3]);
        *reinterpret_cast<uint2*>(t.copy + base + h * 128 + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&c));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (aw_elem(lane, i) < left) t.copy[base + aw_elem(lane, i)] = __float2bfloat16_rn(p[i]);
    }
  }
  if (bits8) {
    uint32_t rnd[8];
    const uint32_t e0 = (b * AW_BLOCK + 4 * lane) * 0x9E3779B1u + now.key;
#pragma unroll
    for (int i = 0; i < 8; ++i) rnd[i] = aw_mix(e0 + (uint32_t)((i >> 2) * 128 + (i & 3)) * 0x9E3779B1u);
    aw_store_codes<FULL, AW_LOW, true>(t.m, t.m_scale + mine, base, left, lane, m, rnd);
    aw_store_codes<FULL, AW_HIGH, false>(t.v, t.v_scale + mine, base, left, lane, root, rnd);
  } else {
    aw_store_f32<FULL>(static_cast<float*>(t.m), base, left, lane, m);
    aw_store_f32<FULL>(static_cast<float*>(t.v), base, left, lane, v);
  }
}

// Calls f(tensor, first block, blocks) for the blocks of this warp: runs of up to `run` neighbours of one tensor.
template <class F>
__device__ __forceinline__ void aw_each(const AwView& w, uint32_t blocks, uint32_t run, F&& f) {
  const uint32_t warps = gridDim.x * AW_WARPS, me = blockIdx.x * AW_WARPS + (threadIdx.x >> 5);
  int k = 0;
  for (unsigned long long b0 = (unsigned long long)me * run; b0 < blocks; b0 += (unsigned long long)warps * run) {
    uint32_t b = (uint32_t)b0;
    const uint32_t end = (uint32_t)min((unsigned long long)blocks, b0 + run);
    while (b < end) {
      k = aw_find(w, b, k);
      const AwTensor t = w.table[k];
      const uint32_t stop = min(end, __ldg(w.first + k + 1));
      f(t, b, stop - b);
      b = stop;
    }
  }
}
__device__ __forceinline__ bool aw_full(const AwTensor& t, uint32_t b) {
  return t.wide && (long long)(b - t.first + 1) * AW_BLOCK <= t.n;
}
// Neighbouring blocks per warp and turn: `most` where every warp has some turns of them, else fewer, so that all SMs have work.  (125 M
// elements.  States in 32 bits, runs of 1, 2, 4, 8: 609, 606, 607, 620 us.  In 8 bits, 4 and 8: 565 and 552, with 16 to a run of the norm;
// the norm's of 4, 16, 64: 595, 565, 572, single blocks throughout 750.  One turn or 16 in place of four: 565 and 576.)
__device__ __forceinline__ uint32_t aw_run(uint32_t blocks, uint32_t most) {
  return min(most, max(1u, blocks / (gridDim.x * AW_WARPS * 4)));
}

// BITS: of the states of all tensors; 0: they are mixed
template <int BITS>
__global__ void __launch_bounds__(AW_THREADS, 3) adamw_kernel(const __grid_constant__ AwStep s) {
  const int lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const AwView& w = s.w;
  const int taken = *reinterpret_cast<volatile const int*>(s.steps);
  AwNow now;
  now.factor = s.clipped ? *reinterpret_cast<volatile const float*>(&w.ctl->factor) : 1.0f;
  const uint32_t blocks = w.ctl->blocks;
  if (now.factor >= 0.f) {
    const double t = (double)taken + 1.0;
    // 1 - beta^t, without the cancellation that beta^t near 1 would bring
    now.up1 = __fdiv_rn(1.0f, -expm1f((float)(t * s.log_b1)));
    now.up2 = sqrtf(__fdiv_rn(1.0f, -expm1f((float)(t * s.log_b2))));
    now.lr = *s.lr;
    now.key = aw_mix(aw_mix(s.seed) + (uint32_t)(taken + 1));
    aw_each(w, blocks, aw_run(blocks, BITS == 8 ? 8 : 4), [&](const AwTensor& t, uint32_t b, uint32_t n) {
      uint32_t i = 0;
      if (BITS == 8) {                         // few bytes to a block: the loads of two on their way at once
        for (; i + 2 <= n && aw_full(t, b + i + 1); i += 2) {
          AwRaw<BITS> r0, r1;
          aw_fetch<BITS, true>(t, b + i, lane, r0);
          aw_fetch<BITS, true>(t, b + i + 1, lane, r1);
          aw_update<BITS, true>(s, now, t, b + i, lane, r0);
          aw_update<BITS, true>(s, now, t, b + i + 1, lane, r1);
        }
      }
      for (; i < n; ++i) {
        AwRaw<BITS> r;
        if (aw_full(t, b + i)) {
          aw_fetch<BITS, true>(t, b + i, lane, r);
          aw_update<BITS, true>(s, now, t, b + i, lane, r);
        } else {
          aw_fetch<BITS, false>(t, b + i, lane, r);
          aw_update<BITS, false>(s, now, t, b + i, lane, r);
        }
      }
    });
  }
  // every CTA has read the count when the last one comes here
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&w.ctl->step_ticket, 1u) + 1u == gridDim.x) {
      w.ctl->step_ticket = 0u;
      if (now.factor >= 0.f) *s.steps = taken + 1;
    }
  }
}

// ---- the norm: every CTA sums its blocks, the one that ends last the CTAs' sums, in order -----------------------------------------
__global__ void __launch_bounds__(AW_THREADS) adamw_norm_kernel(const __grid_constant__ AwStep s) {
  __shared__ double s_sum[AW_WARPS];
  __shared__ bool s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const AwView& w = s.w;
  const uint32_t blocks = w.ctl->blocks;
  double sum = 0.0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // the step waits for this grid's end before it reads anything
  double sums[4] = {0.0, 0.0, 0.0, 0.0};         // (chains of their own)
  auto add = [&](const float (&g)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[i & 3] = fma((double)g[i], (double)g[i], sums[i & 3]);
  };
  aw_each(w, blocks, aw_run(blocks, 16), [&](const AwTensor& t, uint32_t b, uint32_t n) {
    const long long base = (long long)(b - t.first) * AW_BLOCK;
    uint32_t i = 0;
    for (; i + 4 <= n && aw_full(t, b + i + 3); i += 4) {
      float g[4][8];
#pragma unroll
      for (int j = 0; j < 4; ++j) aw_load_g<true>(t, base + (i + j) * AW_BLOCK, AW_BLOCK, lane, g[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) add(g[j]);
    }
    for (; i < n; ++i) {
      float g[8];
      const long long at = base + i * AW_BLOCK;
      if (aw_full(t, b + i)) aw_load_g<true>(t, at, AW_BLOCK, lane, g);
      else aw_load_g<false>(t, at, (int)min((long long)AW_BLOCK, t.n - at), lane, g);
      add(g);
    }
  });
  sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  auto join = [&](double x) {                  // over the CTA; the result in thread 0
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (lane == 0) s_sum[warp] = x;
    __syncthreads();
    x = 0.0;
    if (threadIdx.x == 0)
      for (int i = 0; i < AW_WARPS; ++i) x += s_sum[i];
    return x;
  };
  sum = join(sum);
  if (threadIdx.x == 0) {
    w.parts[blockIdx.x] = sum;
    __threadfence();
    s_last = atomicAdd(&w.ctl->norm_ticket, 1u) + 1u == gridDim.x;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  sum = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += AW_THREADS) sum += *reinterpret_cast<volatile double*>(w.parts + i);
  sum = join(sum);
  if (threadIdx.x == 0) {
    const double root = sqrt(sum);
    const float norm = (float)root;
    w.ctl->norm_ticket = 0u;
    // a norm past fp32's range is not finite either
    w.ctl->factor = !(norm <= FLT_MAX) ? -1.0f : s.max_norm > 0.0 && root > s.max_norm ? (float)(s.max_norm / root) : 1.0f;
    if (s.norm) *s.norm = norm;
  }
}

bool ptr_ok(const void* p, size_t a) { return p && reinterpret_cast<uintptr_t>(p) % a == 0; }

int sm_count(int* sms) {
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  return QBLORA_OK;
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" {

size_t qblora_adamw_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 1 || n_tensors > AW_MAX_TENSORS) return 0;
  return align_up(aw_first_at(n_tensors) + (size_t)(n_tensors + 1) * 4, 256);
}

int qblora_adamw_prepare(const qblora_adamw_tensor* tensors, int32_t n_tensors, void* ws, size_t ws_bytes, int64_t* blocks,
                         void* stream) {
  if (!tensors || !blocks || n_tensors < 1) return QBLORA_ERR_INVALID_ARG;
  if (n_tensors > AW_MAX_TENSORS) return QBLORA_ERR_UNSUPPORTED;
  int64_t total = 0;
  int kinds = 0;                               // 1: some states in 32 bits, 2: some in 8
  for (int i = 0; i < n_tensors; ++i) {
    const qblora_adamw_tensor& t = tensors[i];
    if (t.n < 0 || (t.g_dtype != QBLORA_F32 && t.g_dtype != QBLORA_BF16) || (t.state_bits != 32 && t.state_bits != 8)) return QBLORA_ERR_INVALID_ARG;
    if (!std::isfinite(t.lr_mult) || !std::isfinite(t.weight_decay)) return QBLORA_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    const size_t sa = t.state_bits == 8 ? 1 : 4;
    if (!ptr_ok(t.p, 4) || !ptr_ok(t.g, t.g_dtype == QBLORA_F32 ? 4 : 2) || !ptr_ok(t.m, sa) || !ptr_ok(t.v, sa)) return QBLORA_ERR_INVALID_ARG;
    if (t.copy && !ptr_ok(t.copy, 2)) return QBLORA_ERR_INVALID_ARG;
    if (t.state_bits == 8 && (!ptr_ok(t.m_scale, 4) || !ptr_ok(t.v_scale, 4))) return QBLORA_ERR_INVALID_ARG;
    kinds |= t.state_bits == 8 ? 2 : 1;
    if (t.n > (int64_t)AW_BLOCK * 0x7fffffff) return QBLORA_ERR_UNSUPPORTED;
    total += (t.n + AW_BLOCK - 1) / AW_BLOCK;
    if (total > 0x7fffffff) return QBLORA_ERR_UNSUPPORTED;
  }
  if (!ws || !aligned16(ws) || ws_bytes < qblora_adamw_workspace_bytes(n_tensors)) return QBLORA_ERR_WORKSPACE;
  uint32_t first = 0;
  for (int at = 0; at < n_tensors; at += AW_TABLE_PART) {
    AwTablePart part{};
    const int count = n_tensors - at < AW_TABLE_PART ? n_tensors - at : AW_TABLE_PART;
    for (int i = 0; i < count; ++i) {
      const qblora_adamw_tensor& t = tensors[at + i];
      AwTensor& d = part.t[i];
      d.p = t.p; d.g = t.g; d.copy = static_cast<__nv_bfloat16*>(t.copy); d.m = t.m; d.v = t.v; d.m_scale = t.m_scale; d.v_scale = t.v_scale;
      d.n = t.n; d.first = first; d.g16 = t.g_dtype == QBLORA_BF16; d.bits8 = t.state_bits == 8;
      d.lr_mult = t.lr_mult; d.decay = t.weight_decay;
      const size_t sa = d.bits8 ? 4 : 16;
      d.wide = t.n > 0 && ptr_ok(t.p, 16) && ptr_ok(t.g, d.g16 ? 8 : 16) && ptr_ok(t.m, sa) && ptr_ok(t.v, sa) &&
               (!t.copy || ptr_ok(t.copy, 8));
      first += (uint32_t)((t.n + AW_BLOCK - 1) / AW_BLOCK);
    }
    adamw_table_kernel<<<1, AW_TABLE_PART, 0, static_cast<cudaStream_t>(stream)>>>(part, at, count, n_tensors, (uint32_t)total,
                                                                                   static_cast<char*>(ws), aw_first_at(n_tensors));
    count_launch();
    QB_CUDA(cudaGetLastError());
  }
  *blocks = total | (int64_t)kinds << 32;
  return QBLORA_OK;
}

int qblora_adamw_step(const qblora_adamw_cfg* cfg, int32_t n_tensors, int64_t blocks, void* ws, size_t ws_bytes, void* stream) {
  if (!cfg || n_tensors < 1 || n_tensors > AW_MAX_TENSORS || blocks < 0) return QBLORA_ERR_INVALID_ARG;
  const int kinds = (int)(blocks >> 32);       // as qblora_adamw_prepare has put them together
  blocks &= 0xffffffff;
  if (kinds > 3 || blocks > 0x7fffffff) return QBLORA_ERR_INVALID_ARG;
  if (!ptr_ok(cfg->lr, 4) || !ptr_ok(cfg->steps, 4) || (cfg->norm && !ptr_ok(cfg->norm, 4))) return QBLORA_ERR_INVALID_ARG;
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return QBLORA_ERR_INVALID_ARG;
  if (!(cfg->eps == 0.0 || (cfg->eps >= FLT_MIN && cfg->eps <= FLT_MAX)) || !(cfg->max_norm >= 0.0 && std::isfinite(cfg->max_norm)))
    return QBLORA_ERR_INVALID_ARG;
  if (!ws || !aligned16(ws) || ws_bytes < qblora_adamw_workspace_bytes(n_tensors)) return QBLORA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  AwStep s{};
  s.w = aw_view(ws, n_tensors);
  s.lr = cfg->lr; s.steps = cfg->steps; s.norm = cfg->norm;
  s.log_b1 = std::log(cfg->beta1); s.log_b2 = std::log(cfg->beta2);
  s.b1 = (float)cfg->beta1; s.b2 = (float)cfg->beta2; s.c1 = (float)(1.0 - cfg->beta1); s.c2 = (float)(1.0 - cfg->beta2);
  s.eps = (float)cfg->eps; s.max_norm = cfg->max_norm; s.seed = cfg->seed;
  s.clipped = cfg->max_norm > 0.0 || cfg->norm != nullptr;
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc) return rc;
  const int64_t want = (blocks + AW_WARPS - 1) / AW_WARPS;
  if (s.clipped) {
    int64_t grid = 4LL * sms < AW_NORM_CTAS ? 4LL * sms : AW_NORM_CTAS;
    if (grid > want) grid = want;
    if (grid < 1) grid = 1;
    adamw_norm_kernel<<<(unsigned)grid, AW_THREADS, 0, st>>>(s);
    count_launch();
    QB_CUDA(cudaGetLastError());
  }
  int64_t grid = 3LL * sms;
  if (grid > want) grid = want;
  if (grid < 1) grid = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)grid);
  lc.blockDim = dim3(AW_THREADS);
  lc.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = attr; lc.numAttrs = s.clipped ? 1 : 0;
  QB_CUDA(cudaLaunchKernelEx(&lc, kinds == 2 ? adamw_kernel<8> : kinds == 3 ? adamw_kernel<0> : adamw_kernel<32>, s));
  count_launch();
  return QBLORA_OK;
}

}  // extern "C"
