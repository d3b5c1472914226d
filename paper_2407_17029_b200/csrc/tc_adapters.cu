// Many adapters over one weight on the tensor cores (tcgen05): forward and backward of qblora_adapters_fwd / _bwd for rows of any
// number, fast sizes (tc_adapters_supported).
//
// The adapter's products are thin: their operands are small beside X, Y and dX, which pass once.  So three kinds of kernels, all
// over the rows in the plan's order, where every adapter's rows are neighbours:
//   pool    x' of every row (and the sums of dY's neighbours) as pairs of bf16 numbers, hi + lo: reads X at the memory's rate
//   shrink  u = x' A (and du = dv B^T): the pairs in, pairs out
//   spread  Y += s repeat(u B) (and dX += repeat(du A^T) / lambda): the memory-bound end
//   grad    dA = x'^T du, dB = u^T dv: sums over an adapter's rows
// In shrink and spread the weights are the 128 rows of the tensor core's tile and the tokens its columns, 16 to 128 of them as an
// adapter has rows: a lone decoding row costs a tile of 16, not of 128, and in the result a warp's lanes are neighbouring
// outputs, so that Y is read and written in whole lines straight from tensor memory.  Pairs: one bf16 number would put 2^-9 on
// everything that the adapter adds; hi and lo are two MMAs with the same weights, 2^-16 at worst.
//
// Rows in the workspace: adapter a's begin at a multiple of 16 (pad[a]) and are filled up to one with zeros, so that the sums over
// rows in grad run in whole steps of 16.  Which adapter has which tile is found by every CTA for itself from the plan's offsets.
//
// All loops are persistent: 148 CTAs take the (row tile, weight tile) units in turn; warp 0 loads by TMA, warp 1 issues the MMAs, eight
// warps empty one accumulator while the next is filled.
#include <algorithm>
#include <atomic>

#include "adapters.cuh"
#include "tc_ptx.cuh"
#include "tc_small.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int AG_THREADS = 320, AG_EPI = 256;       // TMA warp, MMA warp, eight epilogue warps
constexpr int AG_TN = 128;                          // most rows of a tile
constexpr int AG_PART = 16384;                      // bytes of one 128 x 64 operand tile
constexpr int AG_POOL_THREADS = 256;

// ---- adapters' rows: where they lie in the workspace, and their tiles ------------------------------------------------------------
struct AgGroups {
  const uint32_t* pad;      // [n + 1] first row of each adapter in the workspace, multiples of 16
  const uint32_t* tile;     // [n + 1] tiles in front of it
  int kept;                 // adapters whose rows lie in the workspace: all, for a plan whose offsets rise
};
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }   // both below 2^31

// by the whole CTA; s: 2 (n + 1) words of shared memory
template <int NT>
__device__ AgGroups ag_groups(const AdaptersCall& c, uint32_t* s, uint32_t rows_there) {
  __shared__ uint32_t s_part[2][NT / 32];
  __shared__ int s_kept;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = c.k.n;
  uint32_t *pad = s, *tile = s + n + 1;
  const int per = (n + NT - 1) / NT, lo = min(tid * per, n), hi = min(lo + per, n);
  uint32_t mine = 0, tiles = 0;
  for (int a = lo; a < hi; ++a) {
    const uint32_t rows = (uint32_t)max(plan_start(c, a + 1) - plan_start(c, a), 0);
    const uint32_t p = (min(rows, 0x7ffffff0u) + 15u) & ~15u, t = (rows + AG_TN - 1) / AG_TN;
    pad[a] = p;
    tile[a] = t;
    mine = sat_add(mine, p);
    tiles = sat_add(tiles, t);
  }
  uint32_t x = mine, y = tiles;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t px = __shfl_up_sync(0xffffffffu, x, d), py = __shfl_up_sync(0xffffffffu, y, d);
    if (lane >= d) { x = sat_add(x, px); y = sat_add(y, py); }
  }
  // exclusive within the warp (the saturated case only has to stay large)
  uint32_t ex = __shfl_up_sync(0xffffffffu, x, 1), ey = __shfl_up_sync(0xffffffffu, y, 1);
  if (lane == 0) ex = ey = 0;
  if (lane == 31) { s_part[0][warp] = x; s_part[1][warp] = y; }
  if (tid == 0) s_kept = n;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 32; ++w)
    if (w < warp) { ex = sat_add(ex, s_part[0][w]); ey = sat_add(ey, s_part[1][w]); }
  for (int a = lo; a < hi; ++a) {
    const uint32_t p = pad[a], t = tile[a];
    pad[a] = ex;
    tile[a] = ey;
    ex = sat_add(ex, p);
    ey = sat_add(ey, t);
    if (ex > rows_there) atomicMin(&s_kept, a);
  }
  if (lo < hi && hi == n) { pad[n] = ex; tile[n] = ey; }
  __syncthreads();
  return {pad, tile, s_kept};
}
// the last a in [0, n) with v[a] <= x; v[0] <= x < v[n]
__device__ __forceinline__ int ag_find(const uint32_t* v, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// ---- pool ---------------------------------------------------------------------------------------------------------------------
struct AgPool {
  RowsView x;
  int d, lam, small, ld, wide;          // elements of a row, of its pooled form and its pitch; wide: 16-byte loads, lam a power of two
  float factor;                         // 1 / lam or 1
  __nv_bfloat16 *hi, *lo;               // lo == nullptr: the pooled values are bf16 numbers already (lam 1)
};
struct AgPoolParams { AdaptersCall c; AgPool src[2]; int sources; uint32_t rows_there; int* status; };

__device__ __forceinline__ void ag_pair(float x, __nv_bfloat16& hi, __nv_bfloat16& lo) {
  hi = __float2bfloat16_rn(x);
  lo = __float2bfloat16_rn(x - __bfloat162float(hi));
}
__device__ __forceinline__ float ag_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float ag_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// One row by one warp.  x: nullptr for a row of zeros.
__device__ void ag_pool_row(const AgPool& p, const __nv_bfloat16* x, int64_t out, int lane) {
  __nv_bfloat16 *hi = p.hi + out * p.ld, *lo = p.lo ? p.lo + out * p.ld : nullptr;
  if (!x) {
    for (int i = lane; i < p.small; i += 32) {
      hi[i] = __float2bfloat16_rn(0.f);
      if (lo) lo[i] = __float2bfloat16_rn(0.f);
    }
    return;
  }
  if (!p.wide) {
    for (int i = lane; i < p.small; i += 32) {
      float acc = 0.f;
      for (int l = 0; l < p.lam; ++l) acc += __bfloat162float(x[(int64_t)i * p.lam + l]);
      __nv_bfloat16 h, l;
      ag_pair(p.factor == 1.f ? acc : acc / (float)p.lam, h, l);
      hi[i] = h;
      if (lo) lo[i] = l;
    }
    return;
  }
  const int chunks = p.d >> 3;
  constexpr int U = 4;                                  // 16-byte loads in flight per lane
  for (int c0 = 0; c0 < chunks; c0 += 32 * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ch = c0 + u * 32 + lane;
      w[u] = ch < chunks ? *reinterpret_cast<const uint4*>(x + 8 * (int64_t)ch) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ch = c0 + u * 32 + lane;
      const uint32_t e[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
      if (p.lam == 1) {
        if (ch < chunks) *reinterpret_cast<uint4*>(hi + 8 * (int64_t)ch) = w[u];
        continue;
      }
      float s[4];                                       // sums of neighbouring two
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = ag_low(e[i]) + ag_high(e[i]);
      if (p.lam == 2) {
        if (ch < chunks) {
          __nv_bfloat16 h[4], l[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) ag_pair(s[i] * p.factor, h[i], l[i]);
          *reinterpret_cast<uint2*>(hi + 4 * (int64_t)ch) = *reinterpret_cast<const uint2*>(h);
          *reinterpret_cast<uint2*>(lo + 4 * (int64_t)ch) = *reinterpret_cast<const uint2*>(l);
        }
        continue;
      }
      const float f0 = s[0] + s[1], f1 = s[2] + s[3];
      if (p.lam == 4) {
        if (ch < chunks) {
          __nv_bfloat16 h[2], l[2];
          ag_pair(f0 * p.factor, h[0], l[0]);
          ag_pair(f1 * p.factor, h[1], l[1]);
          *reinterpret_cast<uint32_t*>(hi + 2 * (int64_t)ch) = *reinterpret_cast<const uint32_t*>(h);
          *reinterpret_cast<uint32_t*>(lo + 2 * (int64_t)ch) = *reinterpret_cast<const uint32_t*>(l);
        }
        continue;
      }
      float g = f0 + f1;                                // of eight; lam / 8 lanes have the rest
      const int lanes = p.lam >> 3;
      for (int d = 1; d < lanes; d <<= 1) g += __shfl_xor_sync(0xffffffffu, g, d);
      if (ch < chunks && (ch & (lanes - 1)) == 0) {
        __nv_bfloat16 h, l;
        ag_pair(g * p.factor, h, l);
        hi[ch / lanes] = h;
        lo[ch / lanes] = l;
      }
    }
  }
}

__global__ void __launch_bounds__(AG_POOL_THREADS) adapters_pool_kernel(const __grid_constant__ AgPoolParams p) {
  extern __shared__ uint32_t ag_smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = QBLORA_OK;
  const AgGroups g = ag_groups<AG_POOL_THREADS>(p.c, ag_smem, p.rows_there);
  const int lane = threadIdx.x & 31, warps = AG_POOL_THREADS / 32;
  const uint32_t rows = g.pad[g.kept];
  for (int64_t i = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); i < (int64_t)rows * p.sources; i += (int64_t)gridDim.x * warps) {
    const int which = i >= rows ? 1 : 0;
    const uint32_t at = (uint32_t)(which ? i - rows : i);
    const int a = ag_find(g.pad, g.kept, at), j = plan_start(p.c, a) + (int)(at - g.pad[a]);
    int row = -1;
    if (j < plan_start(p.c, a + 1)) row = __ldg(p.c.rows + j);
    const AgPool& s = p.src[which];
    const bool real = row >= 0 && row < p.c.T;
    ag_pool_row(s, real ? static_cast<const __nv_bfloat16*>(s.x.data) + row * s.x.stride : nullptr, at, lane);
  }
}

// ---- shrink, spread, grad --------------------------------------------------------------------------------------------------------
enum { AG_SHRINK = 0, AG_SPREAD = 1, AG_GRAD = 2 };

struct AgMaps {
  CUtensorMap w;                        // shrink, spread: the bank's matrix, three dimensions
  CUtensorMap hi, lo, hi16, lo16;       // their rows: boxes of 128 and of 16.  grad: x' and du
  CUtensorMap hi2, lo2, u_hi, u_lo;     // grad: (hi, lo) x', (hi2, lo2) du, (u_hi, u_lo) u, (hi16, lo16) dv; boxes 64 x 64
};
struct AgParams {
  AdaptersCall c;
  uint32_t rows_there;
  int m_tiles, M;                       // shrink: of the rank; spread: of Q or P
  int K;                                // shrink: P or Q
  int w_kmajor;                         // the weight's contiguous dimension is the contraction's
  int lo_on, lo2_on;                    // x' (dv) has a lo part
  int scaled;                           // times the adapter's factor
  __nv_bfloat16 *hi, *lo; int ld;       // shrink: out
  RowsView y; int lam; float factor;    // spread
  float *dA, *dB;                       // grad
  int* status;
  long long wait_limit;
};

// One unit of work: a tile of 128 weights' rows by the rows of one adapter's tile; grad: 128 by 128 of dA or dB.
struct AgUnit {
  int a, m0, n0;                        // adapter, first row and (grad) column of the result
  uint32_t at;                          // first row in the workspace
  int j, rows, n16;                     // first entry in the plan, rows, rows or columns in whole steps
  int steps;                            // of 16 along the contraction; 0: nothing to contract
  int which;                            // grad: 0 dA, 1 dB
  int rank;
};

template <int KIND>
struct AgWork {
  const AgParams& p;
  const AgGroups& g;
  int ta, tb, na, nb;                   // grad: tiles of dA (ta x na) and dB (tb x nb)
  long long units;
  __device__ AgWork(const AgParams& p_, const AgGroups& g_) : p(p_), g(g_) {
    if (KIND == AG_GRAD) {
      const BankView& k = p.c.k;
      na = p.dA ? (k.r + 127) / 128 : 0;
      ta = (k.P + 127) / 128;
      tb = p.dB ? (k.r + 127) / 128 : 0;
      nb = (k.Q + 127) / 128;
      units = (long long)k.n * (ta * na + tb * nb);
    } else {
      units = (long long)g.tile[g.kept] * p.m_tiles;
    }
  }
  __device__ __forceinline__ void get(long long u, AgUnit& t) const {
    const BankView& k = p.c.k;
    if (KIND == AG_GRAD) {
      const int per = ta * na + tb * nb;
      t.a = (int)(u / per);
      int x = (int)(u - (long long)t.a * per);
      t.which = x >= ta * na;
      if (t.which) x -= ta * na;
      const int cols = t.which ? nb : na;
      t.m0 = x / cols * 128;
      t.n0 = x % cols * 128;
      t.rank = bank_rank(k, t.a);
      t.n16 = min(128, ((t.which ? k.Q : k.r) - t.n0 + 15) & ~15);
      t.at = t.a < g.kept ? g.pad[t.a] : 0;
      t.rows = t.a < g.kept ? (int)(g.pad[t.a + 1] - g.pad[t.a]) : 0;
      t.steps = (t.which ? t.m0 : t.n0) < t.rank ? t.rows / 16 : 0;
      t.j = 0;
    } else {
      const uint32_t tile = (uint32_t)(u / p.m_tiles);
      t.a = ag_find(g.tile, g.kept, tile);
      const int i = (int)(tile - g.tile[t.a]) * AG_TN, s0 = plan_start(p.c, t.a);
      t.at = g.pad[t.a] + i;
      t.j = s0 + i;
      t.rows = min(AG_TN, plan_start(p.c, t.a + 1) - t.j);
      t.n16 = (t.rows + 15) & ~15;
      t.m0 = (int)(u - (long long)tile * p.m_tiles) * 128;
      t.n0 = 0;
      t.which = 0;
      t.rank = bank_rank(k, t.a);
      t.steps = KIND == AG_SHRINK ? (t.m0 < t.rank ? (p.K + 15) / 16 : 0) : (t.rank + 15) / 16;
    }
  }
};

template <int KIND> struct AgShape {
  static constexpr int A_PARTS = KIND == AG_GRAD ? 2 : 1;          // 128 x 64: weights, or the pair of x' or u
  static constexpr int STAGE = (A_PARTS + 2) * AG_PART;            // and a pair of 64 x up to 128
  static constexpr int STAGES = KIND == AG_GRAD ? 3 : 4;
  static constexpr int COLS = KIND == AG_GRAD ? 256 : 128;         // tensor memory of one accumulator
};
template <int KIND> size_t ag_smem_bytes(int n) {
  return (size_t)AgShape<KIND>::STAGES * AgShape<KIND>::STAGE + 1024 + 256 + (size_t)2 * (n + 1) * 4;
}

// y[0 .. W bytes) += x at element type F32 or bf16, W = 2, 4, 8, 16
template <int W, bool F32> struct AgVec;
template <> struct AgVec<2, false> { using T = uint16_t; };
template <> struct AgVec<4, false> { using T = uint32_t; };
template <> struct AgVec<8, false> { using T = uint2; };
template <> struct AgVec<16, false> { using T = uint4; };
template <> struct AgVec<4, true> { using T = float; };
template <> struct AgVec<8, true> { using T = float2; };
template <> struct AgVec<16, true> { using T = float4; };
template <class T, bool F32>
__device__ __forceinline__ T ag_add(T y, float x) {
  if constexpr (F32) {
    float* e = reinterpret_cast<float*>(&y);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) e[i] += x;
  } else if constexpr (sizeof(T) == 2) {
    const __nv_bfloat16 b = __float2bfloat16_rn(__uint_as_float((uint32_t)y << 16) + x);
    y = *reinterpret_cast<const uint16_t*>(&b);
  } else {
    uint32_t* e = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) e[i] = pack_bf16x2(ag_low(e[i]) + x, ag_high(e[i]) + x);
  }
  return y;
}

// 32 columns (rows of Y, numbers in `row` of lane j, -1: none) of 32 weights' rows from m on, one per lane, in v.
template <int W, bool F32>
__device__ __forceinline__ void ag_spread_narrow(const AgParams& p, const float (&v)[32], int row, int m, bool there) {
  using V = typename AgVec<W, F32>::T;
  char* base = static_cast<char*>(p.y.data) + (int64_t)m * W;
  const int64_t pitch = p.y.stride * (F32 ? 4 : 2);
#pragma unroll
  for (int j0 = 0; j0 < 32; j0 += 8) {
    V y[8];
    int r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      r[j] = __shfl_sync(0xffffffffu, row, j0 + j);
      if (!there) r[j] = -1;
      if (r[j] >= 0) y[j] = *reinterpret_cast<const V*>(base + r[j] * pitch);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (r[j] >= 0) *reinterpret_cast<V*>(base + r[j] * pitch) = ag_add<V, F32>(y[j], v[j0 + j]);
  }
}
// lam elements of 16 * per bytes: chunk i of 16 bytes of the 32 weights' rows belongs to row i / per
template <bool F32>
__device__ __forceinline__ void ag_spread_wide(const AgParams& p, const float (&v)[32], int row, int m_first, int per, int M, int lane) {
  using V = typename AgVec<16, F32>::T;
  char* base = static_cast<char*>(p.y.data) + (int64_t)m_first * per * 16;
  const int64_t pitch = p.y.stride * (F32 ? 4 : 2);
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const int r = __shfl_sync(0xffffffffu, row, j);
    if (r < 0) continue;
    char* out = base + r * pitch;
#pragma unroll 1
    for (int i0 = 0; i0 < per; i0 += 4) {
      V y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = (i0 + i) * 32 + lane;
        if (i0 + i < per && m_first + ch / per < M) y[i] = *reinterpret_cast<const V*>(out + (int64_t)ch * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = (i0 + i) * 32 + lane;
        const float x = __shfl_sync(0xffffffffu, v[j], min(ch / per, 31));
        if (i0 + i < per && m_first + ch / per < M) *reinterpret_cast<V*>(out + (int64_t)ch * 16) = ag_add<V, F32>(y[i], x);
      }
    }
  }
}
// any lam
__device__ __forceinline__ void ag_spread_any(const AgParams& p, const float (&v)[32], int row, int m, bool there) {
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const int r = __shfl_sync(0xffffffffu, row, j);
    if (r < 0 || !there) continue;
    const int64_t at = r * p.y.stride + (int64_t)m * p.lam;
    for (int l = 0; l < p.lam; ++l) {
      if (p.y.dtype == QBLORA_F32) static_cast<float*>(p.y.data)[at + l] += v[j];
      else {
        __nv_bfloat16* y = static_cast<__nv_bfloat16*>(p.y.data) + at + l;
        *y = __float2bfloat16_rn(__bfloat162float(*y) + v[j]);
      }
    }
  }
}
template <bool F32>
__device__ __forceinline__ void ag_spread(const AgParams& p, const float (&v)[32], int row, int m_first, int M, int lane) {
  const int w = p.lam * (F32 ? 4 : 2);
  const bool there = m_first + lane < M;
  if (w == 16) ag_spread_narrow<16, F32>(p, v, row, m_first + lane, there);
  else if (w == 8) ag_spread_narrow<8, F32>(p, v, row, m_first + lane, there);
  else if (w == 4) ag_spread_narrow<4, F32>(p, v, row, m_first + lane, there);
  else if (!F32 && w == 2) ag_spread_narrow<F32 ? 4 : 2, F32>(p, v, row, m_first + lane, there);
  else if (w % 16 == 0) ag_spread_wide<F32>(p, v, row, m_first, w / 16, M, lane);
  else ag_spread_any(p, v, row, m_first + lane, there);
}

template <int KIND>
__global__ void __launch_bounds__(AG_THREADS, 1) adapters_gemm_kernel(const __grid_constant__ AgMaps maps, const __grid_constant__ AgParams p) {
  using Sh = AgShape<KIND>;
  constexpr int STAGES = Sh::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t bars = base + STAGES * Sh::STAGE;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (STAGES + s); };
  auto accfull = [&](int b) { return bars + 8u * (2 * STAGES + b); };
  auto accempty = [&](int b) { return bars + 8u * (2 * STAGES + 2 + b); };
  const uint32_t tmem_slot = bars + 8u * (2 * STAGES + 4);
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
  uint32_t* table = reinterpret_cast<uint32_t*>(smem_raw + (bars + 256 - raw));

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accfull(b), 1); mbar_init(accempty(b), AG_EPI); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(2 * Sh::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const AgGroups groups = ag_groups<AG_THREADS>(p.c, table, p.rows_there);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot_g;
  const AgWork<KIND> work(p, groups);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // what the kernels in front have written

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0, ph = 0;
      int s = 0;
      bool ok = true;
      for (long long u = blockIdx.x; u < work.units && ok; u += gridDim.x) {
        AgUnit t;
        work.get(u, t);
        for (int k = 0; k < t.steps; k += 4, ++it) {
          if (!mbar_wait(empty(s), ph ^ 1u, p.status, p.wait_limit)) { ok = false; break; }
          const uint32_t a = base + s * Sh::STAGE, b = a + Sh::A_PARTS * AG_PART;
          const int k0 = k * 16;
          if (KIND == AG_GRAD) {
            const CUtensorMap *ah = t.which ? &maps.u_hi : &maps.hi, *al = t.which ? &maps.u_lo : &maps.lo;
            const CUtensorMap *bh = t.which ? &maps.hi16 : &maps.hi2, *bl = t.which ? &maps.lo16 : &maps.lo2;
            const bool a_lo = t.which ? true : p.lo_on, b_lo = t.which ? p.lo2_on : true;
            const int nb = (t.n16 + 63) / 64, y0 = (int)t.at + k0;
            mbar_arrive_expect_tx(full(s), (uint32_t)(8192 * (2 * (1 + a_lo) + nb * (1 + b_lo))));
            for (int i = 0; i < 2; ++i) {
              tma_load_2d(a + i * 8192, ah, full(s), t.m0 + i * 64, y0);
              if (a_lo) tma_load_2d(a + AG_PART + i * 8192, al, full(s), t.m0 + i * 64, y0);
            }
            for (int i = 0; i < nb; ++i) {
              tma_load_2d(b + i * 8192, bh, full(s), t.n0 + i * 64, y0);
              if (b_lo) tma_load_2d(b + AG_PART + i * 8192, bl, full(s), t.n0 + i * 64, y0);
            }
          } else {
            const bool lo = KIND == AG_SPREAD || p.lo_on;
            mbar_arrive_expect_tx(full(s), (uint32_t)(AG_PART + t.n16 * 128 * (1 + lo)));
            if (p.w_kmajor) {
              tma_load_3d(a, &maps.w, full(s), k0, t.m0, t.a);
            } else {
              tma_load_3d(a, &maps.w, full(s), t.m0, k0, t.a);
              tma_load_3d(a + 8192, &maps.w, full(s), t.m0 + 64, k0, t.a);
            }
            if (t.n16 == AG_TN) {
              tma_load_2d(b, &maps.hi, full(s), k0, (int)t.at);
              if (lo) tma_load_2d(b + AG_PART, &maps.lo, full(s), k0, (int)t.at);
            } else {
              for (int i = 0; i < t.n16; i += 16) {
                tma_load_2d(b + i * 128, &maps.hi16, full(s), k0, (int)t.at + i);
                if (lo) tma_load_2d(b + AG_PART + i * 128, &maps.lo16, full(s), k0, (int)t.at + i);
              }
            }
          }
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
        const uint32_t lo = it > (uint32_t)STAGES ? it - STAGES : 0;
        for (uint32_t j = lo; j < it; ++j) mbar_wait(full(j % STAGES), (j / STAGES) & 1u, p.status, p.wait_limit);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t ph = 0, done = 0;
      int s = 0;
      bool ok = true;
      const bool w_kmajor = KIND != AG_GRAD && p.w_kmajor;
      for (long long u = blockIdx.x; u < work.units && ok; u += gridDim.x) {
        AgUnit t;
        work.get(u, t);
        if (t.steps == 0) continue;
        const int b = done & 1;
        if (!mbar_wait(accempty(b), ((done >> 1) & 1u) ^ 1u, p.status, p.wait_limit)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem_base + b * Sh::COLS;
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((w_kmajor ? 0u : 1u) << 15) | ((KIND == AG_GRAD ? 1u : 0u) << 16) |
                               ((uint32_t)(t.n16 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        const bool a_lo = KIND == AG_GRAD && (t.which || p.lo_on);
        const bool b_lo = KIND == AG_GRAD ? !t.which || p.lo2_on : KIND == AG_SPREAD || p.lo_on;
        for (int k = 0; k < t.steps; k += 4) {
          if (!mbar_wait(full(s), ph, p.status, p.wait_limit)) { ok = false; break; }
          tc_fence_after();
          const uint32_t pa = base + s * Sh::STAGE, pb = pa + Sh::A_PARTS * AG_PART;
          const int n = min(4, t.steps - k);
          for (int e = 0; e < n; ++e) {
            const uint32_t acc = k + e > 0 ? 1u : 0u;
            const uint64_t ad = w_kmajor ? smem_desc(pa + e * 32, 16, 1024) : smem_desc(pa + e * 2048, 8192, 1024);
            const uint64_t bd = KIND == AG_GRAD ? smem_desc(pb + e * 2048, 8192, 1024) : smem_desc(pb + e * 32, 16, 1024);
            constexpr uint64_t next = AG_PART >> 4;                   // a pair's lo part, in descriptor units
            tc_mma(d, ad, bd, idesc, acc);
            if (KIND == AG_GRAD) {
              // the small products apart, so that the sum of the large ones is rounded no more often than it must
              if (b_lo) tc_mma(d + 128, ad, bd + next, idesc, acc);
              if (a_lo) tc_mma(d + 128, ad + next, bd, idesc, b_lo ? 1u : acc);
            } else if (b_lo) {
              tc_mma(d, ad, bd + next, idesc, 1u);
            }
          }
          tc_commit(empty(s));
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
        if (ok) tc_commit(accfull(b));
        ++done;
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;        // quarter of tensor memory's lanes; half of the columns
    uint32_t done = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < work.units && ok; u += gridDim.x) {
      AgUnit t;
      work.get(u, t);
      if (t.steps == 0 && KIND != AG_GRAD) continue;
      const int b = done & 1;
      if (t.steps > 0) {
        ok = mbar_wait(accfull(b), (done >> 1) & 1u, p.status, p.wait_limit);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
      }
      const uint32_t d = tmem_base + ((uint32_t)(q * 32) << 16) + b * Sh::COLS;
      const int m_first = t.m0 + q * 32, m = m_first + lane;
      const float scale = p.scaled && t.rows > 0 ? __ldg(p.c.k.s + t.a) : 1.0f;
#pragma unroll 1
      for (int c = half * 64; c < min(half * 64 + 64, t.n16); c += 32) {
        uint32_t w[32];
        float v[32];
        if (t.steps > 0) {
          tc_ld32(d + c, w);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(w[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0.f;
        }
        if (KIND == AG_GRAD) {
          if (t.steps > 0) {
            tc_ld32(d + 128 + c, w);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += __uint_as_float(w[j]);
          }
          const BankView& k = p.c.k;
          const int M = t.which ? k.r : k.P, N = t.which ? k.Q : k.r;
          if (m < M) {
            const float f = t.which ? scale : 1.0f;
            float* out = (t.which ? p.dB : p.dA) + ((int64_t)t.a * M + m) * N + t.n0 + c;
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              if (t.n0 + c + j >= N) break;                // N is a multiple of 8
              float x[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = (t.which ? m : t.n0 + c + j + e) < t.rank ? v[j + e] * f : 0.f;
              *reinterpret_cast<float4*>(out + j) = make_float4(x[0], x[1], x[2], x[3]);
            }
          }
        } else if (KIND == AG_SHRINK) {
          // lanes 2 i and 2 i + 1 swap, so that each has two neighbouring ranks of every other row
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float send = (lane & 1) ? v[j] : v[j + 1], keep = ((lane & 1) ? v[j + 1] : v[j]) * scale;
            const float got = __shfl_xor_sync(0xffffffffu, send, 1) * scale;
            const float x0 = (lane & 1) ? got : keep, x1 = (lane & 1) ? keep : got;
            const int col = c + j + (lane & 1), mm = m & ~1;
            if (col >= t.n16 || mm >= p.M) continue;       // M (the rank) is a multiple of 8
            const uint32_t h = pack_bf16x2(x0, x1);
            const int64_t o = (int64_t)(t.at + col) * p.ld + mm;
            *reinterpret_cast<uint32_t*>(p.hi + o) = h;
            *reinterpret_cast<uint32_t*>(p.lo + o) = pack_bf16x2(x0 - ag_low(h), x1 - ag_high(h));
          }
        } else {
          int row = -1;
          if (c + lane < t.rows) row = __ldg(p.c.rows + t.j + c + lane);
          if (row >= p.c.T) row = -1;
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] *= scale * p.factor;
          if (p.y.dtype == QBLORA_F32) ag_spread<true>(p, v, row, m_first, p.M, lane);
          else ag_spread<false>(p, v, row, m_first, p.M, lane);
        }
      }
      if (t.steps > 0) {
        tc_fence_before();
        mbar_arrive(accempty(b));
        ++done;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * Sh::COLS) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------------------
// A pair of bf16 matrices in the workspace.
struct Pair { __nv_bfloat16 *hi, *lo; int width, ld; };
struct Layout { Pair x, dv, u, du; size_t bytes; uint32_t rows; };

int pitch8(int n) { return (n + 7) & ~7; }

Layout ag_layout(const BankView& k, int64_t T, bool backward, char* ws) {
  Layout l{};
  l.rows = (uint32_t)std::min<int64_t>(T + 15 * std::min<int64_t>(T, k.n), 0x7ffffff0);
  size_t at = kStatusBytes;
  auto pair = [&](Pair& p, int width, bool lo) {
    p.width = width;
    p.ld = pitch8(width);
    const size_t bytes = align_up((size_t)l.rows * p.ld * 2, 256);
    p.hi = reinterpret_cast<__nv_bfloat16*>(ws + at);
    at += bytes;
    p.lo = lo ? reinterpret_cast<__nv_bfloat16*>(ws + at) : nullptr;
    if (lo) at += bytes;
  };
  pair(l.x, k.P, k.l1 > 1);
  pair(l.u, k.r, true);
  if (backward) {
    pair(l.dv, k.Q, k.l2 > 1);
    pair(l.du, k.r, true);
  }
  l.bytes = align_up(at, 256);
  return l;
}

AgPool ag_source(const RowsView& x, int d, int lam, bool mean, const Pair& out) {
  AgPool p{x, d, lam, out.width, out.ld, 0, mean ? 1.0f / (float)lam : 1.0f, out.hi, out.lo};
  p.wide = lam <= 256 && (lam & (lam - 1)) == 0;
  return p;
}

int ag_sms(int* n) {
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
  return QBLORA_OK;
}

template <int KIND>
int ag_launch(const AgMaps& maps, const AgParams& p, int64_t most_units, cudaStream_t st) {
  int sms = 0, rc = ag_sms(&sms);
  if (rc) return rc;
  auto kernel = adapters_gemm_kernel<KIND>;
  static std::atomic<bool> done[64];
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  if (!done[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ag_smem_bytes<KIND>(kMaxAdapters)));
    done[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(sms, most_units)));
  cfg.blockDim = dim3(AG_THREADS);
  cfg.dynamicSmemBytes = ag_smem_bytes<KIND>(p.c.k.n);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, kernel, maps, p));
  count_launch();
  return QBLORA_OK;
}

int ag_launch_pool(const AgPoolParams& p, int64_t rows, cudaStream_t st) {
  int sms = 0;
  const int rc = ag_sms(&sms);
  if (rc) return rc;
  const int64_t want = (rows * p.sources + AG_POOL_THREADS / 32 - 1) / (AG_POOL_THREADS / 32);
  adapters_pool_kernel<<<(unsigned)std::min<int64_t>(want, 8LL * sms), AG_POOL_THREADS, (size_t)2 * (p.c.k.n + 1) * 4, st>>>(p);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

int rows_map(CUtensorMap* tm, const __nv_bfloat16* ptr, const Pair& p, uint32_t rows, int box_rows) {
  return make_tensor_map_2d(tm, false, ptr, (uint64_t)p.width, rows, (uint64_t)p.ld * 2, 64, (uint32_t)box_rows, true);
}
// element (i, j) of slot a at a * rows * width + i * width + j: boxes of 64 j by `box` i
int bank_map(CUtensorMap* tm, const __nv_bfloat16* ptr, int width, int rows, int n, int box) {
  const uint64_t dims[3] = {(uint64_t)width, (uint64_t)rows, (uint64_t)n};
  const uint64_t pitch[2] = {(uint64_t)width * 2, (uint64_t)width * rows * 2};
  const uint32_t b[3] = {64, (uint32_t)box, 1};
  return make_tensor_map_nd(tm, 3, ptr, dims, pitch, b);
}

#define QB_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

int pair_maps(AgMaps* m, const Pair& p, uint32_t rows) {
  const __nv_bfloat16* lo = p.lo ? p.lo : p.hi;
  QB_TRY(rows_map(&m->hi, p.hi, p, rows, 128));
  QB_TRY(rows_map(&m->lo, lo, p, rows, 128));
  QB_TRY(rows_map(&m->hi16, p.hi, p, rows, 16));
  return rows_map(&m->lo16, lo, p, rows, 16);
}

AgParams ag_params(const AdaptersCall& c, const Layout& l, int* status) {
  AgParams p{};
  p.c = c;
  p.rows_there = l.rows;
  p.status = status;
  p.wait_limit = wait_limit_cycles();
  p.lam = 1;
  p.factor = 1.0f;
  return p;
}

int64_t most_tiles(const AdaptersCall& c) { return c.T / AG_TN + std::min<int64_t>(c.T, c.k.n); }

// u = x' A, or du = s dv B^T
int ag_shrink(const AdaptersCall& c, const Layout& l, int* status, const Pair& in, const Pair& out, const __nv_bfloat16* W, bool kmajor,
              bool scaled, cudaStream_t st) {
  AgMaps maps{};
  AgParams p = ag_params(c, l, status);
  QB_TRY(pair_maps(&maps, in, l.rows));
  // A [P][r]: the contraction runs over its rows; B [r][Q]: along them
  QB_TRY(kmajor ? bank_map(&maps.w, W, in.width, c.k.r, c.k.n, 128) : bank_map(&maps.w, W, c.k.r, in.width, c.k.n, 64));
  p.m_tiles = (c.k.r + 127) / 128; p.M = c.k.r; p.K = in.width;
  p.w_kmajor = kmajor; p.lo_on = in.lo != nullptr; p.scaled = scaled;
  p.hi = out.hi; p.lo = out.lo; p.ld = out.ld;
  return ag_launch<AG_SHRINK>(maps, p, most_tiles(c) * p.m_tiles, st);
}
// Y += s repeat(u B), or dX += repeat(du A^T) / lam
int ag_expand(const AdaptersCall& c, const Layout& l, int* status, const Pair& in, const __nv_bfloat16* W, int M, bool kmajor, const RowsView& y,
              int lam, bool forward, cudaStream_t st) {
  AgMaps maps{};
  AgParams p = ag_params(c, l, status);
  QB_TRY(pair_maps(&maps, in, l.rows));
  QB_TRY(kmajor ? bank_map(&maps.w, W, c.k.r, M, c.k.n, 128) : bank_map(&maps.w, W, M, c.k.r, c.k.n, 64));
  p.m_tiles = (M + 127) / 128; p.M = M;
  p.w_kmajor = kmajor; p.scaled = forward;
  p.y = y; p.lam = lam; p.factor = forward ? 1.0f : 1.0f / (float)lam;
  return ag_launch<AG_SPREAD>(maps, p, most_tiles(c) * p.m_tiles, st);
}
int ag_grad(const AdaptersCall& c, const Layout& l, int* status, cudaStream_t st) {
  AgMaps maps{};
  AgParams p = ag_params(c, l, status);
  auto both = [&](CUtensorMap* hi, CUtensorMap* lo, const Pair& q) -> int {
    QB_TRY(rows_map(hi, q.hi, q, l.rows, 64));
    return rows_map(lo, q.lo ? q.lo : q.hi, q, l.rows, 64);
  };
  QB_TRY(both(&maps.hi, &maps.lo, l.x));
  QB_TRY(both(&maps.hi2, &maps.lo2, l.du));
  QB_TRY(both(&maps.u_hi, &maps.u_lo, l.u));
  QB_TRY(both(&maps.hi16, &maps.lo16, l.dv));
  p.lo_on = l.x.lo != nullptr; p.lo2_on = l.dv.lo != nullptr; p.scaled = 1;
  p.dA = c.dA; p.dB = c.dB;
  const int64_t per = (int64_t)((c.k.P + 127) / 128 + (c.k.Q + 127) / 128) * ((c.k.r + 127) / 128);
  return ag_launch<AG_GRAD>(maps, p, per * c.k.n, st);
}

}  // namespace

size_t tc_adapters_ws_bytes(const BankView& k, int64_t T, bool backward) { return ag_layout(k, T, backward, nullptr).bytes; }

bool tc_adapters_sizes_ok(const BankView& k, int64_t T) {
  return k.r % 8 == 0 && k.Q % 8 == 0 && k.d_in % 8 == 0 && k.d_out % 8 == 0 && T + 15 * std::min<int64_t>(T, k.n) <= 0x7ffffff0;
}

bool tc_adapters_supported(const AdaptersCall& c) {
  if (!tc_adapters_sizes_ok(c.k, c.T) || !aligned16(c.k.A) || !aligned16(c.k.B)) return false;
  for (const RowsView* v : {&c.X, &c.Y, &c.dX})
    if (v->data && (!aligned16(v->data) || v->stride % 8)) return false;
  return aligned16(c.dA) && aligned16(c.dB);
}

int tc_adapters_fwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  const Layout l = ag_layout(c.k, c.T, false, ws);
  int* status = reinterpret_cast<int*>(ws);
  AgPoolParams pool{};
  pool.c = c; pool.rows_there = l.rows; pool.status = status; pool.sources = 1;
  pool.src[0] = ag_source(c.X, c.k.d_in, c.k.l1, true, l.x);
  QB_TRY(ag_launch_pool(pool, l.rows, st));
  QB_TRY(ag_shrink(c, l, status, l.x, l.u, c.k.A, false, false, st));
  return ag_expand(c, l, status, l.u, c.k.B, c.k.Q, false, c.Y, c.k.l2, true, st);
}

int tc_adapters_bwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  const Layout l = ag_layout(c.k, c.T, true, ws);
  int* status = reinterpret_cast<int*>(ws);
  const bool grads = c.dA || c.dB;
  AgPoolParams pool{};
  pool.c = c; pool.rows_there = l.rows; pool.status = status; pool.sources = grads ? 2 : 1;
  pool.src[0] = ag_source(c.Y, c.k.d_out, c.k.l2, false, l.dv);
  if (grads) pool.src[1] = ag_source(c.X, c.k.d_in, c.k.l1, true, l.x);
  QB_TRY(ag_launch_pool(pool, l.rows, st));
  if (c.dX.data || c.dA) QB_TRY(ag_shrink(c, l, status, l.dv, l.du, c.k.B, true, true, st));
  if (c.dB) QB_TRY(ag_shrink(c, l, status, l.x, l.u, c.k.A, false, false, st));
  if (c.dX.data) QB_TRY(ag_expand(c, l, status, l.du, c.k.A, c.k.P, true, c.dX, c.k.l1, false, st));
  if (grads) QB_TRY(ag_grad(c, l, status, st));
  return QBLORA_OK;
}

}  // namespace qb
