// Many adapters over one weight on the tensor cores (tcgen05): forward and backward of qblora_adapters_fwd / _bwd for rows of any
// number, fast sizes (tc_adapters_supported).
//
// The adapter's products are thin: their operands are small beside X, Y and dX, which pass once.  So four kinds of kernels, all
// over the rows in the plan's order, where every adapter's rows are neighbours:
//   pool    x' of every row (and the sums of dY's neighbours) as two or three bf16 parts: reads X at the memory's rate
//   shrink  u = x' A (and du = dv B^T): parts in, parts out
//   spread  Y += s repeat(u B) (and dX += repeat(du A^T) / lambda): the memory-bound end
//   grad    dA = x'^T du, dB = u^T dv: sums over an adapter's rows
// In shrink and spread the weights are the 128 rows of the tensor core's tile and the tokens its columns, 16 to 128 of them as an
// adapter has rows: a lone decoding row costs a tile of 16, not of 128.
//
// Parts: a number in fp32 is the sum of bf16 numbers, each the rounding of what the ones before leave.  One would put 2^-9 on everything
// that the adapter adds; two leave 2^-16 and are taken where the result is bf16; results in fp32 take three (2^-24, the rounding of
// fp32 itself).  Each part is an MMA with the same weights; x' of lambda = 1 is a bf16 number, one part.
//
// Rows in the workspace: adapter a's begin at a multiple of 16 (pad[a]) and are filled up to one with zeros, so that the sums over
// rows in grad run in whole steps of 16.  Which adapter has which tile is found by every CTA for itself from the plan's offsets.
//
// The loops of the last three are persistent: one CTA per SM takes the units in turn; warp 0 loads by TMA, warp 1 issues the MMAs, eight
// warps (sixteen in spread) empty one accumulator while the next is filled.
#include <algorithm>
#include <atomic>

#include "adapter_groups.cuh"
#include "tc_ptx.cuh"
#include "tc_small.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int AG_THREADS = 320, AG_EPI = 256;       // TMA warp, MMA warp, eight epilogue warps
constexpr int AG_TILE = 16384;                      // bytes of one 128 x 64 operand tile
constexpr int AG_POOL_THREADS = 256;
constexpr int AG_SMEM = 232448 - 1024 - 1024;        // of a CTA, without alignment and static variables
constexpr int AG_BARS = 512;                        // of those, barriers

// ---- pool ---------------------------------------------------------------------------------------------------------------------
// A matrix of rows in the workspace in np parts: element (part, row, i) at part * stride + row * ld + i.
struct Parts { __nv_bfloat16* p; int np, width, ld; int64_t stride; };

struct AgPool {
  RowsView x;
  int d, lam, log;                      // elements of a row, pooled by lam = 2^log; -1: another lam, or a large one
  float factor;                         // 1 / lam or 1
  Parts out;                            // one part: lam = 1, the values are bf16 numbers already
};
struct AgPoolParams {
  AdaptersCall c;
  AgPool src[2];
  int sources;
  uint32_t rows_there;
  int* status;
  uint32_t* tickets;                    // of grad
  int n_tickets, per, least, sms;
};

// N neighbouring values (1, 2 or 4) as parts, at `at` of the first part
template <int N>
__device__ __forceinline__ void ag_store_parts(const Parts& o, int64_t at, const float (&x)[N]) {
  float left[N];
#pragma unroll
  for (int i = 0; i < N; ++i) left[i] = x[i];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (k >= o.np) break;
    __nv_bfloat16* out = o.p + k * o.stride + at;
    if constexpr (N == 1) {
      const __nv_bfloat16 h = __float2bfloat16_rn(left[0]);
      *out = h;
      left[0] -= __bfloat162float(h);
    } else {
      uint32_t h[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        h[i] = pack_bf16x2(left[2 * i], left[2 * i + 1]);
        left[2 * i] -= ag_low(h[i]);
        left[2 * i + 1] -= ag_high(h[i]);
      }
      if constexpr (N == 2) *reinterpret_cast<uint32_t*>(out) = h[0];
      else *reinterpret_cast<uint2*>(out) = make_uint2(h[0], h[1]);
    }
  }
}

// One row by one warp, lam = 2^LOG, in 16-byte loads: four of them per lane and turn, the next turn's on their way.  The kernel would be bound
// by its instructions (117 per load with lam at run time and a store of its own per load: 3.3 TB/s), so everything here is fixed.
template <int LOG>
__device__ __forceinline__ void ag_pool_fast(const AgPool& p, const __nv_bfloat16* x, int64_t at, int lane) {
  constexpr int U = 4, LANES = LOG > 3 ? 1 << (LOG - 3) : 1;      // lanes that share a result
  const int chunks = p.d >> 3;
  uint4 next[U];
  auto ask = [&](int c0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ch = c0 + u * 32 + lane;
      next[u] = ch < chunks ? __ldcs(reinterpret_cast<const uint4*>(x) + ch) : make_uint4(0, 0, 0, 0);
    }
  };
  ask(0);
  for (int c0 = 0; c0 < chunks; c0 += 32 * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
    ask(c0 + 32 * U);
    float g[U];                                           // LOG >= 3: of eight, then of all
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ch = c0 + u * 32 + lane;
      const uint32_t e[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
      if constexpr (LOG == 0) {
        if (ch < chunks) *reinterpret_cast<uint4*>(p.out.p + at + 8 * (int64_t)ch) = w[u];
      } else {
        float s[4];                                       // sums of neighbouring two
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = ag_low(e[i]) + ag_high(e[i]);
        if constexpr (LOG == 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[i] *= p.factor;
          if (ch < chunks) ag_store_parts<4>(p.out, at + 4 * (int64_t)ch, s);
        } else if constexpr (LOG == 2) {
          const float f[2] = {(s[0] + s[1]) * p.factor, (s[2] + s[3]) * p.factor};
          if (ch < chunks) ag_store_parts<2>(p.out, at + 2 * (int64_t)ch, f);
        } else {
          g[u] = ((s[0] + s[1]) + (s[2] + s[3])) * p.factor;
#pragma unroll
          for (int d = 1; d < LANES; d <<= 1) g[u] += __shfl_xor_sync(0xffffffffu, g[u], d);
        }
      }
    }
    if constexpr (LOG >= 3) {
      // the lanes that share a result hold it for every u: each stores another one's
      constexpr int K = LANES < U ? LANES : U;            // results that go out side by side
      const int mine = lane & (LANES - 1);
#pragma unroll
      for (int u = 0; u < U; u += K) {
        float v[1] = {g[u]};
        int which = 0;
#pragma unroll
        for (int i = 1; i < K; ++i)
          if (mine == i) { v[0] = g[u + i]; which = i; }
        const int ch = c0 + (u + which) * 32 + lane;
        if (mine < K && ch < chunks) ag_store_parts<1>(p.out, at + ch / LANES, v);
      }
    }
  }
}

// One row by one warp.  x: nullptr for a row of zeros.
__device__ void ag_pool_row(const AgPool& p, const __nv_bfloat16* x, int64_t row, int lane) {
  const int64_t at = row * p.out.ld;
  if (!x) {
    const float zero[1] = {0.f};
    for (int i = lane; i < p.out.width; i += 32) ag_store_parts<1>(p.out, at + i, zero);
    return;
  }
  switch (p.log) {
    case 0: return ag_pool_fast<0>(p, x, at, lane);
    case 1: return ag_pool_fast<1>(p, x, at, lane);
    case 2: return ag_pool_fast<2>(p, x, at, lane);
    case 3: return ag_pool_fast<3>(p, x, at, lane);
    case 4: return ag_pool_fast<4>(p, x, at, lane);
    case 5: return ag_pool_fast<5>(p, x, at, lane);
    case 6: return ag_pool_fast<6>(p, x, at, lane);
    case 7: return ag_pool_fast<7>(p, x, at, lane);
    case 8: return ag_pool_fast<8>(p, x, at, lane);
  }
  for (int i = lane; i < p.out.width; i += 32) {
    float acc[1] = {0.f};
    for (int l = 0; l < p.lam; ++l) acc[0] += __bfloat162float(x[(int64_t)i * p.lam + l]);
    if (p.factor != 1.f) acc[0] /= (float)p.lam;
    ag_store_parts<1>(p.out, at + i, acc);
  }
}

// Parts begin at least this far apart in the plan: they have half of `least` rows, as filled up to a multiple of 16.
__host__ __device__ inline int ag_apart(int least) { return least / 2 - 16; }
// Rows above which an adapter is cut: the largest adapter in 1 to 16 parts, whichever takes the least time as counted in rows: rounds of
// the units over the SMs, each the longest part and about 150 rows' time for its beginning and end, and 400 more where tiles go through
// memory. One CTA of the pooling kernel finds it beside the others: in front of the gradients it takes 7 us.  (4096 -> 4096, lambda 4, the
// whole backward pass without dX, us.  Rank 64: one adapter of 8192 rows whole 219, in 4 parts 109, 8 94, 16 102; six of 1100 whole 77,
// cut in two 85.  Rank 256: one of 1800 67, in 4 parts 49; three of 600 46, cut in two 55.)
__device__ int ag_split(const AdaptersCall& c, int per, int least, int sms) {
  __shared__ int s_most, s_units[8], s_longest[8];
  const int tid = threadIdx.x;
  if (tid < 8) s_units[tid] = s_longest[tid] = 0;
  if (tid == 0) s_most = 0;
  __syncthreads();
  auto rows_of = [&](int a) { return max(plan_start(c, a + 1) - plan_start(c, a), 0); };
  int most = 0;
  for (int a = tid; a < c.k.n; a += AG_POOL_THREADS) most = max(most, rows_of(a));
  most = __reduce_max_sync(0xffffffffu, most);
  if ((tid & 31) == 0) atomicMax(&s_most, most);
  __syncthreads();
  most = s_most;
  auto cuts = [](int i) { return i < 4 ? i + 1 : i == 4 ? 6 : i == 5 ? 8 : i == 6 ? 12 : 16; };
  auto rows_at = [&](int i) { return max((uint32_t)least, (((uint32_t)most + cuts(i) - 1) / cuts(i) + 31) & ~31u); };
  for (int i = 0; i < 8; ++i) {
    const uint32_t limit = rows_at(i);
    int units = 0, longest = 0;
    for (int a = tid; a < c.k.n; a += AG_POOL_THREADS) {
      const uint32_t rows = rows_of(a), parts = (rows + limit - 1) / limit;
      units += parts;
      if (parts) longest = max(longest, (int)(rows / parts));
    }
    units = __reduce_add_sync(0xffffffffu, units);
    longest = __reduce_max_sync(0xffffffffu, longest);
    if ((tid & 31) == 0) { atomicAdd(&s_units[i], units); atomicMax(&s_longest[i], longest); }
  }
  __syncthreads();
  int best = 0;
  long long lowest = 0;
  for (int i = 0; i < 8; ++i) {
    const long long rounds = ((long long)s_units[i] * per + sms - 1) / sms, cost = rounds * (s_longest[i] + 150) + (rows_at(i) < (uint32_t)most ? 400 : 0);
    if (i == 0 || cost < lowest) { lowest = cost; best = i; }
  }
  return (int)rows_at(best);
}

__global__ void __launch_bounds__(AG_POOL_THREADS) adapters_pool_kernel(const __grid_constant__ AgPoolParams p) {
  extern __shared__ uint32_t ag_smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = QBLORA_OK;
  const int extra = p.n_tickets > 0, block = (int)blockIdx.x - extra, blocks = (int)gridDim.x - extra;
  if (block < 0) {
    for (int i = threadIdx.x; i < p.n_tickets; i += AG_POOL_THREADS) p.tickets[i] = 0u;
    const AgGroups g = ag_groups<AG_POOL_THREADS>(p.c, ag_smem, p.rows_there, ag_split(p.c, p.per, p.least, p.sms));
    uint32_t* out = p.tickets + p.n_tickets;
    if (threadIdx.x == 0) out[0] = (uint32_t)g.kept;
    for (int i = threadIdx.x; i < 2 * (p.c.k.n + 1); i += AG_POOL_THREADS) out[1 + i] = ag_smem[i];
    return;
  }
  const AgGroups g = ag_groups<AG_POOL_THREADS>(p.c, ag_smem, p.rows_there, 128);
  const int lane = threadIdx.x & 31, warps = AG_POOL_THREADS / 32;
  const uint32_t rows = g.pad[g.kept];
  for (int64_t i = (int64_t)block * warps + (threadIdx.x >> 5); i < (int64_t)rows * p.sources; i += (int64_t)blocks * warps) {
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

// ---- shrink -------------------------------------------------------------------------------------------------------------------
// What bounds it: the operands' way into shared memory, about 40 bytes a cycle of each SM however many there are (a step of 64 of the
// contraction: 24 KB 0.39 us, 32 KB 0.44), and 7 us of beginning and end.  1800 rows, contraction 1024, rank 256, both sides: 19 us.
struct AgMaps3 { CUtensorMap w, rows, rows16; };      // the bank's matrix; the rows' parts in boxes of tn rows and of 16
// u = x' A, du = s dv B^T, or both side by side.
struct AgShrinkSide {
  int np, K, w_kmajor, scaled;          // parts of the input; contraction; the weight's contiguous dimension is the contraction's; times
  Parts out;                            // the adapter's factor
  const __nv_bfloat16 *in, *W;          // what the tensor maps describe: the input's first part, the bank's matrix
  int in_ld;
};
struct AgShrink {
  AdaptersCall c;
  uint32_t rows_there;                  // of the workspace
  int tn, stages, np;                   // rows of a tile; of the ring; most parts
  int segment;                          // 64-wide blocks of the contraction that one accumulator takes
  int m_tiles, sides;                   // tiles of 128 ranks
  AgShrinkSide side[2];
  int* status;
  long long wait_limit;
};
struct AgShrinkMaps { AgMaps3 side[2]; };

// The warps that load and that issue MMAs walk their loops whole, on values that are the same in every lane, and one elected lane
// issues: the operands then lie in uniform registers (12 cycles an MMA; from one lane's private loop 60).
__device__ __forceinline__ int ag_uni(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool ag_elect() {
  uint32_t leader;
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(leader));
  return leader != 0;
}
__device__ __forceinline__ bool ag_wait(uint32_t bar, uint32_t parity, int* status, long long limit) {     // by a whole warp
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, status, limit));
}

// A tile of one adapter's rows; the same in every lane of a warp.
struct AgRows { int a, j, rows, n16; uint32_t at; };   // adapter, first entry in the plan, rows, the same in steps of 16, place in the workspace
__device__ __forceinline__ AgRows ag_rows(const AdaptersCall& c, const AgGroups& g, uint32_t tile, int tn) {
  AgRows t;
  t.a = ag_uni(ag_find(g.tile, g.kept, tile));
  const int i = ag_uni((int)(tile - g.tile[t.a])) * tn;
  t.at = (uint32_t)ag_uni((int)g.pad[t.a]) + i;
  t.j = ag_uni(plan_start(c, t.a)) + i;
  t.rows = min(tn, ag_uni(plan_start(c, t.a + 1)) - t.j);
  t.n16 = (t.rows + 15) & ~15;
  return t;
}
// Rows of part `part`, 64 columns from k0 on.  Returns nothing: the bytes are n16 * 128.
__device__ __forceinline__ void ag_load_rows(const AgMaps3& maps, uint32_t dst, uint32_t bar, int k0, const AgRows& t, int tn, int part) {
  if (t.n16 == tn) {
    tma_load_3d(dst, &maps.rows, bar, k0, (int)t.at, part);
  } else {
    for (int i = 0; i < t.n16; i += 16) tma_load_3d(dst + i * 128, &maps.rows16, bar, k0, (int)t.at + i, part);
  }
}
// 128 rows m of the bank's matrix, 64 of the contraction
__device__ __forceinline__ void ag_load_weights(const AgMaps3& maps, uint32_t dst, uint32_t bar, bool kmajor, int k0, int m0, int a) {
  if (kmajor) {
    tma_load_3d(dst, &maps.w, bar, k0, m0, a);
  } else {
    tma_load_3d(dst, &maps.w, bar, m0, k0, a);
    tma_load_3d(dst + 8192, &maps.w, bar, m0 + 64, k0, a);
  }
}
// D fp32, A and B bf16; transposed: the operand's rows, not the contraction, are contiguous
__device__ __forceinline__ uint32_t ag_idesc(bool a_transposed, bool b_transposed, int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_transposed ? 1u : 0u) << 15) | ((b_transposed ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(128 >> 4) << 24);
}
// Operand descriptors of a block of the contraction: K-major, or transposed with `group` bytes between runs of 64 rows.  A step of 16
// is AG_STEP_K or AG_STEP_T further.
constexpr uint64_t AG_STEP_K = 32 >> 4, AG_STEP_T = 2048 >> 4;
__device__ __forceinline__ uint64_t ag_desc(uint32_t block, bool transposed, uint32_t group = 8192) {
  return transposed ? smem_desc(block, group, 1024) : smem_desc(block, 16, 1024);
}
// The MMAs of up to four steps of 16: the weights by the first part of the rows into d0, by the others (each `part` further) into d1.  One
// lane issues them, and what it computes for an MMA is time between them: whole blocks take constants alone.  fresh: the accumulators
// begin with this block.
template <int NP, bool KMAJOR>
__device__ __forceinline__ void ag_issue(uint32_t d0, uint32_t d1, uint64_t a, uint64_t b, uint64_t part, uint32_t idesc, int n, uint32_t fresh) {
  constexpr uint64_t STEP = KMAJOR ? AG_STEP_K : AG_STEP_T;
  const uint64_t b1 = b + part, b2 = b1 + part;
  auto step = [&](uint64_t x, uint64_t y, uint32_t acc) {
    tc_mma(d0, a + x, b + y, idesc, acc);
    tc_mma(d1, a + x, b1 + y, idesc, acc);
    if constexpr (NP > 2) tc_mma(d1, a + x, b2 + y, idesc, 1u);
  };
  step(0, 0, fresh ^ 1u);
  if (n == 4) {
    step(STEP, AG_STEP_K, 1u);
    step(2 * STEP, 2 * AG_STEP_K, 1u);
    step(3 * STEP, 3 * AG_STEP_K, 1u);
  } else {
    for (int e = 1; e < n; ++e) step(e * STEP, e * AG_STEP_K, 1u);
  }
}
template <bool KMAJOR>
__device__ __forceinline__ void ag_issue_parts(int np, uint32_t d0, uint32_t d1, uint64_t a, uint64_t b, uint64_t part, uint32_t idesc, int n,
                                               uint32_t fresh) {
  if (np == 2) ag_issue<2, KMAJOR>(d0, d1, a, b, part, idesc, n, fresh);
  else ag_issue<3, KMAJOR>(d0, d1, a, b, part, idesc, n, fresh);
}
// v += 32 columns of tensor memory
__device__ __forceinline__ void ag_gather(uint32_t taddr, float* v) {
  uint32_t w[32];
  tc_ld32(taddr, w);
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] += __uint_as_float(w[j]);
}

// What is not finite.  Where a factor is infinite, or a sum is, the products of the first parts have what the formula has there (they are zero only where
// the number is), but the smaller ones make NaN of it: the rest of an infinity is inf - inf, and a part that is zero or of the other sign meets
// an infinite weight.  So a result that is NaN is formed once more, of the first parts alone, on the CUDA cores and out of line.  (A look at each
// number as it leaves tensor memory: 2 to 3 us of each call of 70, for its instructions' way into the SM more than for their number.)
// x: n columns are there, a multiple of 16; what lies behind them is of other tiles
template <int N>
__device__ __forceinline__ bool ag_any_nan(const float* x, int n) {
  float sum[2] = {0.f, 0.f};                              // two numbers by one instruction
#pragma unroll
  for (int c = 0; c < N; c += 16) {
    if (c >= n) break;
#pragma unroll
    for (int j = c; j < c + 16; j += 2)
      asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
          : "+f"(sum[0]), "+f"(sum[1]) : "f"(x[j]), "f"(x[j + 1]));
  }
  return isnan(sum[0] + sum[1]);
}
// sum[e] = sum over i of a[i a_step] b[i b_step + e b_next]; nothing changes a sum that is NaN already
template <int N>
__device__ __forceinline__ void ag_first_parts(float (&sum)[N], const __nv_bfloat16* a, int64_t a_step, const __nv_bfloat16* b, int64_t b_step,
                                               int64_t b_next, int n) {
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  for (int i0 = 0; i0 < n; i0 += 64) {
#pragma unroll 4
    for (int i = i0; i < min(n, i0 + 64); ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] = fmaf(__bfloat162float(a[i * a_step]), __bfloat162float(b[i * b_step + e * b_next]), sum[e]);
    bool done = true;
#pragma unroll
    for (int e = 0; e < N; ++e) done = done && isnan(sum[e]);
    if (done) break;
  }
}

// The same, with the parts one behind the other (and a third apart, if not 0, whose sums go to the second's): the weights are read once for
// all of them (contraction 4096, 1800 rows, three parts: 39.5 -> 35.6 us).
template <bool KMAJOR, bool THIRD>
__device__ __forceinline__ void ag_issue_together(uint32_t d, uint32_t d1, uint64_t a, uint64_t b, uint64_t third, uint32_t idesc, uint32_t idesc1, int n,
                                                  uint32_t fresh) {
  constexpr uint64_t STEP = KMAJOR ? AG_STEP_K : AG_STEP_T;
  const uint64_t b2 = b + third;
  auto step = [&](uint64_t x, uint64_t y, uint32_t acc) {
    tc_mma(d, a + x, b + y, idesc, acc);
    if constexpr (THIRD) tc_mma(d1, a + x, b2 + y, idesc1, 1u);
  };
  step(0, 0, fresh ^ 1u);
  if (n == 4) {
    step(STEP, AG_STEP_K, 1u);
    step(2 * STEP, 2 * AG_STEP_K, 1u);
    step(3 * STEP, 3 * AG_STEP_K, 1u);
  } else {
    for (int e = 1; e < n; ++e) step(e * STEP, e * AG_STEP_K, 1u);
  }
}

// NaN among a tile's results: rows at .. of the workspace, one rank m to a lane.
__device__ __noinline__ void ag_mend_shrink(const AgShrink& p, int side, int a, uint32_t at, int rows, int m) {
  const AgShrinkSide& s = p.side[side];
  if (m >= bank_rank(p.c.k, a)) return;
  const __nv_bfloat16* W = s.W + (int64_t)a * p.c.k.r * s.K + (s.w_kmajor ? (int64_t)m * s.K : m);
  const float scale = s.scaled ? __ldg(p.c.k.s + a) : 1.0f;
  for (int j = 0; j < rows; j += 8) {                     // (the workspace has rows up to a multiple of 16)
    __nv_bfloat16* to = s.out.p + (int64_t)(at + j) * s.out.ld + m;
    bool odd[8], any = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) any |= odd[e] = j + e < rows && isnan(__bfloat162float(to[e * s.out.ld]));
    if (!any) continue;
    float sum[8];
    ag_first_parts(sum, W, s.w_kmajor ? 1 : p.c.k.r, s.in + (int64_t)(at + j) * s.in_ld, 1, s.in_ld, s.K);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x[1] = {sum[e] * scale};
      if (odd[e]) ag_store_parts<1>(s.out, (int64_t)(at + j + e) * s.out.ld + m, x);
    }
  }
}

__global__ void __launch_bounds__(AG_THREADS, 1) adapters_shrink_kernel(const __grid_constant__ AgShrinkMaps maps, const __grid_constant__ AgShrink p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t stage_bytes = AG_TILE + (uint32_t)p.np * p.tn * 128, bars = base + p.stages * stage_bytes;
  auto full = [&](int s) { return bars + 16u * s; };
  auto empty = [&](int s) { return bars + 16u * s + 8; };
  auto accfull = [&](int b) { return bars + 16u * p.stages + 8u * b; };
  auto accempty = [&](int b) { return bars + 16u * p.stages + 16 + 8u * b; };
  const uint32_t tmem_slot = bars + 16u * p.stages + 32;
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accfull(b), 1); mbar_init(accempty(b), AG_EPI / 32); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const AgGroups g = ag_groups<AG_THREADS>(p.c, reinterpret_cast<uint32_t*>(smem_raw + (bars + AG_BARS - raw)), p.rows_there, p.tn);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot_g;
  const uint32_t tiles = (uint32_t)ag_uni((int)g.tile[g.kept]);
  const long long per_side = (long long)tiles * p.m_tiles, units = per_side * p.sides;
  asm volatile("griddepcontrol.wait;" ::: "memory");     // what the kernels in front have written
  // unit u: a side, tile u / m_tiles of it, ranks from 128 (u % m_tiles) on; an adapter of a lower rank has none there
  AgRows t;
  int m0, side, steps;
  auto unit = [&](long long u) {
    side = u >= per_side ? 1 : 0;
    if (side) u -= per_side;
    const uint32_t tile = (uint32_t)(u / p.m_tiles);
    m0 = (int)(u - (long long)tile * p.m_tiles) * 128;
    t = ag_rows(p.c, g, tile, p.tn);
    steps = (p.side[side].K + 15) / 16;
    return m0 < ag_uni(bank_rank(p.c.k, t.a));
  };
  if (warp == 0) {
    const uint32_t ring = (uint32_t)ag_uni((int)base);
    const bool leader = ag_elect();
    uint32_t it = 0, ph = 0;
    int s = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      if (!unit(u)) continue;
      const int np = p.side[side].np, kmajor = p.side[side].w_kmajor;
      for (int k = 0; k < steps; k += 4, ++it) {
        ok = ag_wait(empty(s), ph ^ 1u, p.status, p.wait_limit);
        if (!ok) break;
        const uint32_t w = ring + s * stage_bytes;
        if (leader) {
          mbar_arrive_expect_tx(full(s), AG_TILE + (uint32_t)np * t.n16 * 128);
          ag_load_weights(maps.side[side], w, full(s), kmajor, k * 16, m0, t.a);
          for (int i = 0; i < np; ++i) ag_load_rows(maps.side[side], w + AG_TILE + i * t.n16 * 128, full(s), k * 16, t, p.tn, i);
        }
        __syncwarp();
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      const uint32_t n = (uint32_t)p.stages, lo = it > n ? it - n : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(full(j % n), (j / n) & 1u, p.status, p.wait_limit);
    }
  } else if (warp == 1) {
    const uint32_t ring = (uint32_t)ag_uni((int)base), tmem = (uint32_t)ag_uni((int)tmem_base);
    const bool leader = ag_elect();
    uint32_t ph = 0, done = 0;
    int s = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      if (!unit(u)) continue;
      const int np = p.side[side].np, kmajor = p.side[side].w_kmajor;
      // the parts lie one behind the other: one MMA takes them all as its columns, or the first two where three are too many
      const int together = np * t.n16 <= 256 ? np : 2;
      const uint32_t idesc = ag_idesc(!kmajor, false, together * t.n16), idesc1 = ag_idesc(!kmajor, false, t.n16);
      int left = 0, b = 0;                                 // blocks left of the segment; its accumulator
      for (int k = 0; k < steps; k += 4) {
        const bool fresh = left == 0;
        if (fresh) {
          left = p.segment;
          b = done & 1;
          ok = ag_wait(accempty(b), ((done >> 1) & 1u) ^ 1u, p.status, p.wait_limit);
          if (!ok) break;
        }
        ok = ag_wait(full(s), ph, p.status, p.wait_limit);
        if (!ok) break;
        tc_fence_after();
        const uint32_t w = ring + s * stage_bytes, d = tmem + b * 256;
        const bool last = --left == 0 || k + 4 >= steps;
        if (leader) {
          const uint64_t rows = ag_desc(w + AG_TILE, false), third = together < np ? (uint64_t)(2 * t.n16 * 128) >> 4 : 0;
          const int n = min(4, steps - k);
          const uint64_t dk = ag_desc(w, !kmajor);
          if (third && kmajor) ag_issue_together<true, true>(d, d + t.n16, dk, rows, third, idesc, idesc1, n, fresh);
          else if (third) ag_issue_together<false, true>(d, d + t.n16, dk, rows, third, idesc, idesc1, n, fresh);
          else if (kmajor) ag_issue_together<true, false>(d, d, dk, rows, 0, idesc, idesc, n, fresh);
          else ag_issue_together<false, false>(d, d, dk, rows, 0, idesc, idesc, n, fresh);
          tc_commit(empty(s));
          if (last) tc_commit(accfull(b));
        }
        __syncwarp();
        if (last) { ++done; left = 0; }
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;        // quarter of tensor memory's lanes; half of the columns
    uint32_t done = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      if (!unit(u)) continue;
      const AgShrinkSide& sd = p.side[side];
      const int together = sd.np * t.n16 <= 256 ? sd.np : 2;
      // which of its columns are rows; the others, also those that are passed over, are zeros for the gradients, whatever the weights are
      uint32_t real[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = half * 64 + e * 32 + lane, row = i < t.rows ? __ldg(p.c.rows + t.j + i) : -1;
        real[e] = __ballot_sync(0xffffffffu, row >= 0 && row < p.c.T) >> (lane & 1);
      }
      float v[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) v[j] = 0.f;
      for (int k = 0; k < steps && ok; k += 4 * p.segment) {
        const int b = done & 1;
        ok = __all_sync(0xffffffffu, mbar_wait(accfull(b), (done >> 1) & 1u, p.status, p.wait_limit));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem_base + ((uint32_t)(q * 32) << 16) + b * 256 + half * 64;
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          if (half * 64 + c >= t.n16) break;
          for (int i = 0; i < together; ++i) ag_gather(d + i * t.n16 + c, v + c);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(accempty(b));
        ++done;
      }
      if (!ok) break;
      const float scale = sd.scaled ? __ldg(p.c.k.s + t.a) : 1.0f;
      const int m = m0 + q * 32 + (lane & ~1);
      // lanes 2 i and 2 i + 1 swap, so that each has two neighbouring ranks of every other row
#pragma unroll
      for (int j = 0; j < 64; j += 2) {
        if (half * 64 + j >= t.n16) break;
        const float v0 = v[j] * scale, v1 = v[j + 1] * scale;
        const float got = __shfl_xor_sync(0xffffffffu, (lane & 1) ? v0 : v1, 1);
        const int col = half * 64 + j + (lane & 1);
        const bool there = real[j >> 5] & 1u << (j & 31);
        const float x[2] = {!there ? 0.f : (lane & 1) ? got : v0, !there ? 0.f : (lane & 1) ? v1 : got};
        if (m < sd.out.width) ag_store_parts<2>(sd.out, (int64_t)(t.at + col) * sd.out.ld + m, x);      // (the rank is a multiple of 8)
      }
      if (__any_sync(0xffffffffu, ag_any_nan<64>(v, t.n16 - half * 64))) {
        __syncwarp();
        ag_mend_shrink(p, side, t.a, t.at + half * 64, min(64, t.rows - half * 64), m0 + q * 32 + lane);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ---- spread -------------------------------------------------------------------------------------------------------------------
// One row tile's u stays in shared memory while tiles of 128 outputs of the pooled kind (q) pass.  What bounds it: Y, in and out.  The
// products go through shared memory (V), so that Y comes and goes in whole rows' pieces whatever lambda is: slabs of up to 16 KB, asked
// for as long as one is free by a warp of its own and sent back by another -- in one copy where the tile's rows are neighbours
// in Y, else row by row.  (Plain loads have no place to come to: what the operands leave of an SM's memory for its L1 is 24 KB,
// 2.2 TB/s at most.)  7168 rows by 11008 columns in bf16, lambda 4: 316 MB in 66 us, 4.8 TB/s; 6700 rows by 13824 in fp32, lambda 64: 741 MB in
// 120 us, 6.2 TB/s.
constexpr int AS_EPI = 512, AS_THREADS = 128 + AS_EPI;     // loads, MMAs, slabs in, slabs out; sixteen warps
constexpr int AS_SLAB = 16384, AS_RING = 3;
struct AgSpread {
  AdaptersCall c;
  uint32_t rows_there;                  // of the workspace
  int tn, np, kb;                       // rows of a tile (at most 64); parts of u, 2 or 3; 64-wide blocks of the slots' rank
  int slabs;
  int segment;                          // as in AgShrink
  int m_tiles, M, w_kmajor, scaled;
  const __nv_bfloat16 *u, *W;           // what the tensor maps describe: u's first part, the bank's matrix
  int u_ld;
  RowsView y;
  int lam, shift;                       // shift: log2 of the bytes of one q, where they are a power of two
  int boxes;                            // whole slabs of neighbouring rows by tensor copies: pieces of a row's 128 q; 0: none
  float factor;
  int* status;
  long long wait_limit;
};
struct AsMaps { AgMaps3 in; CUtensorMap y; };

__device__ __forceinline__ void as_bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void as_bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void as_tensor_store(const CUtensorMap* tm, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(tm), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// whether any thread of the epilogue warps says so; a barrier of theirs
__device__ __forceinline__ bool as_any(bool x) {
  uint32_t y;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 512, p;\n selp.u32 %0, 1, 0, q;\n}"
               : "=r"(y) : "r"((uint32_t)x) : "memory");
  return y != 0;
}
__device__ __forceinline__ void ag_gather16(uint32_t taddr, float* v) {
  uint32_t w[16];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]), "=r"(w[8]), "=r"(w[9]),
                 "=r"(w[10]), "=r"(w[11]), "=r"(w[12]), "=r"(w[13]), "=r"(w[14]), "=r"(w[15])
               : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 16; ++j) v[j] += __uint_as_float(w[j]);
}

// Y's part of one (row tile, q tile) in slabs: `count` rows from r0 on, bytes off .. off + len - 1 of each.  Where a row's 128 q fit a slab
// several times, whole rows; else pieces of one row.
struct AsSlabs {
  int rows, row_bytes, per, pitch;             // of the tile; bytes of a row's q; rows to a slab; bytes of a row in a slab
  int r0, off, count, len;
  __device__ __forceinline__ AsSlabs(const AgSpread& p, int whole, int m, int rows_) : rows(rows_) {
    row_bytes = min(128, p.M - m * 128) * (whole >> 7);
    per = whole <= AS_SLAB ? AS_SLAB / whole : 1;
    pitch = min(whole, AS_SLAB);
    r0 = off = 0;
    size();
  }
  __device__ __forceinline__ void size() {
    count = min(per, rows - r0);
    len = min(pitch, row_bytes - off);
  }
  __device__ __forceinline__ bool there() const { return r0 < rows; }
  __device__ __forceinline__ void next() {
    if (off + pitch < row_bytes) {
      off += pitch;
    } else {
      off = 0;
      r0 += per;
    }
    size();
  }
};

// The products of a chunk of 16 bytes of Y.  QPC: different q in it.
template <int QPC>
__device__ __forceinline__ void as_products(const float* f, float (&q)[QPC]) {
  if constexpr (QPC == 1) q[0] = *f;
  else if constexpr (QPC == 2) { const float2 x = *reinterpret_cast<const float2*>(f); q[0] = x.x; q[1] = x.y; }
  else {
#pragma unroll
    for (int j = 0; j < QPC; j += 4) {
      const float4 x = *reinterpret_cast<const float4*>(f + j);
      q[j] = x.x; q[j + 1] = x.y; q[j + 2] = x.z; q[j + 3] = x.w;
    }
  }
}
template <bool F32, int QPC>
__device__ __forceinline__ uint4 as_add(uint4 y, const float (&q)[QPC]) {
  constexpr int E = F32 ? 4 : 8;
  uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (F32) w[e] = __float_as_uint(__uint_as_float(w[e]) + q[e * QPC / E]);
    else w[e] = pack_bf16x2(ag_low(w[e]) + q[2 * e * QPC / E], ag_high(w[e]) + q[(2 * e + 1) * QPC / E]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Any slab; v: the products of its first row, the others 128 floats on.  QPC 0: lam is no power of two.
template <bool F32, int QPC>
__device__ __noinline__ void as_sums(uint8_t* slab, int pitch, const float* v, int count, int off, int len, int lam, int shift, int tid) {
  const int per = len >> 4, all = per * count;
  for (int i = tid; i < all; i += AS_EPI) {
    const int row = i / per, b = (i - row * per) << 4;
    uint4* at = reinterpret_cast<uint4*>(slab + row * pitch + b);
    const float* f = v + row * 128;
    if constexpr (QPC == 0) {
      constexpr int E = F32 ? 4 : 8;
      float q[E];
#pragma unroll
      for (int e = 0; e < E; ++e) q[e] = f[((off + b) / (F32 ? 4 : 2) + e) / lam];
      *at = as_add<F32, E>(*at, q);
    } else {
      float q[QPC];
      as_products<QPC>(f + ((off + b) >> shift), q);
      *at = as_add<F32, QPC>(*at, q);
    }
  }
}

// NaN among V's rows j .. j + 15 of the tile, column q of it, which is output m.
__device__ __noinline__ void as_mend(const AgSpread& p, float* v, int a, uint32_t at, int rows, int m, float scale) {
  if (m >= p.M) return;
  const int r = bank_rank(p.c.k, a);
  const __nv_bfloat16* W = p.W + (int64_t)a * p.c.k.r * p.M + (p.w_kmajor ? (int64_t)m * p.c.k.r : m);
  for (int j = 0; j < rows; ++j)
    if (isnan(v[j * 128])) {
      float sum[1];
      ag_first_parts(sum, p.u + (int64_t)(at + j) * p.u_ld, 1, W, p.w_kmajor ? 1 : p.M, 0, r);
      v[j * 128] = sum[0] * scale;
    }
}

template <bool F32, int QPC>
__global__ void __launch_bounds__(AS_THREADS, 1) adapters_spread_kernel(const __grid_constant__ AsMaps maps, const __grid_constant__ AgSpread p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), s_u = (raw + 1023u) & ~1023u;
  const uint32_t block = (uint32_t)p.tn * 128;                        // one part's 64 ranks
  const uint32_t s_w = s_u + p.np * p.kb * block, s_slab = s_w + AS_RING * AG_TILE, s_v = s_slab + p.slabs * AS_SLAB;
  const uint32_t bars = s_v + p.tn * 512;
  auto wfull = [&](int s) { return bars + 16u * s; };
  auto wempty = [&](int s) { return bars + 16u * s + 8; };
  const uint32_t ufull = bars + 16u * AS_RING, uempty = ufull + 8;
  auto accfull = [&](int b) { return ufull + 16 + 8u * b; };
  auto accempty = [&](int b) { return ufull + 32 + 8u * b; };
  auto in = [&](int i) { return ufull + 48 + 24u * i; };              // the slab's rows have come
  auto summed = [&](int i) { return ufull + 56 + 24u * i; };
  auto gone = [&](int i) { return ufull + 64 + 24u * i; };            // they have been read by their stores
  const uint32_t tmem_slot = ufull + 48 + 24u * p.slabs;
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    for (int s = 0; s < AS_RING; ++s) { mbar_init(wfull(s), 1); mbar_init(wempty(s), 1); }
    mbar_init(ufull, 1);
    mbar_init(uempty, 1);
    for (int b = 0; b < 2; ++b) { mbar_init(accfull(b), 1); mbar_init(accempty(b), AS_EPI / 32); }
    for (int i = 0; i < p.slabs; ++i) { mbar_init(in(i), 1); mbar_init(summed(i), AS_EPI / 32); mbar_init(gone(i), 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(256) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const AgGroups g = ag_groups<AS_THREADS>(p.c, reinterpret_cast<uint32_t*>(smem_raw + (bars + AG_BARS - raw)), p.rows_there, p.tn);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot_g;
  // A unit is one row tile and every `runs`-th q tile: as many as leave every CTA about four units, so that u is loaded seldom and the
  // CTAs still end together; neighbouring CTAs are at neighbouring parts of the same rows.
  const uint32_t tiles = (uint32_t)ag_uni((int)g.tile[g.kept]);
  const int run = (int)min((long long)p.m_tiles, max(1LL, (long long)tiles * p.m_tiles / (4 * gridDim.x)));
  const int runs = (p.m_tiles + run - 1) / run;
  const long long units = (long long)tiles * runs;
  asm volatile("griddepcontrol.wait;" ::: "memory");                  // what the kernels in front have written
  // calls f(rows, steps of 16 ranks, first q tile) for this CTA's units, until it returns false
  auto each = [&](auto&& f) {
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
      const uint32_t tile = (uint32_t)(u / runs);
      const int first = (int)(u - (long long)tile * runs);
      const AgRows t = ag_rows(p.c, g, tile, p.tn);
      const int steps = (ag_uni(bank_rank(p.c.k, t.a)) + 15) / 16;
      if (steps > 0 && !f(t, steps, first)) return;
    }
  };
  constexpr int ES = F32 ? 4 : 2;
  const int whole = 128 * p.lam * ES;                                 // bytes of a row's 128 q
  const int64_t y_pitch = p.y.stride * ES;

  if (warp == 0) {
    const uint32_t ring = (uint32_t)ag_uni((int)s_w), at_u = (uint32_t)ag_uni((int)s_u);
    const bool leader = ag_elect();
    uint32_t it = 0, ph = 0, n = 0;
    int s = 0;
    bool ok = true;
    each([&](const AgRows& t, int steps, int first) {
      const int kb = (steps + 3) / 4;
      ok = ag_wait(uempty, (n & 1u) ^ 1u, p.status, p.wait_limit);
      if (!ok) return false;
      if (leader) {
        mbar_arrive_expect_tx(ufull, (uint32_t)(p.np * kb * t.n16 * 128));
        for (int i = 0; i < p.np; ++i)
          for (int k = 0; k < kb; ++k) ag_load_rows(maps.in, at_u + (i * p.kb + k) * block, ufull, k * 64, t, p.tn, i);
      }
      __syncwarp();
      ++n;
      for (int m = first; m < p.m_tiles; m += runs)
        for (int k = 0; k < kb; ++k, ++it) {
          ok = ag_wait(wempty(s), ph ^ 1u, p.status, p.wait_limit);
          if (!ok) return false;
          if (leader) {
            mbar_arrive_expect_tx(wfull(s), AG_TILE);
            ag_load_weights(maps.in, ring + s * AG_TILE, wfull(s), p.w_kmajor, k * 64, m * 128, t.a);
          }
          __syncwarp();
          if (++s == AS_RING) { s = 0; ph ^= 1u; }
        }
      return true;
    });
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      if (n) mbar_wait(ufull, (n - 1) & 1u, p.status, p.wait_limit);
      const uint32_t lo = it > (uint32_t)AS_RING ? it - AS_RING : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(wfull(j % AS_RING), (j / AS_RING) & 1u, p.status, p.wait_limit);
    }
  } else if (warp == 1) {
    const uint32_t ring = (uint32_t)ag_uni((int)s_w), at_u = (uint32_t)ag_uni((int)s_u), tmem = (uint32_t)ag_uni((int)tmem_base);
    const bool leader = ag_elect();
    uint32_t ph = 0, done = 0, n = 0;
    int s = 0;
    each([&](const AgRows& t, int steps, int first) {
      if (!ag_wait(ufull, n & 1u, p.status, p.wait_limit)) return false;
      const uint32_t idesc = ag_idesc(!p.w_kmajor, false, t.n16);
      for (int m = first; m < p.m_tiles; m += runs)
        for (int k0 = 0; k0 < steps; k0 += 4 * p.segment, ++done) {
          const int b = done & 1, end = min(steps, k0 + 4 * p.segment);
          if (!ag_wait(accempty(b), ((done >> 1) & 1u) ^ 1u, p.status, p.wait_limit)) return false;
          tc_fence_after();
          for (int k = k0; k < end; k += 4) {
            if (!ag_wait(wfull(s), ph, p.status, p.wait_limit)) return false;
            tc_fence_after();
            const uint32_t d = tmem + b * 128;
            if (leader) {
              const uint32_t w = ring + s * AG_TILE;
              const uint64_t rows = ag_desc(at_u + (k / 4) * block, false), part = (uint64_t)(p.kb * block) >> 4;
              const int some = min(4, steps - k);
              if (p.w_kmajor) ag_issue_parts<true>(p.np, d, d + 64, ag_desc(w, false), rows, part, idesc, some, k == k0);
              else ag_issue_parts<false>(p.np, d, d + 64, ag_desc(w, true), rows, part, idesc, some, k == k0);
              tc_commit(wempty(s));
              if (k + 4 >= end) {
                tc_commit(accfull(b));
                if (end == steps && m + runs >= p.m_tiles) tc_commit(uempty);
              }
            }
            __syncwarp();
            if (++s == AS_RING) { s = 0; ph ^= 1u; }
          }
        }
      ++n;
      return true;
    });
  } else if (warp == 2 || warp == 3) {
    // ---- Y's slabs in (warp 2) and out.  The tile's row numbers are looked up once: lane l has rows l and l + 32.
    const bool out = warp == 3;
    uint32_t it = 0, ph = 0;
    int s = 0;
    bool ok = true;
    each([&](const AgRows& t, int, int first) {
      int rows0 = lane < t.rows ? __ldg(p.c.rows + t.j + lane) : -1, rows1 = lane + 32 < t.rows ? __ldg(p.c.rows + t.j + lane + 32) : -1;
      if (rows0 >= p.c.T) rows0 = -1;
      if (rows1 >= p.c.T) rows1 = -1;
      const int row_a = __shfl_sync(0xffffffffu, rows0, 0);
      const bool neighbours = p.boxes && row_a >= 0 &&
                              __all_sync(0xffffffffu, (lane >= t.rows || rows0 == row_a + lane) && (lane + 32 >= t.rows || rows1 == row_a + lane + 32));
      for (int m = first; m < p.m_tiles; m += runs) {
        char* tile = static_cast<char*>(p.y.data) + (int64_t)m * whole;
        for (AsSlabs y(p, whole, m, t.rows); y.there(); y.next(), ++it) {
          if (!ag_wait(out ? summed(s) : gone(s), out ? ph : ph ^ 1u, p.status, p.wait_limit)) return ok = false;
          const uint32_t slab = s_slab + s * AS_SLAB;
          if (neighbours && y.count == y.per) {
            // one copy of `per` rows' pieces; what would lie behind the row's end is filled with zeros, and left out on the way back
            if (lane == 0) {
              if (out) {
                as_tensor_store(&maps.y, slab, 0, m * p.boxes, row_a + y.r0);
              } else {
                mbar_arrive_expect_tx(in(s), (uint32_t)(y.per * whole));
                tma_load_3d(slab, &maps.y, in(s), 0, m * p.boxes, row_a + y.r0);
              }
            }
          } else {
            // this lane's rows of the slab: r0 + lane and r0 + lane + 32
            int row[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int r = y.r0 + lane + 32 * e, x0 = __shfl_sync(0xffffffffu, rows0, r & 31), x1 = __shfl_sync(0xffffffffu, rows1, r & 31);
              row[e] = lane + 32 * e < y.count ? (r < 32 ? x0 : x1) : -1;
            }
            if (!out) {
              const int there = __popc(__ballot_sync(0xffffffffu, row[0] >= 0)) + __popc(__ballot_sync(0xffffffffu, row[1] >= 0));
              if (lane == 0) mbar_arrive_expect_tx(in(s), (uint32_t)(there * y.len));
              __syncwarp();
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (row[e] < 0) continue;
              const uint32_t at = slab + (lane + 32 * e) * y.pitch;
              char* g = tile + row[e] * y_pitch + y.off;
              if (out) as_bulk_store(g, at, (uint32_t)y.len);
              else as_bulk_load(at, g, (uint32_t)y.len, in(s));
            }
          }
          if (out) {
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            // the slab before has been read by its stores; this one's go on
            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
            if (lane == 0 && it > 0) mbar_arrive(gone(s == 0 ? p.slabs - 1 : s - 1));
          }
          if (++s == p.slabs) { s = 0; ph ^= 1u; }
        }
      }
      return true;
    });
    if (out) {
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // written, not only read
    } else if (!ok) {
      const uint32_t n = (uint32_t)p.slabs, lo = it > n ? it - n : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(in(j % n), (j / n) & 1u, p.status, p.wait_limit);
    }
  } else {
    const int q = warp & 3, part = (warp - 4) >> 2, etid = tid - 128;    // quarter of the lanes, 16 of the columns
    float* v = reinterpret_cast<float*>(smem_raw + (s_v - raw));
    // Where a row's 128 q are a power of two of bytes, a whole slab's chunks have the same places every time: chunk etid and
    // chunk etid + 512 of the slab's 1024, their bytes in the slab and their products in V.
    const int at0 = etid * 16, at1 = at0 + AS_EPI * 16;
    int f0 = 0, f1 = 0;
    if constexpr (QPC > 0) {
      const int pitch = min(whole, AS_SLAB);
      f0 = at0 / pitch * 128 + ((at0 & (pitch - 1)) >> p.shift);
      f1 = at1 / pitch * 128 + ((at1 & (pitch - 1)) >> p.shift);
    }
    uint32_t done = 0, ph = 0;
    int s = 0;
    each([&](const AgRows& t, int steps, int first) {
      const float scale = p.scaled ? __ldg(p.c.k.s + t.a) * p.factor : p.factor;
      for (int m = first; m < p.m_tiles; m += runs) {
        float x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = 0.f;
        bool ok = true;
        for (int k = 0; k < steps && ok; k += 4 * p.segment, ++done) {
          const int b = done & 1;
          ok = __all_sync(0xffffffffu, mbar_wait(accfull(b), (done >> 1) & 1u, p.status, p.wait_limit));
          if (!ok) break;                                             // (all leave together, below)
          tc_fence_after();
          if (part * 16 < t.n16) {
            const uint32_t d = tmem_base + ((uint32_t)(q * 32) << 16) + b * 128 + part * 16;
            ag_gather16(d, x);
            ag_gather16(d + 64, x);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(accempty(b));
        }
        if (as_any(!ok)) return false;                                // (and V's readers of the tile before are done)
        if (part * 16 < t.n16) {
#pragma unroll
          for (int j = 0; j < 16; ++j) v[(part * 16 + j) * 128 + q * 32 + lane] = x[j] * scale;
          if (ag_any_nan<16>(x, 16))
            as_mend(p, v + part * 16 * 128 + q * 32 + lane, t.a, t.at + part * 16, min(16, t.rows - part * 16), m * 128 + q * 32 + lane, scale);
        }
        asm volatile("bar.sync 1, 512;" ::: "memory");
        for (AsSlabs y(p, whole, m, t.rows); y.there(); y.next()) {
          ok = __all_sync(0xffffffffu, mbar_wait(in(s), ph, p.status, p.wait_limit));
          if (ok) {
            uint8_t* slab = smem_raw + (s_slab - raw) + s * AS_SLAB;
            if (QPC > 0 && y.count * y.len == AS_SLAB) {
              constexpr int N = QPC > 0 ? QPC : 1;
              const float* f = v + y.r0 * 128 + (y.off >> p.shift);
              uint4 *a0 = reinterpret_cast<uint4*>(slab + at0), *a1 = reinterpret_cast<uint4*>(slab + at1);
              const uint4 y0 = *a0, y1 = *a1;
              float q0[N], q1[N];
              as_products<N>(f + f0, q0);
              as_products<N>(f + f1, q1);
              *a0 = as_add<F32, N>(y0, q0);
              *a1 = as_add<F32, N>(y1, q1);
            } else {
              as_sums<F32, QPC>(slab, y.pitch, v + y.r0 * 128, y.count, y.off, y.len, p.lam, p.shift, etid);
            }
          }
          fence_async_proxy();                                        // the stores read what was written here
          __syncwarp();
          if (lane == 0) mbar_arrive(summed(s));
          if (++s == p.slabs) { s = 0; ph ^= 1u; }
        }
      }
      return true;
    });
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256) : "memory");
  }
}

// ---- grad ---------------------------------------------------------------------------------------------------------------------
// Tiles of 128 x 128 of dA and dB.  Both operands are rows of the workspace, contraction over the rows: parts 0 x 0 are one
// accumulator, the smaller products (0 x 1, 1 x 0, 1 x 1, 0 x 2, 2 x 0: the others are below 2^-24) a second, so that the sum of the large
// ones is rounded no more often than it must be.
// Every AR_SEGMENT blocks of 32 rows the accumulators are emptied into registers: the tensor core's sums lose about 2^-26 of themselves
// per step of 16, always towards zero (4096 terms in one go: 4e-6 of the result; in pieces of 256: below 1e-6).
// What bounds it: for 6700 rows of six adapters (216 and 640 by 256) 33 us, for 1800 of three (1024 both) 24, a third of it beginning and end; the
// MMAs are 5 of them.  Few adapters have few tiles, so the rows of one are cut where that makes use of more SMs (ag_split); a part's tile then goes
// through memory, and the part that comes last adds them in the parts' order: equal inputs give equal bits.
constexpr int AR_BLOCK = AG_TILE / 2, AR_STAGES = 4, AR_STAGE = 6 * AR_BLOCK, AR_SEGMENT = 8;
// up to two steps of 16: parts 0 x 0 into d, the smaller products into d + 128
template <int PA, int PB>
__device__ __forceinline__ void ar_issue(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, int n, bool fresh) {
  constexpr uint64_t part = AR_BLOCK >> 4;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (e >= n) break;
    uint32_t acc = fresh && e == 0 ? 0u : 1u;
    tc_mma(d, a, b, idesc, acc);
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
      for (int j = 0; j < PB; ++j)
        if (i + j > 0 && i + j <= 2) {
          tc_mma(d + 128, a + i * part, b + j * part, idesc, acc);
          acc = 1u;
        }
    a += AG_STEP_T;
    b += AG_STEP_T;
  }
}
struct AgGradSide { int parts_a, parts_b, M, N; float* out; const __nv_bfloat16 *a, *b; int a_ld, b_ld; };     // dA: x' (P) by du (r); dB: u (r) by dv (Q)
struct AgGrad {
  AdaptersCall c;
  uint32_t rows_there;
  AgGradSide side[2];                   // out == nullptr: not wanted
  int least;                            // an adapter of more rows than ag_split says is cut into parts; it says no less than this
  float* parts;                         // their tiles, [slot][tile][128 x 128], where a part's slot is its first place in the plan / ag_apart(least)
  uint32_t* tickets;                    // [slot][tile]: parts that are there; zero before the call.  Then its AgGroups: kept, pad, tile
  int n_tickets;                        // 0: no adapter can be cut
  int* status;
  long long wait_limit;
};
struct AgGradMaps { CUtensorMap a[2], b[2]; };

// whether any of the eight epilogue warps says so; a barrier of theirs
__device__ __forceinline__ bool ar_any(bool x) {
  uint32_t y;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 256, p;\n selp.u32 %0, 1, 0, q;\n}"
               : "=r"(y) : "r"((uint32_t)x) : "memory");
  return y != 0;
}

// NaN among a thread's results: row m, columns n .. of them, at `out`; the adapter's rows in the workspace.
__device__ __noinline__ void ar_mend(const AgGradSide& s, float* out, int m, int n, int columns, uint32_t at, int rows, float scale) {
  for (int j = 0; j < columns; j += 8) {                  // (they are a multiple of 8)
    bool any = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) any |= isnan(out[j + e]);
    if (!any) continue;
    float sum[8];
    ag_first_parts(sum, s.a + (int64_t)at * s.a_ld + m, s.a_ld, s.b + (int64_t)at * s.b_ld + n + j, s.b_ld, 1, rows);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (isnan(out[j + e])) out[j + e] = sum[e] * scale;
  }
}

__global__ void __launch_bounds__(AG_THREADS, 1) adapters_grad_kernel(const __grid_constant__ AgGradMaps maps, const __grid_constant__ AgGrad p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ bool s_last;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u, bars = base + AR_STAGES * AR_STAGE;
  auto full = [&](int s) { return bars + 16u * s; };
  auto empty = [&](int s) { return bars + 16u * s + 8; };
  auto accfull = [&](int b) { return bars + 16u * AR_STAGES + 8u * b; };
  auto accempty = [&](int b) { return bars + 16u * AR_STAGES + 16 + 8u * b; };
  const uint32_t tmem_slot = bars + 16u * AR_STAGES + 32;
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    for (int s = 0; s < AR_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accfull(b), 1); mbar_init(accempty(b), AG_EPI / 32); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const BankView& k = p.c.k;
  const AgGradSide &sa = p.side[0], &sb = p.side[1];
  const int ca = (sa.N + 127) / 128, cb = (sb.N + 127) / 128;
  const int ta = sa.out ? (sa.M + 127) / 128 * ca : 0, tb = sb.out ? (sb.M + 127) / 128 * cb : 0;
  const int per = ta + tb;
  uint32_t* table = reinterpret_cast<uint32_t*>(smem_raw + (bars + AG_BARS - raw));
  AgGroups g;
  if (p.n_tickets == 0) g = ag_groups<AG_THREADS>(p.c, table, p.rows_there, 0x7fffffe0);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // what the kernels in front have written
  if (p.n_tickets > 0) {
    const uint32_t* from = p.tickets + p.n_tickets;
    for (int i = tid; i < 2 * (k.n + 1); i += AG_THREADS) table[i] = from[1 + i];
    g = {table, table + k.n + 1, (int)from[0]};
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot_g;
  // Units: the tiles of all parts, then those of all adapters, of which only those without rows have anything to do: zeros.
  const long long work = (long long)ag_uni((int)g.tile[g.kept]) * per, units = work + (long long)k.n * per;
  struct Unit { int a, side, m0, n0, n16, steps, rank, first, all, part, parts, tile; uint32_t at; bool skip; };
  auto part_at = [](const Unit& t, int i) { return t.parts > 1 ? (int)((long long)t.all * i / t.parts) : i ? t.all : 0; };   // in 16 rows
  auto unit = [&](long long u) {
    Unit t;
    const bool zeros = u >= work;
    if (zeros) u -= work;
    const int w = (int)(u / per);
    int x = (int)(u - (long long)w * per);
    t.tile = x;
    t.a = zeros ? w : ag_find(g.tile, g.kept, (uint32_t)w);
    t.side = x >= ta;
    if (t.side) x -= ta;
    const int cols = t.side ? cb : ca;
    t.m0 = x / cols * 128;
    t.n0 = x % cols * 128;
    t.n16 = min(128, ((t.side ? sb.N : sa.N) - t.n0 + 15) & ~15);
    t.rank = bank_rank(k, t.a);
    const bool there = t.a < g.kept;
    t.first = there ? (int)g.pad[t.a] : 0;
    t.all = there ? (int)(g.pad[t.a + 1] - g.pad[t.a]) / 16 : 0;
    t.parts = zeros ? 1 : (int)(g.tile[t.a + 1] - g.tile[t.a]);
    t.part = zeros ? 0 : w - (int)g.tile[t.a];
    const int from = part_at(t, t.part);
    t.at = (uint32_t)(t.first + from * 16);
    t.steps = (t.side ? t.m0 : t.n0) < t.rank ? part_at(t, t.part + 1) - from : 0;
    t.skip = zeros ? t.all > 0 : t.steps == 0 && t.part > 0;
    return t;
  };
  auto uniform = [&](Unit t) {
    t.a = ag_uni(t.a); t.side = ag_uni(t.side); t.m0 = ag_uni(t.m0); t.n0 = ag_uni(t.n0); t.n16 = ag_uni(t.n16); t.steps = ag_uni(t.steps);
    t.at = (uint32_t)ag_uni((int)t.at); t.skip = ag_uni(t.skip) != 0;
    return t;
  };
  if (warp == 0) {
    const uint32_t ring = (uint32_t)ag_uni((int)base);
    const bool leader = ag_elect();
    uint32_t it = 0, ph = 0;
    int s = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit t = uniform(unit(u));
      if (t.skip) continue;
      const int parts_a = p.side[t.side].parts_a, parts_b = p.side[t.side].parts_b, nb = (t.n16 + 63) / 64;
      for (int x = 0; x < t.steps; x += 2, ++it) {
        ok = ag_wait(empty(s), ph ^ 1u, p.status, p.wait_limit);
        if (!ok) break;
        const uint32_t a = ring + s * AR_STAGE, b = a + 3 * AR_BLOCK;
        const int y = (int)t.at + x * 16;
        if (leader) {
          mbar_arrive_expect_tx(full(s), (uint32_t)(4096 * (2 * parts_a + nb * parts_b)));
          for (int i = 0; i < parts_a; ++i)
            for (int j = 0; j < 2; ++j) tma_load_3d(a + i * AR_BLOCK + j * 4096, &maps.a[t.side], full(s), t.m0 + j * 64, y, i);
          for (int i = 0; i < parts_b; ++i)
            for (int j = 0; j < nb; ++j) tma_load_3d(b + i * AR_BLOCK + j * 4096, &maps.b[t.side], full(s), t.n0 + j * 64, y, i);
        }
        __syncwarp();
        if (++s == AR_STAGES) { s = 0; ph ^= 1u; }
      }
    }
    if (!ok) {
      const uint32_t lo = it > (uint32_t)AR_STAGES ? it - AR_STAGES : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(full(j % AR_STAGES), (j / AR_STAGES) & 1u, p.status, p.wait_limit);
    }
  } else if (warp == 1) {
    const uint32_t ring = (uint32_t)ag_uni((int)base), tmem = (uint32_t)ag_uni((int)tmem_base);
    const bool leader = ag_elect();
    uint32_t ph = 0, done = 0;
    int s = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit t = uniform(unit(u));
      if (t.skip) continue;
      const int parts_a = p.side[t.side].parts_a, parts_b = p.side[t.side].parts_b;
      const uint32_t idesc = ag_idesc(true, true, t.n16);
      int left = 0, b = 0;                                 // blocks left of the segment; its accumulator
      for (int x = 0; x < t.steps; x += 2) {
        const bool fresh = left == 0;
        if (fresh) {
          left = AR_SEGMENT;
          b = done & 1;
          ok = ag_wait(accempty(b), ((done >> 1) & 1u) ^ 1u, p.status, p.wait_limit);
          if (!ok) break;
        }
        ok = ag_wait(full(s), ph, p.status, p.wait_limit);
        if (!ok) break;
        tc_fence_after();
        const uint32_t pa = ring + s * AR_STAGE, d = tmem + b * 256;
        const bool last = --left == 0 || x + 2 >= t.steps;
        if (leader) {
          const uint64_t da = ag_desc(pa, true, 4096), db = ag_desc(pa + 3 * AR_BLOCK, true, 4096);
          const int n = min(2, t.steps - x);
          if (parts_a == 3 && parts_b == 3) ar_issue<3, 3>(d, da, db, idesc, n, fresh);
          else if (parts_a == 3) ar_issue<3, 1>(d, da, db, idesc, n, fresh);
          else ar_issue<1, 3>(d, da, db, idesc, n, fresh);
          tc_commit(empty(s));
          if (last) tc_commit(accfull(b));
        }
        __syncwarp();
        if (last) { ++done; left = 0; }
        if (++s == AR_STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint32_t done = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit t = unit(u);
      if (t.skip) continue;
      const AgGradSide& side = p.side[t.side];
      float v[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) v[j] = 0.f;
      for (int x = 0; x < t.steps && ok; x += 2 * AR_SEGMENT) {
        const int b = done & 1;
        ok = __all_sync(0xffffffffu, mbar_wait(accfull(b), (done >> 1) & 1u, p.status, p.wait_limit));
        if (!ok) break;                                               // (all leave together, below)
        tc_fence_after();
        const uint32_t d = tmem_base + ((uint32_t)(q * 32) << 16) + b * 256 + half * 64;
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          if (half * 64 + c >= t.n16) break;
          ag_gather(d + c, v + c);
          ag_gather(d + 128 + c, v + c);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(accempty(b));
        ++done;
      }
      ok = !ar_any(!ok);
      if (!ok) break;
      if (t.parts > 1 && t.steps > 0) {
        // This part's tile goes to memory; whoever comes last adds all of them up, in the parts' order
        const int etid = tid - 64;
        auto slot = [&](int i) { return (int64_t)((plan_start(p.c, t.a) + part_at(t, i) * 16) / ag_apart(p.least)) * per + t.tile; };
        float4* mine = reinterpret_cast<float4*>(p.parts + slot(t.part) * 16384) + etid;
#pragma unroll
        for (int j = 0; j < 16; ++j) mine[j * 256] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        __threadfence();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (etid == 0) s_last = atomicAdd(p.tickets + slot(0), 1u) + 1u == (uint32_t)t.parts;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (!s_last) continue;
        __threadfence();
#pragma unroll
        for (int j = 0; j < 64; ++j) v[j] = 0.f;
        for (int i = 0; i < t.parts; ++i) {
          const float4* from = reinterpret_cast<const float4*>(p.parts + slot(i) * 16384) + etid;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float4 x = __ldcg(from + j * 256);
            v[4 * j] += x.x; v[4 * j + 1] += x.y; v[4 * j + 2] += x.z; v[4 * j + 3] += x.w;
          }
        }
      }
      const int m = t.m0 + q * 32 + lane;
      const float scale = t.side ? __ldg(k.s + t.a) : 1.0f;           // du has it already
      if (m < side.M) {
        float* out = side.out + ((int64_t)t.a * side.M + m) * side.N + t.n0 + half * 64;
#pragma unroll
        for (int j = 0; j < 64; j += 4) {
          if (t.n0 + half * 64 + j >= side.N) break;                  // N is a multiple of 8
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = (t.side ? m : t.n0 + half * 64 + j + e) < t.rank ? v[j + e] * scale : 0.f;
          *reinterpret_cast<float4*>(out + j) = make_float4(x[0], x[1], x[2], x[3]);
        }
        if (ag_any_nan<64>(v, t.n16 - half * 64))
          ar_mend(side, out, m, t.n0 + half * 64, min(64, side.N - t.n0 - half * 64), (uint32_t)t.first, t.all * 16, scale);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------------------
struct Layout {
  Parts x, dv, u, du;
  int least;                            // of the gradients: AgGrad
  float* parts; uint32_t* tickets; int n_tickets;
  size_t bytes; uint32_t rows;
};

// tiles of one adapter's dA and dB
int64_t ag_tiles(const BankView& k) { return (int64_t)((k.P + 127) / 128 + (k.Q + 127) / 128) * ((k.r + 127) / 128); }
// parts: of numbers that are no bf16 numbers
Layout ag_layout(const BankView& k, int64_t T, bool backward, int parts, char* ws) {
  Layout l{};
  l.rows = (uint32_t)std::min<int64_t>(T + 15 * std::min<int64_t>(T, k.n), 0x7ffffff0);
  size_t at = kStatusBytes;
  auto place = [&](Parts& p, int width, int np) {
    p.np = np;
    p.width = width;
    p.ld = (width + 7) & ~7;
    p.stride = (int64_t)align_up((size_t)l.rows * p.ld, 128);
    p.p = reinterpret_cast<__nv_bfloat16*>(ws + at);
    at += (size_t)p.stride * 2 * np;
  };
  place(l.x, k.P, k.l1 > 1 ? parts : 1);
  place(l.u, k.r, parts);
  if (backward) {
    place(l.dv, k.Q, k.l2 > 1 ? parts : 1);
    place(l.du, k.r, parts);
    // parts of no fewer rows than would make two rounds over 148 SMs of one adapter's: that bounds their tiles' memory
    const int64_t per = ag_tiles(k);
    l.least = (int)std::min<int64_t>(std::max<int64_t>(256, (T * per / 296 + 31) / 32 * 32), 0x3fffffe0);
    // Room for tickets and tiles must not shrink as T grows, since a workspace serves fewer rows too: it is a bound on what follows, (T + 15) /
    // ag_apart + 1 parts, with ag_apart >= 7/16 least and least >= T per / 296.
    const int64_t room = T <= 256 || per >= 296 ? 0 : std::min<int64_t>(((T + 15) / ag_apart(256) + 1) * per, 720 + per);
    const int64_t want = T > l.least ? ((T + 15) / ag_apart(l.least) + 1) * per : 0;
    l.n_tickets = want <= room ? (int)want : 0;
    l.tickets = reinterpret_cast<uint32_t*>(ws + at);
    at += align_up(((size_t)room + 1) * 4 + ag_table_bytes(k.n), 256);
    l.parts = reinterpret_cast<float*>(ws + at);
    at += (size_t)room * 65536;
  }
  l.bytes = align_up(at, 256);
  return l;
}

AgPool ag_source(const RowsView& x, int d, int lam, bool mean, const Parts& out) {
  AgPool p{x, d, lam, -1, mean ? 1.0f / (float)lam : 1.0f, out};
  for (int i = 0; i <= 8; ++i)
    if (lam == 1 << i) p.log = i;
  return p;
}

int ag_sms(int* n) {
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
  return QBLORA_OK;
}

// A persistent kernel behind the ones in front, which it may overlap.
template <class Maps, class Params>
int ag_launch(void (*kernel)(Maps, Params), std::atomic<bool>* ready, const Maps& maps, const Params& p, int threads, size_t smem, int64_t most_units,
              cudaStream_t st) {
  int sms = 0, dev = 0;
  const int rc = ag_sms(&sms);
  if (rc) return rc;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  if (!ready[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, AG_SMEM + 1024));
    ready[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(sms, most_units)));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, kernel, maps, p));
  count_launch();
  return QBLORA_OK;
}

// The first of a call, behind all that is in front of it on the stream.
int ag_launch_pool(const AgPoolParams& p, int64_t rows, cudaStream_t st) {
  int sms = 0;
  const int rc = ag_sms(&sms);
  if (rc) return rc;
  const int64_t want = (rows * p.sources + AG_POOL_THREADS / 32 - 1) / (AG_POOL_THREADS / 32);
  cudaLaunchConfig_t cfg = {};
  AgPoolParams q = p;
  q.sms = sms;
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(want, 8LL * sms) + (p.n_tickets > 0));
  cfg.blockDim = dim3(AG_POOL_THREADS);
  cfg.dynamicSmemBytes = ag_table_bytes(p.c.k.n);
  cfg.stream = st;
  QB_CUDA(cudaLaunchKernelEx(&cfg, adapters_pool_kernel, q));
  count_launch();
  return QBLORA_OK;
}

int parts_map(CUtensorMap* tm, const Parts& p, uint32_t rows, int box_rows) {
  const uint64_t dims[3] = {(uint64_t)p.width, rows, (uint64_t)p.np};
  const uint64_t pitch[2] = {(uint64_t)p.ld * 2, (uint64_t)p.stride * 2};
  const uint32_t box[3] = {64, (uint32_t)box_rows, 1};
  return make_tensor_map_nd(tm, 3, p.p, dims, pitch, box);
}
// element (i, j) of slot a at a * rows * width + i * width + j: boxes of 64 j by `box` i
int bank_map(CUtensorMap* tm, const __nv_bfloat16* ptr, int width, int rows, int n, int box) {
  const uint64_t dims[3] = {(uint64_t)width, (uint64_t)rows, (uint64_t)n};
  const uint64_t pitch[2] = {(uint64_t)width * 2, (uint64_t)width * rows * 2};
  const uint32_t b[3] = {64, (uint32_t)box, 1};
  return make_tensor_map_nd(tm, 3, ptr, dims, pitch, b);
}

#define QB_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

int64_t most_tiles(const AdaptersCall& c, int tn) { return c.T / tn + std::min<int64_t>(c.T, c.k.n); }

// 64-wide blocks between two emptyings of an accumulator.  Results in fp32, which are three parts: see AR_SEGMENT.
int ag_segment(int parts) { return parts == 3 ? 4 : 1 << 20; }

struct ShrinkWork { const Parts *in, *out; const __nv_bfloat16* W; bool kmajor, scaled; };
// u = x' A, du = s dv B^T, or both
int ag_shrink(const AdaptersCall& c, const Layout& l, int* status, const ShrinkWork* work, int sides, cudaStream_t st) {
  static std::atomic<bool> ready[64];
  AgShrinkMaps maps{};
  AgShrink p{};
  p.c = c; p.rows_there = l.rows; p.status = status; p.wait_limit = wait_limit_cycles();
  p.m_tiles = (c.k.r + 127) / 128; p.sides = sides;
  for (int i = 0; i < sides; ++i) p.np = std::max(p.np, work[i].in->np);
  // Rows of a tile: what takes the least time as counted in rows of 128 bytes: rounds of the units over the SMs, each its steps' operands
  // and about 1280 for beginning and end.  (Backward pass without dX, us, tiles of 128 / 64 / 32: 4096 -> 4096, rank 64, lambda 4, 20
  // adapters of 300 rows 75 / 82 / 87, three of 600 - / 41 / 39; lambda 1, six of 1100 123 / 145 / 161.)
  int sms = 0;
  QB_TRY(ag_sms(&sms));
  int64_t least = -1, blocks = 0;
  for (int i = 0; i < sides; ++i) blocks = std::max<int64_t>(blocks, (work[i].in->width + 63) / 64);
  for (int tn = 128; tn >= 32; tn /= 2) {
    const int64_t tiles = c.T / tn + 1, units = (tiles + std::min<int64_t>(c.k.n, tiles) / 2) * p.m_tiles * sides;
    const int64_t cost = (units + sms - 1) / sms * ((128 + p.np * tn) * blocks + 1280);
    if (least < 0 || cost < least) { least = cost; p.tn = tn; }
  }
  for (int i = 0; i < sides; ++i) {
    const ShrinkWork& w = work[i];
    const Parts& in = *w.in;
    p.side[i] = {in.np, in.width, w.kmajor, w.scaled, *w.out, in.p, w.W, in.ld};
    p.segment = ag_segment(w.out->np);
    QB_TRY(parts_map(&maps.side[i].rows, in, l.rows, p.tn));
    QB_TRY(parts_map(&maps.side[i].rows16, in, l.rows, 16));
    // A [P][r]: the contraction runs over its rows; B [r][Q]: along them
    QB_TRY(w.kmajor ? bank_map(&maps.side[i].w, w.W, in.width, c.k.r, c.k.n, 128) : bank_map(&maps.side[i].w, w.W, c.k.r, in.width, c.k.n, 64));
  }
  const size_t stage = AG_TILE + (size_t)p.np * p.tn * 128, table = ag_table_bytes(c.k.n);
  p.stages = (int)std::min<size_t>(8, (AG_SMEM - AG_BARS - table) / stage);
  return ag_launch(adapters_shrink_kernel, ready, maps, p, AG_THREADS, p.stages * stage + AG_BARS + table, most_tiles(c, p.tn) * p.m_tiles * sides, st);
}

// shared memory of the spread kernel without slabs
size_t as_fixed(int n, int np, int kb, int tn) {
  return (size_t)np * kb * tn * 128 + AS_RING * AG_TILE + (size_t)tn * 512 + AG_BARS + ag_table_bytes(n);
}
// rows of a tile: as many as leave room for five slabs, or for two where even the least do not; 0: none.  (7168 rows by 11008, rank 256, the
// whole call: tiles of 64 with five slabs 109 us, of 32 with eight 128.)
int as_rows(const BankView& k, int np) {
  for (int slabs : {5, 2})
    for (int tn = 64; tn >= 16; tn /= 2)
      if (as_fixed(k.n, np, (k.r + 63) / 64, tn) + (size_t)slabs * AS_SLAB <= (size_t)AG_SMEM) return tn;
  return 0;
}
// Y as [rows][pieces][elements of a piece]: a box is all pieces of 128 q by the rows of a slab.  The number of pieces, or 0 where
// such boxes cannot be had: rows that are no whole pieces, slabs that are less than a row.
int as_y_map(CUtensorMap* tm, const RowsView& y, int64_t T, int d, int lam, int* rc) {
  const int size = y.dtype == QBLORA_F32 ? 4 : 2, q = 128 * lam, whole = q * size, inner = q % 256 ? 128 : 256, n = q / inner;
  *rc = QBLORA_OK;
  if (whole > AS_SLAB || q % inner || d % inner || n > 256) return 0;
  *rc = make_tensor_map_rows(tm, y.dtype == QBLORA_F32, y.data, (uint64_t)inner, (uint64_t)(d / inner), (uint64_t)T, (uint64_t)inner * size,
                             (uint64_t)y.stride * size, (uint32_t)n, (uint32_t)(AS_SLAB / whole));
  return n;
}
// Y += s repeat(u B), or dX += repeat(du A^T) / lam
int ag_spread(const AdaptersCall& c, const Layout& l, int* status, const Parts& in, const __nv_bfloat16* W, int M, bool kmajor, const RowsView& y,
              int lam, bool forward, cudaStream_t st) {
  static std::atomic<bool> ready[9][64];
  AsMaps maps{};
  AgSpread p{};
  p.c = c; p.rows_there = l.rows; p.status = status; p.wait_limit = wait_limit_cycles();
  p.np = in.np; p.kb = (c.k.r + 63) / 64; p.tn = as_rows(c.k, in.np);
  const size_t fixed = as_fixed(c.k.n, p.np, p.kb, p.tn);
  p.slabs = (int)std::min<size_t>(8, (AG_SMEM - fixed) / AS_SLAB);
  p.segment = ag_segment(in.np); p.m_tiles = (M + 127) / 128; p.M = M; p.w_kmajor = kmajor; p.scaled = forward; p.y = y; p.lam = lam;
  p.u = in.p; p.u_ld = in.ld; p.W = W;
  p.factor = forward ? 1.0f : 1.0f / (float)lam;
  const int w = lam * (y.dtype == QBLORA_F32 ? 4 : 2);
  p.shift = -1;
  for (int i = 0; i < 31; ++i)
    if (w == 1 << i) p.shift = i;
  int rc = QBLORA_OK;
  p.boxes = as_y_map(&maps.y, y, c.T, M * lam, lam, &rc);
  QB_TRY(rc);
  QB_TRY(parts_map(&maps.in.rows, in, l.rows, p.tn));
  QB_TRY(parts_map(&maps.in.rows16, in, l.rows, 16));
  QB_TRY(kmajor ? bank_map(&maps.in.w, W, c.k.r, M, c.k.n, 128) : bank_map(&maps.in.w, W, M, c.k.r, c.k.n, 64));
  auto launch = [&](auto kernel, int form) {
    return ag_launch(kernel, ready[form], maps, p, AS_THREADS, fixed + (size_t)p.slabs * AS_SLAB, most_tiles(c, p.tn) * p.m_tiles, st);
  };
  if (y.dtype == QBLORA_F32) {
    if (p.shift < 0) return launch(adapters_spread_kernel<true, 0>, 0);
    if (p.shift >= 4) return launch(adapters_spread_kernel<true, 1>, 1);
    return p.shift == 3 ? launch(adapters_spread_kernel<true, 2>, 2) : launch(adapters_spread_kernel<true, 4>, 3);
  }
  if (p.shift < 0) return launch(adapters_spread_kernel<false, 0>, 4);
  if (p.shift >= 4) return launch(adapters_spread_kernel<false, 1>, 5);
  if (p.shift == 3) return launch(adapters_spread_kernel<false, 2>, 6);
  return p.shift == 2 ? launch(adapters_spread_kernel<false, 4>, 7) : launch(adapters_spread_kernel<false, 8>, 8);
}
int ag_grad(const AdaptersCall& c, const Layout& l, int* status, cudaStream_t st) {
  static std::atomic<bool> ready[64];
  AgGradMaps maps{};
  AgGrad p{};
  p.c = c; p.rows_there = l.rows; p.status = status; p.wait_limit = wait_limit_cycles();
  p.least = l.least; p.parts = l.parts; p.tickets = l.tickets; p.n_tickets = l.n_tickets;
  p.side[0] = {l.x.np, l.du.np, c.k.P, c.k.r, c.dA, l.x.p, l.du.p, l.x.ld, l.du.ld};
  p.side[1] = {l.u.np, l.dv.np, c.k.r, c.k.Q, c.dB, l.u.p, l.dv.p, l.u.ld, l.dv.ld};
  QB_TRY(parts_map(&maps.a[0], l.x, l.rows, 32));
  QB_TRY(parts_map(&maps.b[0], l.du, l.rows, 32));
  QB_TRY(parts_map(&maps.a[1], l.u, l.rows, 32));
  QB_TRY(parts_map(&maps.b[1], l.dv, l.rows, 32));
  const int64_t per = ag_tiles(c.k), most = per * (2 * c.k.n + 2 * (int64_t)c.T / l.least);
  return ag_launch(adapters_grad_kernel, ready, maps, p, AG_THREADS, AR_STAGES * AR_STAGE + AG_BARS + ag_table_bytes(c.k.n), most, st);
}

constexpr int kBackwardParts = 3;
int forward_parts(int y_dtype) { return y_dtype == QBLORA_F32 ? 3 : 2; }

}  // namespace

size_t tc_adapters_ws_bytes(const BankView& k, int64_t T, bool backward) { return ag_layout(k, T, backward, 3, nullptr).bytes; }

bool tc_adapters_sizes_ok(const BankView& k, int64_t T) {
  constexpr int most = (1 << 22) - 1;             // 128 q of a row in fp32 are below 2^31 bytes
  return k.l1 <= most && k.l2 <= most && k.r % 8 == 0 && k.Q % 8 == 0 && k.d_in % 8 == 0 && k.d_out % 8 == 0 && T + 15 * std::min<int64_t>(T, k.n) <= 0x7ffffff0 &&
         as_rows(k, 3) > 0;
}

bool tc_adapters_supported(const AdaptersCall& c) {
  if (!tc_adapters_sizes_ok(c.k, c.T) || !aligned16(c.k.A) || !aligned16(c.k.B)) return false;
  for (const RowsView* v : {&c.X, &c.Y, &c.dX})
    if (v->data && (!aligned16(v->data) || v->stride % 8)) return false;
  return aligned16(c.dA) && aligned16(c.dB);
}

int tc_adapters_fwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  const Layout l = ag_layout(c.k, c.T, false, forward_parts(c.Y.dtype), ws);
  int* status = reinterpret_cast<int*>(ws);
  AgPoolParams pool{};
  pool.c = c; pool.rows_there = l.rows; pool.status = status; pool.sources = 1;
  pool.src[0] = ag_source(c.X, c.k.d_in, c.k.l1, true, l.x);
  QB_TRY(ag_launch_pool(pool, l.rows, st));
  const ShrinkWork u{&l.x, &l.u, c.k.A, false, false};
  QB_TRY(ag_shrink(c, l, status, &u, 1, st));
  return ag_spread(c, l, status, l.u, c.k.B, c.k.Q, false, c.Y, c.k.l2, true, st);
}

int tc_adapters_bwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  const Layout l = ag_layout(c.k, c.T, true, kBackwardParts, ws);
  int* status = reinterpret_cast<int*>(ws);
  const bool grads = c.dA || c.dB;
  AgPoolParams pool{};
  pool.c = c; pool.rows_there = l.rows; pool.status = status; pool.sources = grads ? 2 : 1;
  pool.tickets = l.tickets; pool.n_tickets = grads ? l.n_tickets : 0;
  pool.per = (int)ag_tiles(c.k);      // (also where one of the two is wanted: the same sums)
  pool.least = l.least;
  pool.src[0] = ag_source(c.Y, c.k.d_out, c.k.l2, false, l.dv);
  if (grads) pool.src[1] = ag_source(c.X, c.k.d_in, c.k.l1, true, l.x);
  QB_TRY(ag_launch_pool(pool, l.rows, st));
  ShrinkWork work[2];
  int sides = 0;
  if (c.dX.data || c.dA) work[sides++] = {&l.dv, &l.du, c.k.B, true, true};
  if (c.dB) work[sides++] = {&l.x, &l.u, c.k.A, false, false};
  QB_TRY(ag_shrink(c, l, status, work, sides, st));
  if (c.dX.data) QB_TRY(ag_spread(c, l, status, l.du, c.k.A, c.k.P, true, c.dX, c.k.l1, false, st));
  if (grads) QB_TRY(ag_grad(c, l, status, st));
  return QBLORA_OK;
}

}  // namespace qb
