// Many adapters over one weight, forward, few rows per adapter (decoding): one launch.
//
// An item is up to 8 rows of one adapter and belongs to a cluster of 1 to 8 CTAs.  Each CTA pools its part of the rows' input and
// forms its part of the sum u = x' A; the parts are added over the cluster's shared memory; then each CTA has all of u and takes its
// share of the outputs, Y += s repeat(u B).
//
// What bounds it: with an adapter per request the adapters' bytes (200 requests of as many adapters, 5120 -> 5120, rank 256: 262 MB in 49
// us, 5.4 TB/s), with few requests latency (one token, 4096 -> 4096: 8 us: the plan, the rows, x', the sums over the cluster, one after
// another). A and B are read once per item.  Each warp has a ring of its own, steps of 16 by 64 weights brought by asynchronous copies, so
// no barrier lies on that way; loads straight into registers came to 3.7 TB/s, as a warp cannot wait for the older of two loads alone.
// The products are mma.sync.m16n8k16, 16 ranks (outputs) by 8 tokens: a tile of 128 ranks on the other path's tensor memory would want a
// tile of 16 tokens and a kernel to itself for each product (64 adapters of 4 rows, 4096 -> 11008, rank 256: 56 us against 32 here).  x'
// and u are two bf16 parts (three where Y is fp32), as in tc_adapters.cu.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "adapter_groups.cuh"
#include "mma_frag.cuh"
#include "tc_ptx.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int NR_THREADS = 256, NR_WARPS = 8, NR_ROWS = 8;
constexpr int NR_CHUNK = 512;                     // of the pooled input in shared memory at a time
constexpr int NR_MAX_RANK = 512;
constexpr int NR_BATCH = 2;                       // rows of Y that a lane has on their way
constexpr int NR_STEP = 2048;                     // bytes of a step's weights: 16 of the contraction by 64 ranks (outputs)
constexpr int NR_PART = NR_WARPS * NR_ROWS * (64 + 4) * 4;
// steps of a warp whose weights are on their way: with four, two CTAs share an SM
template <int NP> constexpr int NR_AHEAD = NP == 3 ? 6 : 4;

struct NrParams {
  AdaptersCall c;
  int shift, qpc;                                 // log2 of the bytes of one q of Y, q in 16 bytes; 0: no power of two
  int* status;
};

// Bytes of shared memory: the warps' weights, pooled input (later the products), partial sums of u, u.
struct NrLayout { int x, part, u, table, all; };
__host__ __device__ constexpr NrLayout nr_layout(int np, int r, int n) {
  NrLayout l{};
  l.x = NR_WARPS * NR_STEP * (np == 3 ? NR_AHEAD<3> : NR_AHEAD<2>);
  const int x = np * NR_ROWS * (NR_CHUNK + 8) * 2;
  l.part = l.x + (x > NR_PART ? x : NR_PART);
  l.u = l.part + NR_PART;                         // (at most eight sums of 64 ranks: more warps share a contraction where ranks are few)
  l.table = l.u + np * NR_ROWS * ((r + 63) / 64 * 64 + 8) * 2;
  l.all = l.table + 2 * (n + 1) * 4 + 127;
  return l;
}
static_assert(nr_layout(3, NR_MAX_RANK, kMaxAdapters).all <= 230 * 1024 && nr_layout(2, NR_MAX_RANK, kMaxAdapters).all <= 230 * 1024, "shared memory");

// A matrix [K][pitch] from rank (output) m on, of which the first M are there, and a warp's steps through its contraction: first, first +
// stride, ... < last.  A lane copies 16 bytes, chunk lane % 8, of rows lane / 8 + 0, 4, 8, 12 of a step; chunk c of row k lies at place c ^ (k % 8)
// of the row's 128 bytes.  What is not there becomes zeros, also behind an adapter's own rank.
struct NrSteps {
  const __nv_bfloat16* at;                        // of the lane, at the step that is copied next
  int64_t next, four;                             // elements from step to step; of four rows
  int rows, first, last, stride;                  // rows from the lane's first on
  bool in, all_in;
};
__device__ __forceinline__ NrSteps nr_steps(const __nv_bfloat16* W, int pitch, int K, int m, int M, int first, int last, int stride, int lane) {
  const int c = m + 8 * (lane & 7), k = lane >> 3;
  return {W + (int64_t)(first * 16 + k) * pitch + c, (int64_t)stride * 16 * pitch, (int64_t)4 * pitch, K - k, first, last, stride, c < M, m + 64 <= M};
}
__device__ __forceinline__ void nr_copy(NrSteps& w, int s, uint32_t stage, int lane) {
  if (s < w.last) {
    const int k = lane >> 3, c = lane & 7;
    const uint32_t to = stage + k * 128 + ((c ^ k) << 4), to4 = stage + k * 128 + ((c ^ k ^ 4) << 4);      // rows 4 and 12 further: to4
    const __nv_bfloat16 *f0 = w.at, *f1 = f0 + w.four, *f2 = f1 + w.four, *f3 = f2 + w.four;
    w.at += w.next;
    auto copy = [](uint32_t to, const __nv_bfloat16* from) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    };
    auto copy_if = [&](uint32_t to, const __nv_bfloat16* from, int row) {
      if (w.in && row < w.rows) copy(to, from);
      else asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
    };
    if (w.all_in && s * 16 + 12 < w.rows) {
      copy(to, f0); copy(to4 + 512, f1); copy(to + 1024, f2); copy(to4 + 1536, f3);
    } else {
      copy_if(to, f0, s * 16); copy_if(to4 + 512, f1, s * 16 + 4); copy_if(to + 1024, f2, s * 16 + 8); copy_if(to4 + 1536, f3, s * 16 + 12);
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
// the first steps' weights on their way
template <int AHEAD>
__device__ __forceinline__ void nr_ahead(NrSteps& w, uint32_t ring, int lane) {
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) nr_copy(w, w.first + i * w.stride, ring + i * NR_STEP, lane);
}

// d[tile] += the step's weights by the rows' parts; x: this lane's place in [part][8 rows][pitch] bf16, at the step's first column
template <int NP>
__device__ __forceinline__ void nr_step(float (&d)[4][4], uint32_t w, const __nv_bfloat16* x, int part) {
  uint32_t b[NP][2];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    b[p][0] = *reinterpret_cast<const uint32_t*>(x + p * part);
    b[p][1] = *reinterpret_cast<const uint32_t*>(x + p * part + 8);
  }
  uint32_t a[4][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) frag_ldm4t(a[t], w ^ (t * 32));
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int t = 0; t < 4; ++t) frag_mma(d[t], a[t], b[p][0], b[p][1]);
}
// All of w's steps, after nr_ahead; x: the rows at step 0.  NP = 3: emptied every 16 steps, as the tensor core's sums lose a little per step.
template <int NP>
__device__ __forceinline__ void nr_product(float (&sum)[4][4], NrSteps& w, uint32_t ring, const __nv_bfloat16* x, int pitch, int part, int lane) {
  constexpr int AHEAD = NR_AHEAD<NP>;
  // ldmatrix: lanes 8 i ... give the rows of matrix i; contraction 0..7 of ranks 0..7 and 8..15, then 8..15 of them
  const int k = (lane & 7) + 8 * (lane >> 4);
  const uint32_t mine = ring + k * 128 + ((((lane >> 3) & 1) ^ (k & 7)) << 4);
  const __nv_bfloat16* xl = x + (lane >> 2) * pitch + 2 * (lane & 3);
  float d[4][4];
  auto each = [&](auto&& f) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) f(d[t][e], sum[t][e]);
  };
  if (NP == 3) each([](float& x, float&) { x = 0.f; });
  int count = 0;
  uint32_t stage = 0;
  for (int s = w.first; s < w.last; s += w.stride) {
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
    __syncwarp();
    if constexpr (NP == 3) nr_step<NP>(d, mine + stage, xl + s * 16, part);
    else nr_step<NP>(sum, mine + stage, xl + s * 16, part);
    __syncwarp();
    nr_copy(w, s + AHEAD * w.stride, ring + stage, lane);
    if ((stage += NR_STEP) == AHEAD * NR_STEP) stage = 0;
    if (NP == 3 && ++count == 16) {
      each([](float& x, float& y) { y += x; x = 0.f; });
      count = 0;
    }
  }
  if (NP == 3) each([](float& x, float& y) { y += x; });
}
// this lane's sums to out[row][rank]
__device__ __forceinline__ void nr_put(const float (&d)[4][4], float* out, int pitch, int lane) {
  float* to = out + 2 * (lane & 3) * pitch + (lane >> 2);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    to[16 * t] = d[t][0];
    to[16 * t + pitch] = d[t][1];
    to[16 * t + 8] = d[t][2];
    to[16 * t + 8 + pitch] = d[t][3];
  }
}

template <int NP>
__device__ __forceinline__ void nr_store_parts(__nv_bfloat16* out, int part, float x) {
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const __nv_bfloat16 h = __float2bfloat16_rn(x);
    out[p * part] = h;
    x -= __bfloat162float(h);
  }
}

// What is not finite.  Where a factor is infinite, or a sum is, the smaller parts make NaN of it: the rest of an infinity is inf - inf, and a part that
// is zero or of the other sign meets an infinite weight.  So where u or a product has come out as NaN it is formed once more: u from x' whole,
// a product from u's first part, which is zero only where u is.  Out of line, as all that a call runs it fetches for the first time: 0.1 us a call;
// inline 0.3; the warp's steps once more through its ring 0.2 to 0.8.
// four ranks of u, at `to` in parts; A: the first of them
template <int NP>
__device__ __noinline__ void nr_mend_u(const AdaptersCall& c, int row, const __nv_bfloat16* A, __nv_bfloat16* to, int part) {
  for (int e = 0; e < 4; ++e) {
    if (!isnan(__bfloat162float(to[e]))) continue;
    const __nv_bfloat16 *x = static_cast<const __nv_bfloat16*>(c.X.data) + row * c.X.stride, *a = A + e;
    float sum = 0.f;
    for (int p = 0; p < c.k.P && !isnan(sum); ++p, a += c.k.r) {
      float mean = 0.f;
      for (int l = 0; l < c.k.l1; ++l) mean += __bfloat162float(*x++);
      sum = fmaf(mean / (float)c.k.l1, __bfloat162float(*a), sum);
    }
    nr_store_parts<NP>(to + e, part, sum);
  }
}
// A lane's products as nr_put has put them, of u's first part and steps first, first + stride ... of B.
__device__ __noinline__ void nr_mend_put(float* put, int pitch, const __nv_bfloat16* u, int u_pitch, const __nv_bfloat16* B, int Q, int q0, int r, int n,
                                         int first, int stride) {
  const int lane = threadIdx.x & 31;
  for (int i = 0; i < 16; ++i) {
    const int row = 2 * (lane & 3) + (i & 1), q = (i >> 1) * 8 + (lane >> 2);
    if (row >= n || q0 + q >= Q || !isnan(put[row * pitch + q])) continue;
    float sum = 0.f;
    for (int s = first * 16; s < r; s += stride * 16)
      for (int k = s; k < min(s + 16, r); ++k) sum = fmaf(__bfloat162float(u[row * u_pitch + k]), __bfloat162float(B[(int64_t)k * Q + q0 + q]), sum);
    put[row * pitch + q] = sum;
  }
}
// whether there is NaN among a lane's products of the first n rows
__device__ __forceinline__ bool nr_any_nan(const float (&d)[4][4], int n, int lane) {
  float any[2] = {0.f, 0.f};                      // rows 2 (lane % 4) and the next; two numbers by one instruction
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; e += 2)
      asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
          : "+f"(any[0]), "+f"(any[1]) : "f"(d[t][e]), "f"(d[t][e + 1]));
  const int row = 2 * (lane & 3);
  return (row < n && isnan(any[0])) || (row + 1 < n && isnan(any[1]));
}

// Columns [lo, hi) of x' of the rows, as parts, at out[p * part + row * pitch + column - lo].
template <int NP>
__device__ __forceinline__ void nr_pool(const AdaptersCall& c, const int* rows, int n, int lo, int hi, __nv_bfloat16* out, int pitch, int part) {
  const int lam = c.k.l1, width = hi - lo, tid = threadIdx.x;
  const float factor = 1.0f / (float)lam;
  auto source = [&](int row) { return static_cast<const __nv_bfloat16*>(c.X.data) + rows[row] * c.X.stride; };
  const int per = lam < 8 && (lam & (lam - 1)) == 0 ? 8 / lam : 1;          // columns of a 16-byte load
  if (per > 1 || lam % 8 == 0) {
    const int groups = (width + per - 1) / per, loads = per > 1 ? 1 : lam >> 3;
    for (int i = tid; i < n * groups; i += NR_THREADS) {
      const int row = i / groups, g = i - row * groups;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
      if (rows[row] >= 0) {
        // (columns come in whole loads: lo and the rows' length are multiples of 16 columns and 8 elements)
        const uint4* x = reinterpret_cast<const uint4*>(source(row) + ((int64_t)lo + (int64_t)g * per) * lam);
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int l = 0; l < loads; ++l) {
          const uint4 y = __ldg(x + l);
          const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) { sum[2 * e] += ag_low(w[e]); sum[2 * e + 1] += ag_high(w[e]); }
        }
        if (lam == 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = sum[e];
        } else {
          const float s2[4] = {sum[0] + sum[1], sum[2] + sum[3], sum[4] + sum[5], sum[6] + sum[7]};
          if (lam == 2) { v[0] = s2[0]; v[1] = s2[1]; v[2] = s2[2]; v[3] = s2[3]; }
          else {
            const float s4[2] = {s2[0] + s2[1], s2[2] + s2[3]};
            if (lam == 4) { v[0] = s4[0]; v[1] = s4[1]; }
            else v[0] = s4[0] + s4[1];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < per && g * per + e < width) nr_store_parts<NP>(out + row * pitch + g * per + e, part, v[e] * factor);
    }
  } else {
    for (int i = tid; i < n * width; i += NR_THREADS) {
      const int row = i / width, col = i - row * width;
      float sum = 0.f;
      if (rows[row] >= 0)
        for (int l = 0; l < lam; ++l) sum += __bfloat162float(source(row)[((int64_t)lo + col) * lam + l]);
      nr_store_parts<NP>(out + row * pitch + col, part, sum / (float)lam);
    }
  }
}

// One item: n rows (at most 8) of adapter a, entries j ... of the plan, by all CTAs of the cluster.
template <int NP, bool F32>
__device__ __forceinline__ void nr_item(const NrParams& p, const NrLayout& l, uint8_t* nr_smem, int a, int j, int n) {
  __shared__ int s_row[NR_ROWS];
  const AdaptersCall& c = p.c;
  const BankView& k = c.k;
  constexpr int AHEAD = NR_AHEAD<NP>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cs = (int)cluster_ctas(), rank = (int)cluster_ctarank();
  const int r_read = bank_rank(k, a), r16 = (r_read + 15) & ~15;
  if (tid < NR_ROWS) {
    const int row = tid < n ? __ldg(c.rows + j + tid) : -1;
    s_row[tid] = row < c.T ? row : -1;
  }
  const uint32_t ring = smem_u32(nr_smem) + warp * (AHEAD * NR_STEP);
  __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(nr_smem + l.x);
  float* part = reinterpret_cast<float*>(nr_smem + l.part);
  __nv_bfloat16* us = reinterpret_cast<__nv_bfloat16*>(nr_smem + l.u);
  constexpr int XP = NR_CHUNK + 8, XPART = NR_ROWS * XP;
  const int blocks = (r16 + 63) / 64, wide = blocks * 64 + 4, splits = NR_WARPS / blocks;

  // ---- u's part: ranks [64 mb, ...) by warps mb, the contraction's steps dealt out over the splits
  const __nv_bfloat16* A = k.A + (int64_t)a * k.P * k.r;
  const int steps = (k.P + 15) / 16, s_lo = (int)((long long)steps * rank / cs), s_hi = (int)((long long)steps * (rank + 1) / cs);
  const int mb = warp % blocks, split = warp / blocks;
  const bool mine = split < splits;
  float d[4][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f;
  for (int c0 = s_lo; c0 < s_hi; c0 += NR_CHUNK / 16) {
    const int c1 = min(s_hi, c0 + NR_CHUNK / 16);
    NrSteps w = nr_steps(A, k.r, k.P, mb * 64, r_read, c0 + split, c1, splits, lane);
    if (mine) nr_ahead<AHEAD>(w, ring, lane);
    __syncthreads();
    nr_pool<NP>(c, s_row, n, c0 * 16, min(c1 * 16, k.P), xs, XP, XPART);
    // columns behind the last of the contraction: their weights are zeros, but what lies here may be no number
    for (int i = tid; i < NP * n * 16; i += NR_THREADS) {
      const int col = k.P - c0 * 16 + i % 16;
      if (col < (c1 - c0) * 16) xs[i / 16 / n * XPART + i / 16 % n * XP + col] = __float2bfloat16_rn(0.f);
    }
    __syncthreads();
    if (mine) nr_product<NP>(d, w, ring, xs - c0 * 16, XP, XPART, lane);
  }
  if (mine) nr_put(d, part + split * NR_ROWS * wide + mb * 64, wide, lane);
  __syncthreads();
  if (splits > 1) {
    for (int i = tid; i < n * wide; i += NR_THREADS) {
      float x = part[i];
      for (int s = 1; s < splits; ++s) x += part[s * NR_ROWS * wide + i];
      part[i] = x;
    }
  }

  // ---- u: the cluster's parts, in order
  const int up = blocks * 64 + 8, upart = NR_ROWS * up;
  const __nv_bfloat16* B = k.B + (int64_t)a * k.r * k.Q;
  const int q_blocks = (k.Q + 63) / 64, own = rank < q_blocks ? (q_blocks - rank + cs - 1) / cs : 0;
  const int steps2 = r16 / 16;
  // kw warps share a block's contraction: as many as give the fewest rounds of steps, with two more a round for its end (20 blocks of 16 steps:
  // one warp each takes three rounds of 16, two warps each five of 8)
  int kw = 1, best = 0x7fffffff;
  for (int t = 1; t <= NR_WARPS; t *= 2) {
    const int cost = (own * t + NR_WARPS - 1) / NR_WARPS * ((steps2 + t - 1) / t + 2);
    if (cost < best) { best = cost; kw = t; }
  }
  const int team = warp / kw, sub = warp % kw, teams = NR_WARPS / kw;
  auto q0_of = [&](int b) { return (rank + b * cs) * 64; };
  auto b_steps = [&](int b) { return nr_steps(B, k.Q, r_read, q0_of(b), k.Q, sub, steps2, kw, lane); };
  NrSteps w2 = b_steps(team);
  if (team < own) nr_ahead<AHEAD>(w2, ring, lane);
  if (cs > 1) cluster_sync_all();
  else __syncthreads();
  const uint32_t remote = smem_u32(part);
  for (int i = tid; i < n * (r16 / 4); i += NR_THREADS) {
    const int row = i / (r16 / 4), col = 4 * (i - row * (r16 / 4));
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (cs > 1) {
      for (int s = 0; s < cs; ++s) {
        const float4 y = ld_cluster4(map_to_cta(remote + 4 * (row * wide + col), s));
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
    } else {
      x = *reinterpret_cast<const float4*>(part + row * wide + col);
    }
    // no ranks behind the slots' last one: there infinite inputs have met weights of zero
    if (col >= r_read) x = make_float4(0.f, 0.f, 0.f, 0.f);
    __nv_bfloat16* to = us + row * up + col;
    nr_store_parts<NP>(to, upart, x.x);
    nr_store_parts<NP>(to + 1, upart, x.y);
    nr_store_parts<NP>(to + 2, upart, x.z);
    nr_store_parts<NP>(to + 3, upart, x.w);
    if (__builtin_expect(isnan((x.x + x.y) + (x.z + x.w)), 0) && s_row[row] >= 0) nr_mend_u<NP>(c, s_row[row], A + col, to, upart);
  }
  if (cs > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");     // this CTA has read the others' parts
  __syncthreads();

  // ---- Y: blocks of 64 outputs of the pooled kind, in turn over the teams of kw warps
  float* vs = reinterpret_cast<float*>(nr_smem + l.x);  // [warp][row][64]
  const float scale = __ldg(k.s + a);
  constexpr int ES = F32 ? 4 : 2, E = 16 / ES, VP = 64 + 4;
  const int w_q = k.l2 * ES;                      // bytes of one q
  for (int b0 = 0; b0 < own; b0 += teams) {
    const int b = b0 + team;
    const bool there = b < own;
    const int q0 = there ? q0_of(b) : 0;
    // The team's lanes lie over the 16-byte chunks of a row, and over rows where these are few: a lane stays with its chunk, so that where its
    // products are is found once (found for each chunk of each row: 48 requests of 16 adapters 13.8 us, now 11.0).  The first rows' chunks
    // are on their way during the product.
    const int chunks = there ? min(64, k.Q - q0) * w_q / 16 : 0, lanes = kw * 32, l_team = sub * 32 + lane;
    const int over = chunks > 0 && chunks < lanes ? lanes / chunks : 1;              // rows beside one another
    const int row0 = over > 1 ? l_team / chunks : 0, ch0 = row0 < over ? l_team - row0 * chunks : chunks;
    char* y_base = static_cast<char*>(c.Y.data) + (int64_t)q0 * w_q;
    uint4 y[NR_BATCH];
    uint4* at[NR_BATCH];
    auto ask = [&](int ch, int row) {
#pragma unroll
      for (int u = 0; u < NR_BATCH; ++u) {
        const int y_row = row + u * over < n ? s_row[row + u * over] : -1;
        at[u] = nullptr;
        if (y_row >= 0) {
          at[u] = reinterpret_cast<uint4*>(y_base + y_row * c.Y.stride * ES) + ch;
          y[u] = *at[u];
        }
      }
    };
    if (ch0 < chunks) ask(ch0, row0);
    if (there) {
#pragma unroll
      for (int t = 0; t < 4; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f;
      nr_product<NP>(d, w2, ring, us, up, upart, lane);
      w2 = b_steps(b + teams);
      if (b + teams < own) nr_ahead<AHEAD>(w2, ring, lane);
      float* put = vs + warp * NR_ROWS * VP;
      nr_put(d, put, VP, lane);
      if (__builtin_expect(nr_any_nan(d, n, lane), 0)) nr_mend_put(put, VP, us, up, B, k.Q, q0, r_read, n, sub, kw);
    }
    if (kw > 1) __syncthreads();
    else __syncwarp();
    if (there) {
      // the sums of the team's parts and the factor on the way
      const float* v0 = vs + team * kw * NR_ROWS * VP;
      auto add = [&](auto form) {
        constexpr int QPC = decltype(form)::value, N = QPC ? QPC : E;                // different q of a chunk; 0: any
        for (int ch = ch0; ch < chunks; ch += lanes) {
          int q[N];
#pragma unroll
          for (int f = 0; f < N; ++f) q[f] = QPC == 1 ? (ch << 4) >> p.shift : QPC ? ch * QPC + f : (ch * E + f) / k.l2;
          for (int row = row0; row < n; row += NR_BATCH * over) {
            if (ch != ch0 || row != row0) ask(ch, row);
#pragma unroll
            for (int u = 0; u < NR_BATCH; ++u) {
              if (!at[u]) continue;
              const float* v = v0 + (row + u * over) * VP;
              float x[N];
#pragma unroll
              for (int f = 0; f < N; ++f) {
                x[f] = v[q[f]];
                for (int s = 1; s < kw; ++s) x[f] += v[s * NR_ROWS * VP + q[f]];
                x[f] *= scale;
              }
              uint32_t e[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                if constexpr (F32) e[f] = __float_as_uint(__uint_as_float(e[f]) + x[f * N / E]);
                else e[f] = pack_bf16x2(ag_low(e[f]) + x[2 * f * N / E], ag_high(e[f]) + x[(2 * f + 1) * N / E]);
              }
              *at[u] = make_uint4(e[0], e[1], e[2], e[3]);
            }
          }
        }
      };
      if (p.qpc == 1) add(std::integral_constant<int, 1>());
      else if (p.qpc == 2) add(std::integral_constant<int, 2>());
      else if (p.qpc == 4) add(std::integral_constant<int, 4>());
      else if (!F32 && p.qpc == 8) add(std::integral_constant<int, F32 ? 4 : 8>());
      else add(std::integral_constant<int, 0>());
    }
    if (kw > 1) __syncthreads();
    else __syncwarp();
  }
  if (cs > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // no CTA leaves while another reads its part
}

template <int NP, bool F32>
__global__ void __launch_bounds__(NR_THREADS, NP == 3 ? 1 : 2) adapters_rows_kernel(const __grid_constant__ NrParams p) {
  extern __shared__ __align__(16) uint8_t nr_raw[];
  uint8_t* nr_smem = nr_raw + (-smem_u32(nr_raw) & 127u);        // the places of nr_copy
  const AdaptersCall& c = p.c;
  const BankView& k = c.k;
  const NrLayout l = nr_layout(NP, k.r, k.n);
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && tid == 0) *p.status = QBLORA_OK;
  const AgGroups g = ag_groups<NR_THREADS>(c, reinterpret_cast<uint32_t*>(nr_smem + l.table), 0x7fffffffu, NR_ROWS);
  const int cs = (int)cluster_ctas();
  const uint32_t item = blockIdx.x / cs;
  if (item >= g.tile[g.kept]) return;             // (the whole cluster)
  const int a = ag_find(g.tile, g.kept, item), i0 = (int)(item - g.tile[a]) * NR_ROWS, j = plan_start(c, a) + i0;
  const int n = min(NR_ROWS, plan_start(c, a + 1) - j);
  if (bank_rank(k, a) == 0) return;
  nr_item<NP, F32>(p, l, nr_smem, a, j, n);
}

template <int NP, bool F32>
int nr_launch(const NrParams& p, int64_t items, int cs, cudaStream_t st) {
  static std::atomic<bool> ready[64];
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  auto kernel = adapters_rows_kernel<NP, F32>;
  if (!ready[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, nr_layout(NP, NR_MAX_RANK, kMaxAdapters).all));
    ready[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * cs));
  cfg.blockDim = dim3(NR_THREADS);
  cfg.dynamicSmemBytes = (size_t)nr_layout(NP, p.c.k.r, p.c.k.n).all;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)cs, 1, 1};
  cfg.attrs = attr; cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  count_launch();
  return QBLORA_OK;
}

}  // namespace

bool rows_adapters_supported(const AdaptersCall& c) {
  return c.k.r <= NR_MAX_RANK;
}

int rows_adapters_fwd(const AdaptersCall& c, int* status, cudaStream_t st) {
  NrParams p{};
  p.c = c; p.status = status;
  const int w = c.k.l2 * (c.Y.dtype == QBLORA_F32 ? 4 : 2);
  for (int i = 1; i < 31; ++i)
    if (w == 1 << i) {
      p.shift = i;
      p.qpc = i >= 4 ? 1 : 16 >> i;
    }
  // at most: an item for each adapter that begins, and one for each 8 rows
  const int64_t items = std::min<int64_t>(c.T, c.T / NR_ROWS + c.k.n);
  int sms = 0, dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  // Clusters as large as there is room for at once: two CTAs an SM, or one where their shared memory or registers are too many, less what the
  // GPCs have left over that does not make a cluster (six for each CTA above two, as measured).  How many items there are only the plan
  // knows; between this and twice as many.  (4096 -> 11008, rank 256, us by clusters of 1, 2, 4, 8.  bf16, one row each: 16 adapters 35, 21, 16, 14; 48:
  // 39, 23, 20, 27; 100: 47, 38, 47, 61; 200: 69, 77, 75, 110.  fp32, eight rows: 14 70, 40, 27, 19; 16 75, 42, 27, 35; 32 86, 48, 32, 62; seven
  // rows: 36 83, 47, 58, 62; three: 74 61, 41, 71, 81.)
  const int np = c.Y.dtype == QBLORA_F32 ? 3 : 2, fit = np == 2 && nr_layout(np, c.k.r, c.k.n).all <= 113 * 1024 ? 2 : 1;
  const int64_t likely = std::max<int64_t>(std::min(c.T, c.k.n), c.T / NR_ROWS);
  int cs = 8;
  while (cs > 1 && likely * cs > fit * sms - 6 * (cs - 2)) cs /= 2;
  return c.Y.dtype == QBLORA_F32 ? nr_launch<3, true>(p, items, cs, st) : nr_launch<2, false>(p, items, cs, st);
}

}  // namespace qb
