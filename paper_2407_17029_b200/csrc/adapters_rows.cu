// Many adapters over one weight, forward, few rows per adapter (decoding): one launch.
//
// An item is up to 16 rows of one adapter and belongs to a cluster of 1 to 8 CTAs.  Each CTA pools its part of the rows' input and
// forms its part of the sum u = x' A; the parts are added over the cluster's shared memory; then each CTA has all of u and takes its
// share of the outputs, Y += s repeat(u B).
//
// What bounds it: with an adapter per request the adapters' bytes, with few requests latency.  A and B are read once per item,
// straight from memory into the fragments of mma.sync.m16n8k16, whose 16 rows are ranks (outputs) and whose 8 columns are tokens:
// the memory's rows run along the ranks, so a lane takes 16 bytes (8 ranks) of four rows of the contraction, and one byte permutation per
// register makes the pairs that the MMA wants of them; which ranks make up the 16 rows of a tile is free.  No shared memory, no
// barrier lies on that way.  x' and u are two bf16 parts (three where Y is fp32), as in tc_adapters.cu.
#include <algorithm>
#include <atomic>

#include "adapter_groups.cuh"
#include "mma_frag.cuh"
#include "tc_ptx.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int NR_THREADS = 256, NR_WARPS = 8, NR_ROWS = 16;
constexpr int NR_CHUNK = 512;                     // of the pooled input in shared memory at a time
constexpr int NR_MAX_RANK = 512;

struct NrParams {
  AdaptersCall c;
  int most;                                       // rows of an adapter that is this kernel's
  int shift;                                      // log2 of the bytes of one q of Y, -1: no power of two
  int clear;
  int* status;
};

// Bytes of shared memory: pooled input (later the products), partial sums of u, u.
struct NrLayout { int x, part, u, table, all; };
__host__ __device__ inline NrLayout nr_layout(int np, int r, int n) {
  const int blocks = (r + 63) / 64;               // of 64 ranks; an adapter of fewer has more partial sums of each, eight blocks in all
  NrLayout l;
  l.x = 0;
  const int x = np * NR_ROWS * (NR_CHUNK + 8) * 2, v = NR_WARPS * NR_ROWS * 64 * 4;
  l.part = x > v ? x : v;
  l.u = l.part + (blocks > NR_WARPS ? blocks : NR_WARPS) * NR_ROWS * 64 * 4;
  l.table = l.u + np * NR_ROWS * (blocks * 64 + 8) * 2;
  l.all = l.table + 2 * (n + 1) * 4;
  return l;
}

// four rows k of 64 ranks (outputs) from m0 on: this lane's 8 from m0 + 8 (lane / 4) on
struct NrWeights { uint4 w[4]; };
__device__ __forceinline__ void nr_load(NrWeights& x, const __nv_bfloat16* W, int pitch, int k0, int K, int m, int M, int tig) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = k0 + 2 * tig + (i & 1) + 8 * (i >> 1);
    x.w[i] = k < K && m < M ? __ldg(reinterpret_cast<const uint4*>(W + (int64_t)k * pitch + m)) : make_uint4(0, 0, 0, 0);
  }
}
__device__ __forceinline__ uint32_t nr_word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// d[tile][n8] += the step's weights by the rows' parts; x: [part][16 rows][pitch] bf16 from the step's first column on
template <int NP, int N8>
__device__ __forceinline__ void nr_step(float (&d)[4][N8][4], const NrWeights& w, const __nv_bfloat16* x, int pitch, int part, int lane) {
  uint32_t b[NP][N8][2];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int n = 0; n < N8; ++n) {
      const __nv_bfloat16* row = x + p * part + (n * 8 + (lane >> 2)) * pitch + 2 * (lane & 3);
      b[p][n][0] = *reinterpret_cast<const uint32_t*>(row);
      b[p][n][1] = *reinterpret_cast<const uint32_t*>(row + 8);
    }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    // rows of the tile: ranks 8 (lane / 4) + 2 t and + 2 t + 1 of the 64
    const uint32_t k0 = nr_word(w.w[0], t), k1 = nr_word(w.w[1], t), k8 = nr_word(w.w[2], t), k9 = nr_word(w.w[3], t);
    const uint32_t a[4] = {__byte_perm(k0, k1, 0x5410), __byte_perm(k0, k1, 0x7632), __byte_perm(k8, k9, 0x5410), __byte_perm(k8, k9, 0x7632)};
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int n = 0; n < N8; ++n) frag_mma(d[t][n], a, b[p][n][0], b[p][n][1]);
  }
}
// Steps first, first + stride, ... < last of the contraction; w: the weights of the first AHEAD of them (nr_ahead).  NP = 3: emptied every
// 16 steps, as the tensor core's sums lose a little per step.
template <int NP, int N8, int AHEAD, class Rows>
__device__ __forceinline__ void nr_product(float (&sum)[4][N8][4], NrWeights (&w)[AHEAD], const __nv_bfloat16* W, int pitch, int K, int m, int M, int first,
                                           int last, int stride, int lane, Rows&& rows, int x_pitch, int part) {
  float d[4][N8][4];
  auto each = [&](auto&& f) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int n = 0; n < N8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(d[t][n][e], sum[t][n][e]);
  };
  if (NP == 3) each([](float& x, float&) { x = 0.f; });
  int count = 0;
  for (int s = first; s < last; s += AHEAD * stride) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int at = s + i * stride;
      if (at >= last) break;
      if constexpr (NP == 3) nr_step<NP, N8>(d, w[i], rows(at), x_pitch, part, lane);
      else nr_step<NP, N8>(sum, w[i], rows(at), x_pitch, part, lane);
      if (at + AHEAD * stride < last) nr_load(w[i], W, pitch, (at + AHEAD * stride) * 16, K, m, M, lane & 3);
    }
    if (NP == 3 && (count += AHEAD) >= 16) {
      each([](float& x, float& y) { y += x; x = 0.f; });
      count = 0;
    }
  }
  if (NP == 3) each([](float& x, float& y) { y += x; });
}
template <int AHEAD>
__device__ __forceinline__ void nr_ahead(NrWeights (&w)[AHEAD], const __nv_bfloat16* W, int pitch, int K, int m, int M, int first, int last, int stride, int lane) {
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (first + i * stride < last) nr_load(w[i], W, pitch, (first + i * stride) * 16, K, m, M, lane & 3);
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

// One item: n rows (at most 8 N8) of adapter a, entries j ... of the plan, by all CTAs of the cluster.  AHEAD: steps of 16 whose weights a
// warp has on their way, 2 KB each (two of them: 3.2 TB/s with an adapter per request).
template <int NP, int N8, int AHEAD, bool F32>
__device__ __forceinline__ void nr_item(const NrParams& p, const NrLayout& l, uint8_t* nr_smem, int a, int j, int n) {
  __shared__ int s_row[NR_ROWS];
  const AdaptersCall& c = p.c;
  const BankView& k = c.k;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, tig = lane & 3;
  const int cs = (int)cluster_ctas(), rank = (int)cluster_ctarank();
  const int r_read = bank_rank(k, a), r16 = (r_read + 15) & ~15;
  if (tid < NR_ROWS) {
    const int row = tid < n ? __ldg(c.rows + j + tid) : -1;
    s_row[tid] = row < c.T ? row : -1;
  }
  __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(nr_smem);
  float* part = reinterpret_cast<float*>(nr_smem + l.part);
  __nv_bfloat16* us = reinterpret_cast<__nv_bfloat16*>(nr_smem + l.u);
  constexpr int XP = NR_CHUNK + 8, XPART = NR_ROWS * XP;
  const int blocks = (r16 + 63) / 64, wide = blocks * 64, splits = blocks >= NR_WARPS ? 1 : NR_WARPS / blocks;

  // ---- u's part: ranks [64 mb, ...) by warps mb, the contraction's steps dealt out over the splits
  const __nv_bfloat16* A = k.A + (int64_t)a * k.P * k.r;
  const int steps = (k.P + 15) / 16, s_lo = (int)((long long)steps * rank / cs), s_hi = (int)((long long)steps * (rank + 1) / cs);
  const int mb = warp % blocks, split = warp / blocks;
  const bool mine = split < splits;
  const int m = mb * 64 + 8 * (lane >> 2);
  float d[4][N8][4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < N8; ++e) d[t][e][0] = d[t][e][1] = d[t][e][2] = d[t][e][3] = 0.f;
  for (int c0 = s_lo; c0 < s_hi; c0 += NR_CHUNK / 16) {
    const int c1 = min(s_hi, c0 + NR_CHUNK / 16);
    NrWeights w[AHEAD];
    if (mine) nr_ahead<AHEAD>(w, A, k.r, k.P, m, r_read, c0 + split, c1, splits, lane);
    __syncthreads();
    nr_pool<NP>(c, s_row, n, c0 * 16, min(c1 * 16, k.P), xs, XP, XPART);
    // columns behind the last of the contraction: their weights are zeros, but what lies here may be no number
    for (int i = tid; i < NP * n * 16; i += NR_THREADS) {
      const int col = k.P - c0 * 16 + i % 16;
      if (col < (c1 - c0) * 16) xs[i / 16 / n * XPART + i / 16 % n * XP + col] = __float2bfloat16_rn(0.f);
    }
    __syncthreads();
    if (mine)
      nr_product<NP, N8, AHEAD>(d, w, A, k.r, k.P, m, r_read, c0 + split, c1, splits, lane, [&](int s) { return xs + (s - c0) * 16; }, XP, XPART);
  }
  if (mine) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < N8; ++e) {
        float* to = part + (split * NR_ROWS + e * 8 + 2 * tig) * wide + m + 2 * t;
        *reinterpret_cast<float2*>(to) = make_float2(d[t][e][0], d[t][e][2]);
        *reinterpret_cast<float2*>(to + wide) = make_float2(d[t][e][1], d[t][e][3]);
      }
  }
  __syncthreads();
  if (splits > 1) {
    for (int i = tid; i < n * wide; i += NR_THREADS) {
      float x = part[i];
      for (int s = 1; s < splits; ++s) x += part[s * NR_ROWS * wide + i];
      part[i] = x;
    }
  }

  // ---- u: the cluster's parts, in order
  const int up = wide + 8, upart = NR_ROWS * up;
  const __nv_bfloat16* B = k.B + (int64_t)a * k.r * k.Q;
  const int q_blocks = (k.Q + 63) / 64, own = rank < q_blocks ? (q_blocks - rank + cs - 1) / cs : 0;
  const int steps2 = r16 / 16;
  int kw = 1;                                     // warps that share a block's contraction
  while (kw * 2 * own <= NR_WARPS && kw * 2 <= steps2) kw *= 2;
  const int team = warp / kw, sub = warp % kw, teams = NR_WARPS / kw;
  auto q0_of = [&](int b) { return (rank + b * cs) * 64; };
  NrWeights w2[AHEAD];
  if (team < own) nr_ahead<AHEAD>(w2, B, k.Q, r_read, q0_of(team) + 8 * (lane >> 2), k.Q, sub, steps2, kw, lane);
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
    __nv_bfloat16* to = us + row * up + col;
    nr_store_parts<NP>(to, upart, x.x);
    nr_store_parts<NP>(to + 1, upart, x.y);
    nr_store_parts<NP>(to + 2, upart, x.z);
    nr_store_parts<NP>(to + 3, upart, x.w);
  }
  if (cs > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");     // this CTA has read the others' parts
  __syncthreads();

  // ---- Y: blocks of 64 outputs of the pooled kind, in turn over the teams of kw warps
  float* vs = reinterpret_cast<float*>(nr_smem);  // [warp][row][64]
  const float scale = __ldg(k.s + a);
  constexpr int ES = F32 ? 4 : 2, E = 16 / ES;
  const int w_q = k.l2 * ES;                      // bytes of one q
  for (int b0 = 0; b0 < own; b0 += teams) {
    const int b = b0 + team;
    const bool there = b < own;
    const int q0 = there ? q0_of(b) : 0;
    if (there) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < N8; ++e) d[t][e][0] = d[t][e][1] = d[t][e][2] = d[t][e][3] = 0.f;
      nr_product<NP, N8, AHEAD>(d, w2, B, k.Q, r_read, q0 + 8 * (lane >> 2), k.Q, sub, steps2, kw, lane, [&](int s) { return us + s * 16; }, up, upart);
      if (b + teams < own) nr_ahead<AHEAD>(w2, B, k.Q, r_read, q0_of(b + teams) + 8 * (lane >> 2), k.Q, sub, steps2, kw, lane);
      float* v = vs + warp * NR_ROWS * 64;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < N8; ++e) {
          float* to = v + (e * 8 + 2 * tig) * 64 + 8 * (lane >> 2) + 2 * t;
          *reinterpret_cast<float2*>(to) = make_float2(d[t][e][0], d[t][e][2]);
          *reinterpret_cast<float2*>(to + 64) = make_float2(d[t][e][1], d[t][e][3]);
        }
    }
    if (kw > 1) __syncthreads();
    else __syncwarp();
    if (there) {
      // whole rows' 16-byte chunks; the sums of the team's parts and the factor on the way
      const int chunks = min(64, k.Q - q0) * w_q / 16;
      const float* v0 = vs + team * kw * NR_ROWS * 64;
      for (int i = sub * 32 + lane; i < n * chunks; i += kw * 32) {
        const int row = i / chunks, ch = i - row * chunks, y_row = s_row[row];
        if (y_row < 0) continue;
        uint4* at = reinterpret_cast<uint4*>(static_cast<char*>(c.Y.data) + y_row * c.Y.stride * ES + (int64_t)q0 * w_q) + ch;
        const uint4 y = *at;
        uint32_t e[4] = {y.x, y.y, y.z, y.w};
        float x[E];
        int last = -1;
        float now = 0.f;
#pragma unroll
        for (int f = 0; f < E; ++f) {
          const int q = p.shift >= 0 ? (ch * 16 + f * ES) >> p.shift : (ch * E + f) / k.l2;
          if (q != last) {
            now = 0.f;
            for (int s = 0; s < kw; ++s) now += v0[(s * NR_ROWS + row) * 64 + q];
            last = q;
          }
          x[f] = now * scale;
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          if constexpr (F32) e[f] = __float_as_uint(__uint_as_float(e[f]) + x[f]);
          else e[f] = pack_bf16x2(ag_low(e[f]) + x[2 * f], ag_high(e[f]) + x[2 * f + 1]);
        }
        *at = make_uint4(e[0], e[1], e[2], e[3]);
      }
    }
    if (kw > 1) __syncthreads();
    else __syncwarp();
  }
  if (cs > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // no CTA leaves while another reads its part
}

template <int NP, bool F32>
__global__ void __launch_bounds__(NR_THREADS, NP == 3 ? 1 : 2) adapters_rows_kernel(const __grid_constant__ NrParams p) {
  extern __shared__ __align__(16) uint8_t nr_smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const AdaptersCall& c = p.c;
  const BankView& k = c.k;
  const NrLayout l = nr_layout(NP, k.r, k.n);
  const int tid = threadIdx.x;
  if (p.clear && blockIdx.x == 0 && tid == 0) *p.status = QBLORA_OK;
  const AgGroups g = ag_groups<NR_THREADS>(c, reinterpret_cast<uint32_t*>(nr_smem + l.table), 0x7fffffffu, NR_ROWS, 0, (uint32_t)p.most);
  const int cs = (int)cluster_ctas();
  const uint32_t item = blockIdx.x / cs;
  if (item >= g.tile[g.kept]) return;             // (the whole cluster)
  const int a = ag_find(g.tile, g.kept, item), i0 = (int)(item - g.tile[a]) * NR_ROWS, j = plan_start(c, a) + i0;
  const int n = min(NR_ROWS, plan_start(c, a + 1) - j);
  if (bank_rank(k, a) == 0) return;
  if (n <= 8) nr_item<NP, 1, NP == 3 ? 6 : 4, F32>(p, l, nr_smem, a, j, n);
  else nr_item<NP, 2, NP == 3 ? 4 : 3, F32>(p, l, nr_smem, a, j, n);
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
  return c.k.r <= NR_MAX_RANK && nr_layout(c.Y.dtype == QBLORA_F32 ? 3 : 2, c.k.r, c.k.n).all <= 230 * 1024;
}

int rows_adapters_fwd(const AdaptersCall& c, int most, bool first, int* status, cudaStream_t st) {
  NrParams p{};
  p.c = c; p.most = most; p.clear = first; p.status = status;
  const int w = c.k.l2 * (c.Y.dtype == QBLORA_F32 ? 4 : 2);
  p.shift = -1;
  for (int i = 0; i < 31; ++i)
    if (w == 1 << i) p.shift = i;
  // at most: an item for each adapter that begins, and one for each 16 rows
  const int64_t tiles = std::min<int64_t>(c.T / NR_ROWS, (int64_t)c.k.n * (most / NR_ROWS));
  const int64_t items = std::min<int64_t>(c.T, tiles + c.k.n);
  int sms = 0, dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  int cs = 8;
  while (cs > 1 && items * cs > 2 * sms) cs /= 2;
  return c.Y.dtype == QBLORA_F32 ? nr_launch<3, true>(p, items, cs, st) : nr_launch<2, false>(p, items, cs, st);
}

}  // namespace qb
