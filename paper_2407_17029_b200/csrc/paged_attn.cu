// Attention over the paged cache for the head sizes, page sizes and scales that paged_warp.cu and tc_attn.cu do not take.
//
// Mathematics.  A tile is ROWS = 16 WR rows of one request and one key head: row r is token r / G, query head r % G of the
// group that shares the key head, so shared keys are read once for all of them.  Keys are taken 64 at a time with the
// running maximum m and sum l of a softmax in base 2 (scores are scaled by scale * log2 e):
//   m' = max(m, s),  p = 2^(s - m'),  l' = l 2^(m - m') + sum p,  O' = O 2^(m - m') + P V,   out = O / l.
// Partial triples (m, l, O) over disjoint keys join by the same rule, in any grouping: first over the warps of a CTA, then
// over CTAs.
//
// What bounds it: the cache's bytes.  All key tiles of all items (request, key head, row tile) are put in one line and cut
// into equal shares, one per resident CTA, whatever the lengths; a CTA walks its share with a ring of cp.async stages that
// runs on across item borders, so loads never drain.  An item cut by a share's border leaves partial triples in the
// workspace; the CTA that finishes such an item last joins them, in share order, so results do not depend on timing.
// Rows beyond a request's keys are filled with zeros by the copy itself and never read from the cache.
//
// Layout: 64 keys x head size bf16 for K and V per stage, 16-byte chunks XOR-swizzled by the row, read by ldmatrix
// without bank conflicts.  mma.sync m16n8k16 (bf16, fp32 sums): the contraction is far below the tensor rate, and its
// register fragments let P go from scores to the second product without leaving registers.
// Measured with pages of 24 keys, D 128, 8 key heads of 4: 64 requests decoding over up to 8100 keys 309 us = 3.5 TB/s
// (paged_warp.cu with pages of 16: 187 us); 4 requests of 512 tokens behind 3584 keys 886 us = 145 TFLOP/s, bound by mma.sync and the
// work around it (tc_attn.cu with pages of 16: 138 us).  The same with D 96: 262 us (floor 129) and 888 us = 109 TFLOP/s; with D 256 and
// 4 key heads 402 us (floor 172) and 1824 us = 71 TFLOP/s (its forms spill 170 to 610 bytes).
//
// The weights are rounded to bf16 for their product with V, as mma.sync wants them; m, l, O and the parts are fp32.
#include <algorithm>
#include <atomic>

#include "mma_frag.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"

namespace qb {
namespace {

constexpr int PA_THREADS = 128;
constexpr int PA_TILE = 64;          // keys per stage
constexpr float PA_LN2 = 0.69314718055994530942f;

struct PaParams {
  AttnCall c;
  float scale2;         // scale * log2 e
  uint32_t div_page, div_group;   // 2^32 / divisor, rounded up (fast_div)
  uint32_t* counters;   // [grid] zeroed before the launch
  float* part_o;        // [2 * grid][ROWS][DP]
  float* part_ml;       // [2 * grid][ROWS][2]
};

__device__ __forceinline__ void pa_cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pa_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void pa_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Keys [lo, lo + 64 * tiles) that the rows of tile rt of a request see, at least one (possibly empty) tile.
// [all_lo, all_hi): the keys that every row of the tile sees.
struct PaRange { int lo, hi, tiles, all_lo, all_hi; };
template <int ROWS>
__device__ __forceinline__ PaRange pa_range(const PaParams& p, const ReqView& r, int rt) {
  const AttnCall& c = p.c;
  const int i0 = fast_div(rt * ROWS, c.G, p.div_group), i1 = min(r.n - 1, fast_div(rt * ROWS + ROWS - 1, c.G, p.div_group));
  PaRange k;
  k.hi = attn_hi(c, r.kv, r.kv - r.n + i1);
  k.lo = min(attn_lo(c, r.kv - r.n + i0), k.hi);
  k.tiles = max(1, (k.hi - k.lo + PA_TILE - 1) / PA_TILE);
  k.all_lo = attn_lo(c, r.kv - r.n + i1);
  k.all_hi = attn_hi(c, r.kv, r.kv - r.n + i0);
  return k;
}
__device__ __forceinline__ bool pa_mine(const ReqView& r) { return r.n > 0; }
template <int ROWS>
__device__ __forceinline__ int pa_row_tiles(const PaParams& p, const ReqView& r) { return (r.n * p.c.G + ROWS - 1) / ROWS; }
// key tiles of one key head of a request
template <int ROWS>
__device__ __forceinline__ int pa_head_units(const PaParams& p, const ReqView& r) {
  int u = 0;
  const int nrt = pa_row_tiles<ROWS>(p, r);
  for (int rt = 0; rt < nrt; ++rt) u += pa_range<ROWS>(p, r, rt).tiles;
  return u;
}

// A place in the line of key tiles.
template <int ROWS>
struct PaCursor {
  int b, h, rt, nrt, tile;
  ReqView r;
  PaRange k;
  __device__ __forceinline__ void enter_tile(const PaParams& p) { k = pa_range<ROWS>(p, r, rt); }
  __device__ __forceinline__ void next(const PaParams& p) {
    if (++tile < k.tiles) return;
    tile = 0;
    if (++rt == nrt) {
      rt = 0;
      if (++h == p.c.cache.kv_heads) {
        h = 0;
        do { ++b; if (b >= p.c.B) return; r = attn_request(p.c, b); } while (!pa_mine(r));
        nrt = pa_row_tiles<ROWS>(p, r);
      }
    }
    enter_tile(p);
  }
};

template <int DP, int WR, int STAGES>
struct PaShape {
  static constexpr int ROWS = 16 * WR, WK = 4 / WR;
  static constexpr int KV_BYTES = PA_TILE * DP * 2;          // K or V of a stage
  static constexpr int STAGE = 2 * KV_BYTES;
  static constexpr int SMEM = STAGES * STAGE;
};

template <int DP, int WR, int STAGES>
__global__ void __launch_bounds__(PA_THREADS) paged_attention_kernel(const __grid_constant__ PaParams p) {
  using Sh = PaShape<DP, WR, STAGES>;
  constexpr int ROWS = Sh::ROWS, WK = Sh::WK, CH = DP / 8, KPW = PA_TILE / WK;
  constexpr int NT = KPW / 8;                       // 8-key tiles of a warp
  extern __shared__ __align__(128) uint8_t pa_smem[];
  __shared__ long long s_off[2][PA_TILE];           // element offset of each key of the next tile to load; -1: zeros
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ long long s_scan[PA_THREADS / 32];
  __shared__ int s_start_b;
  __shared__ long long s_start_u;
  __shared__ int s_last;
  const AttnCall& c = p.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int wr = warp / WK, wk = warp % WK;
  const uint32_t smem = ptx::smem_u32(pa_smem);

  // ---- the line: units before each request, total, this CTA's share -----------------------------------------------
  const int per = (c.B + PA_THREADS - 1) / PA_THREADS;
  const int b_lo = min(tid * per, c.B), b_hi = min(b_lo + per, c.B);
  long long mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const ReqView r = attn_request(c, b);
    if (pa_mine(r)) mine += (long long)pa_head_units<ROWS>(p, r) * c.cache.kv_heads;
  }
  long long incl = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < PA_THREADS / 32; ++w) {
    if (w < warp) before += s_scan[w];
    total += s_scan[w];
  }
  incl += before;
  const long long shares = min((long long)gridDim.x, max(1LL, total));
  if ((long long)blockIdx.x >= shares) return;
  const long long u0 = total * blockIdx.x / shares, u1 = total * (blockIdx.x + 1) / shares;
  if (u0 >= u1) return;
  if (incl - mine <= u0 && u0 < incl) {   // one thread: the request that holds unit u0
    long long u = incl - mine;
    int b = b_lo;
    for (;; ++b) {
      const ReqView r = attn_request(c, b);
      if (!pa_mine(r)) continue;
      const long long n = (long long)pa_head_units<ROWS>(p, r) * c.cache.kv_heads;
      if (u0 < u + n) break;
      u += n;
    }
    s_start_b = b;
    s_start_u = u0 - u;
  }
  __syncthreads();

  PaCursor<ROWS> ld;
  ld.b = s_start_b;
  ld.r = attn_request(c, ld.b);
  ld.nrt = pa_row_tiles<ROWS>(p, ld.r);
  {
    const int hu = pa_head_units<ROWS>(p, ld.r);
    ld.h = (int)(s_start_u / hu);
    int rest = (int)(s_start_u - (long long)ld.h * hu);
    ld.rt = 0;
    ld.enter_tile(p);
    while (rest >= ld.k.tiles) { rest -= ld.k.tiles; ++ld.rt; ld.enter_tile(p); }
    ld.tile = rest;
  }
  PaCursor<ROWS> cu = ld;
  const long long units = u1 - u0;

  // ---- loads --------------------------------------------------------------------------------------------------------
  // thread < 64: page number of its key in the tile (or -1), and, when that number has arrived, the key's offset
  auto key_page = [&](const PaCursor<ROWS>& at) -> int {
    const int j = at.k.lo + at.tile * PA_TILE + tid;
    return j < at.k.hi ? __ldg(c.table + (long long)at.b * c.width + fast_div(j, c.cache.page_size, p.div_page)) : -1;
  };
  auto key_offset = [&](const PaCursor<ROWS>& at, int page) -> long long {
    const int j = at.k.lo + at.tile * PA_TILE + tid;
    if (j >= at.k.hi) return -1;
    if (page < 0 || page >= c.cache.n_pages) {
      atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
      return -1;
    }
    const int entry = j - fast_div(j, c.cache.page_size, p.div_page) * c.cache.page_size;
    return (long long)page * c.cache.ps + (long long)entry * c.cache.ts + (long long)at.h * c.cache.hs;
  };
  const int ch = tid % CH;                        // this thread's 16-byte column in K, V and Q rows
  const bool col = ch * 8 < c.D;
  const uint32_t my_dst = (uint32_t)((tid / CH) * DP * 2 + ((ch ^ ((tid / CH) & 7)) << 4));
  auto load_tile = [&](int stage, int buf) {
    const uint32_t sk = smem + stage * Sh::STAGE + my_dst;
#pragma unroll
    for (int i = 0; i < PA_TILE * CH / PA_THREADS; ++i) {
      // rows of one thread are PA_THREADS / CH apart; where that is 4 or less the swizzle changes from row to row
      constexpr int STEP = PA_THREADS / CH;
      const int row = tid / CH + i * STEP;
      const long long off = s_off[buf][row];
      const bool there = off >= 0 && col;
      const long long o = there ? off + ch * 8 : 0;
      const uint32_t d = STEP % 8 == 0 ? sk + i * STEP * DP * 2
                                       : smem + stage * Sh::STAGE + (uint32_t)(row * DP * 2 + ((ch ^ (row & 7)) << 4));
      pa_cp16(d, c.cache.k + o, there);
      pa_cp16(d + Sh::KV_BYTES, c.cache.v + o, there);
    }
  };

  // prologue: STAGES - 1 tiles on their way; from then on `ld` is the next tile to load and `page` its page numbers,
  // fetched one iteration before they are needed
  long long issued = 0;
  int buf = 0, page = tid < PA_TILE ? key_page(ld) : -1, ld_stage = 0;
  auto load_next = [&]() {
    load_tile(ld_stage, buf);
    if (++ld_stage == STAGES) ld_stage = 0;
    buf ^= 1;
    if (++issued < units) {
      ld.next(p);
      if (tid < PA_TILE) page = key_page(ld);
    }
  };
  for (int s = 0; s < STAGES - 1; ++s) {
    if (issued < units) {
      if (tid < PA_TILE) s_off[buf][tid] = key_offset(ld, page);
      __syncthreads();
      load_next();
    }
    pa_commit();
  }

  float o[DP / 8][4], m[2], l[2];
  uint32_t qf[DP / 16][4];
  bool first_segment = true;
  int r0 = 0, hi[2] = {0, 0}, lo[2] = {0, 0};

  int stage = -1;
  for (long long it = 0; it < units; ++it) {
    if (++stage == STAGES) stage = 0;
    if (issued < units && tid < PA_TILE) s_off[buf][tid] = key_offset(ld, page);
    pa_wait<STAGES - 2>();
    __syncthreads();
    if (issued < units) load_next();
    pa_commit();

    const uint32_t sk = smem + stage * Sh::STAGE, sv = sk + Sh::KV_BYTES;
    if (it == 0 || cu.tile == 0) {
      r0 = cu.rt * ROWS;
#pragma unroll
      for (int i = 0; i < 2; ++i) {                        // this lane's two rows: queries, and the keys they see
        const int gr = r0 + wr * 16 + (lane >> 2) + 8 * i, tok = fast_div(gr, c.G, p.div_group);
        const int pos = cu.r.kv - cu.r.n + min(tok, cu.r.n - 1);
        hi[i] = attn_hi(c, cu.r.kv, pos);
        lo[i] = attn_lo(c, pos);
        const uint32_t* q = reinterpret_cast<const uint32_t*>(c.q + (long long)(cu.r.t0 + tok) * c.q_ts +
                                                              (long long)(cu.h * c.G + gr - tok * c.G) * c.q_hs) + (lane & 3);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          qf[k][i] = tok < cu.r.n && 16 * k < c.D ? __ldg(q + 8 * k) : 0u;
          qf[k][2 + i] = tok < cu.r.n && 16 * k + 8 < c.D ? __ldg(q + 8 * k + 4) : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
      m[0] = m[1] = -INFINITY;
      l[0] = l[1] = 0.f;
    }

    // scores of this warp's KPW keys: fragment n covers keys 8 n .. 8 n + 7 (lane: rows lane / 4 and + 8, keys 2 (lane % 4) + {0, 1})
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
#pragma unroll
      for (int n2 = 0; n2 < NT / 2; ++n2) {
        // matrices: keys 0-7 chunk 2k, keys 0-7 chunk 2k+1, keys 8-15 chunk 2k, keys 8-15 chunk 2k+1
        const int row = wk * KPW + n2 * 16 + (lane & 7) + ((lane >> 4) << 3), chunk = 2 * k + ((lane >> 3) & 1);
        uint32_t kf[4];
        frag_ldm4(kf, sk + (uint32_t)(row * DP * 2 + ((chunk ^ (row & 7)) << 4)));
        frag_mma(s[2 * n2], qf[k], kf[0], kf[1]);
        frag_mma(s[2 * n2 + 1], qf[k], kf[2], kf[3]);
      }
    }
    // masks: only where some row does not see some key of the tile
    const int k0 = cu.k.lo + cu.tile * PA_TILE;
    const bool partial = k0 + PA_TILE > cu.k.all_hi || k0 < cu.k.all_lo;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] *= p.scale2;
    if (partial) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = k0 + wk * KPW + n * 8 + 2 * (lane & 3) + (e & 1);
          if (j >= hi[e >> 1] || j < lo[e >> 1]) s[n][e] = -INFINITY;
        }
    }
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float t = m[i];
#pragma unroll
      for (int n = 0; n < NT; ++n) t = fmaxf(t, fmaxf(s[n][2 * i], s[n][2 * i + 1]));
      t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
      t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
      const float base = t == -INFINITY ? 0.f : t;       // nothing seen yet: all weights are 2^-inf = 0
      f[i] = fast_exp2(m[i] - base);
      m[i] = t;
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        s[n][2 * i] = fast_exp2(s[n][2 * i] - base);
        s[n][2 * i + 1] = fast_exp2(s[n][2 * i + 1] - base);
        sum += s[n][2 * i] + s[n][2 * i + 1];
      }
      l[i] = l[i] * f[i] + sum;                          // this lane's part; joined over the quad at the end
    }
    if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
      for (int i = 0; i < DP / 8; ++i) { o[i][0] *= f[0]; o[i][1] *= f[0]; o[i][2] *= f[1]; o[i][3] *= f[1]; }
    }
    bool odd = false;                                    // a NaN or infinity in V of a tile with masked keys
#pragma unroll
    for (int k = 0; k < KPW / 16; ++k) {
      uint32_t a[4];
      a[0] = ptx::pack_bf16x2(s[2 * k][0], s[2 * k][1]);
      a[1] = ptx::pack_bf16x2(s[2 * k][2], s[2 * k][3]);
      a[2] = ptx::pack_bf16x2(s[2 * k + 1][0], s[2 * k + 1][1]);
      a[3] = ptx::pack_bf16x2(s[2 * k + 1][2], s[2 * k + 1][3]);
#pragma unroll
      for (int n2 = 0; n2 < DP / 16; ++n2) {
        const int row = wk * KPW + k * 16 + (lane & 15), chunk = 2 * n2 + (lane >> 4);
        uint32_t vf[4];
        frag_ldm4t(vf, sv + (uint32_t)(row * DP * 2 + ((chunk ^ (row & 7)) << 4)));
        if (partial) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            odd |= bf16x2_odd(vf[e]);
            vf[e] = bf16x2_clean(vf[e]);                     // 0 * NaN must not reach the rows that do not see the key
          }
        }
        frag_mma(o[2 * n2], a, vf[0], vf[1]);
        frag_mma(o[2 * n2 + 1], a, vf[2], vf[3]);
      }
    }
    if (partial && __any_sync(0xffffffffu, odd)) {
      // rare: give the values that were taken out back to the rows that see them
      for (int kk = 0; kk < KPW; ++kk) {
        const int row = wk * KPW + kk, j = k0 + row;
#pragma unroll
        for (int n = 0; n < DP / 8; ++n) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(pa_smem + stage * Sh::STAGE + Sh::KV_BYTES + row * DP * 2 +
                                                                ((n ^ (row & 7)) << 4) + 4 * (lane & 3));
          if (!bf16x2_odd(w)) continue;
          const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (j >= hi[i] || j < lo[i]) continue;
            if ((w & 0x7f80u) == 0x7f80u) o[n][2 * i] += v0;
            if ((w & 0x7f800000u) == 0x7f800000u) o[n][2 * i + 1] += v1;
          }
        }
      }
    }

    // ---- end of an item, or of this CTA's part of it ----------------------------------------------------------------
    const bool item_end = cu.tile + 1 == cu.k.tiles;
    if (item_end || it + 1 == units) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        if ((lane & 3) == 0) { s_m[warp][(lane >> 2) + 8 * i] = m[i]; s_l[warp][(lane >> 2) + 8 * i] = l[i]; }
      }
      __syncthreads();                                   // every warp has read the stage: it becomes scratch
      float* so = reinterpret_cast<float*>(pa_smem + stage * Sh::STAGE);   // [4][16][DP]
#pragma unroll
      for (int n = 0; n < DP / 8; ++n) {
        float* d = so + (warp * 16 + (lane >> 2)) * DP + n * 8 + 2 * (lane & 3);
        *reinterpret_cast<float2*>(d) = make_float2(o[n][0], o[n][1]);
        *reinterpret_cast<float2*>(d + 8 * DP) = make_float2(o[n][2], o[n][3]);
      }
      __syncthreads();
      const long long item_first = u0 + it - cu.tile, item_last = item_first + cu.k.tiles - 1;   // units of the item
      const bool whole = item_first >= u0 && item_last < u1;
      // a thread owns columns 4 x .. 4 x + 3 of rows y, y + step, ...
      constexpr int CW = DP / 4, STEP = PA_THREADS / CW > 0 ? PA_THREADS / CW : 1;
      const int x = tid % CW, y = tid / CW;
      const int slot = 2 * (int)blockIdx.x + (first_segment ? 0 : 1);
      for (int row = y; row < ROWS; row += STEP) {
        const int w0 = (row >> 4) * WK, rr = row & 15;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, s_m[w0 + w][rr]);
        const float base = M == -INFINITY ? 0.f : M;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float g = fast_exp2(s_m[w0 + w][rr] - base);
          L += s_l[w0 + w][rr] * g;
          const float4 v = *reinterpret_cast<const float4*>(so + ((w0 + w) * 16 + rr) * DP + 4 * x);
          acc.x += v.x * g; acc.y += v.y * g; acc.z += v.z * g; acc.w += v.w * g;
        }
        if (!whole) {
          *reinterpret_cast<float4*>(p.part_o + ((long long)slot * ROWS + row) * DP + 4 * x) = acc;
          if (x == 0) *reinterpret_cast<float2*>(p.part_ml + ((long long)slot * ROWS + row) * 2) = make_float2(M, L);
          continue;
        }
        const int gr = r0 + row, tok = fast_div(gr, c.G, p.div_group);
        if (tok >= cu.r.n || 4 * x >= c.D) continue;
        const int head = cu.h * c.G + gr - tok * c.G;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const uint2 out = make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
        *reinterpret_cast<uint2*>(c.out + (long long)(cu.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + 4 * x) = out;
        if (c.lse && x == 0) c.lse[(long long)(cu.r.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * PA_LN2;
      }
      if (!whole) {
        // shares first .. last hold parts of this item
        auto share_of = [&](long long u) {
          long long s_ = u * shares / total;
          while (total * (s_ + 1) / shares <= u) ++s_;
          while (total * s_ / shares > u) --s_;
          return (int)s_;
        };
        const int first = share_of(item_first), last = share_of(item_last);
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicAdd(p.counters + first, 1u) == (uint32_t)(last - first);
        __syncthreads();
        if (s_last) {
          __threadfence();
          // the item is the first share's last segment: its slot is 1 unless that share begins with the item
          const int slot0 = 2 * first + (total * first / shares == item_first ? 0 : 1);
          for (int row = y; row < ROWS; row += STEP) {
            const int gr = r0 + row, tok = fast_div(gr, c.G, p.div_group);
            if (tok >= cu.r.n) break;
            float M = -INFINITY;
            for (int q = first; q <= last; ++q)
              M = fmaxf(M, __ldcg(p.part_ml + ((long long)(q == first ? slot0 : 2 * q) * ROWS + row) * 2));
            const float base = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int q = first; q <= last; ++q) {
              const long long at = (long long)(q == first ? slot0 : 2 * q) * ROWS + row;
              const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + at * 2));
              const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * DP + 4 * x));
              const float g = fast_exp2(ml.x - base);
              L += ml.y * g;
              acc.x += v.x * g; acc.y += v.y * g; acc.z += v.z * g; acc.w += v.w * g;
            }
            if (4 * x >= c.D) continue;
            const int head = cu.h * c.G + gr - tok * c.G;
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const uint2 out = make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
            *reinterpret_cast<uint2*>(c.out + (long long)(cu.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + 4 * x) = out;
            if (c.lse && x == 0) c.lse[(long long)(cu.r.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * PA_LN2;
          }
        }
      }
      first_segment = false;
      // the scratch stage is refilled by the next iteration's load, behind its barrier
    }
    cu.next(p);
  }
  pa_wait<0>();
}

template <int DP, int WR, int STAGES>
int pa_launch(PaParams p, char* counters, char* scratch, cudaStream_t st) {
  using Sh = PaShape<DP, WR, STAGES>;
  static std::atomic<int> per_sm[64];   // resident CTAs per SM of this form, 0 = not asked yet
  int dev = 0, sms = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  auto kernel = paged_attention_kernel<DP, WR, STAGES>;
  int occ = per_sm[dev].load(std::memory_order_acquire);
  if (occ == 0) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
    QB_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kernel, PA_THREADS, Sh::SMEM));
    if (occ < 1) return QBLORA_ERR_CUDA;
    occ = std::min(occ, kPagedMaxPerSm);
    per_sm[dev].store(occ, std::memory_order_release);
  }
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  sms = std::min(sms, kPagedMaxSms);
  const int grid = sms * occ;
  p.counters = reinterpret_cast<uint32_t*>(counters);
  p.part_ml = reinterpret_cast<float*>(scratch);
  p.part_o = p.part_ml + (size_t)2 * kPagedMaxSms * kPagedMaxPerSm * Sh::ROWS * 2;
  kernel<<<grid, PA_THREADS, Sh::SMEM, st>>>(p);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

template <int DP>
int pa_launch_rows(const PaParams& p, int wr, char* counters, char* scratch, cudaStream_t st) {
  constexpr int S = DP == 64 ? 5 : 3;
  if (wr == 1) return pa_launch<DP, 1, S>(p, counters, scratch, st);
  if (wr == 2) return pa_launch<DP, 2, S>(p, counters, scratch, st);
  return pa_launch<DP, 4, S>(p, counters, scratch, st);
}

// Row tiles of 16, 32 or 64 rows.  The host knows rows only on average: G per new token, tokens / requests new tokens.
int pa_row_form(const AttnCall& c) {
  const int64_t mean = ((c.T + c.B - 1) / c.B) * c.G;
  return mean <= 16 ? 1 : mean <= 32 ? 2 : 4;
}

}  // namespace

size_t paged_attention_scratch_bytes(int head_dim) {
  // rows of partial results: 2 parts per share, 64-row tiles here, 16-row tiles in paged_warp.cu
  const int dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  const size_t here = (size_t)2 * kPagedMaxSms * kPagedMaxPerSm * 64, there = (size_t)2 * kPagedMaxShares * 16;
  return std::max(here * (dp + 2) * 4, there * (dp + 2) * 4 + kPagedMaxShares * sizeof(JoinCut));
}

int launch_paged_attention(const AttnCall& c, char* counters, char* scratch, cudaStream_t st) {
  PaParams p{};
  p.c = c;
  p.scale2 = c.scale * 1.4426950408889634f;
  p.div_page = fast_div_magic((uint32_t)c.cache.page_size);
  p.div_group = fast_div_magic((uint32_t)c.G);
  const int wr = pa_row_form(c);
  if (c.D <= 64) return pa_launch_rows<64>(p, wr, counters, scratch, st);
  if (c.D <= 128) return pa_launch_rows<128>(p, wr, counters, scratch, st);
  return pa_launch_rows<256>(p, wr, counters, scratch, st);
}

}  // namespace qb
