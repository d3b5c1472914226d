// Attention over the paged cache for few rows per key head (decoding, drafted tokens): the form that streams the cache
// with TMA.  Head sizes 64 and 128, pages that fit its tiles; paged_attn.cu takes the rest.
//
// Mathematics as in paged_attn.cu: a running softmax in base 2 over row tiles of 16 MT rows (tokens x query heads that share
// a key head); partial triples (maximum, sum, weighted values) over disjoint keys join in any grouping.
//
// What bounds it: the cache's bytes, so each warp is made to need little else.  All key tiles of all items (request,
// key head, row tile) are put in one line and cut into equal shares, one per WARP.  A warp streams its share through a ring
// of its own -- lane i issues box i of a tile as the ring's slot becomes free, nothing waits for another warp -- and
// does both products for the whole tile, so a tile costs a warp one wait, one maximum and one rescale.  (With the four
// warps of a CTA sharing each tile, a 64-key tile cost 2160 warp instructions instead of about 500, and the kernel
// was bound by them: 4.5 TB/s.)  In flight per SM: 4 warps x 3 slots x 16 KB.
//
// An item cut by a share's border leaves partial triples in the workspace; when all warps of a CTA are done it joins
// the items that lie within its own shares, and of the items that reach into other CTAs those that it finished last, in share order:
// results do not depend on timing.
//
// Entries behind a request's keys: whole pages are asked for at a page number past the cache, which TMA fills with zeros;
// the rest of the last page is masked (scores set to -infinity, V set to zero in shared memory).
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "mma_frag.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"
#include "tc_small.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int PW_WARPS = 4, PW_THREADS = PW_WARPS * 32;
constexpr int PW_STAGES = 3;
constexpr float PW_LN2 = 0.69314718055994530942f;

template <int D, int MT>
struct PwShape {
  static constexpr int ROWS = 16 * MT;
  static constexpr int KT = D == 64 ? 64 : 32;            // keys per tile: 16 KB of K and V
  static constexpr int KV_BYTES = KT * D * 2;
  static constexpr int STAGE = 2 * KV_BYTES;
  static constexpr int Q_BYTES = MT == 1 ? 0 : ROWS * D * 2;   // per warp; one row tile's queries stay in registers
  static constexpr int WARP_BYTES = PW_STAGES * STAGE + Q_BYTES;
  static constexpr int SMEM = PW_WARPS * WARP_BYTES + 1024;
};

struct PwParams {
  AttnCall c;
  float scale2;              // scale * log2 e
  int narrow_rows;           // requests with more rows than this belong to the tcgen05 kernel
  int min_units;             // a share has at least so many key tiles
  int box_keys;              // keys per TMA box: min(page_size, KT)
  uint32_t div_page, div_group;
  uint32_t zero;             // 0, but not to the compiler
  long long wait_limit;
  uint32_t* counters;        // [grid], zeroed
  float* part_o;             // [2 * shares][ROWS][D]
  float* part_ml;            // [2 * shares][ROWS][2]
};

struct PwRange { int lo, hi, tiles, all_lo, all_hi; };
template <int ROWS, int KT>
__device__ __forceinline__ PwRange pw_range(const PwParams& p, const ReqView& r, int rt) {
  const AttnCall& c = p.c;
  const int i0 = fast_div(rt * ROWS, c.G, p.div_group), i1 = min(r.n - 1, fast_div(rt * ROWS + ROWS - 1, c.G, p.div_group));
  const int p0 = r.kv - r.n;
  PwRange k;
  k.hi = attn_hi(c, r.kv, p0 + i1);
  k.lo = min(attn_lo(c, p0 + i0), k.hi) & ~(KT - 1);
  k.tiles = max(1, (k.hi - k.lo + KT - 1) / KT);
  k.all_lo = attn_lo(c, p0 + i1);
  k.all_hi = attn_hi(c, r.kv, p0 + i0);
  return k;
}
__device__ __forceinline__ bool pw_mine(const PwParams& p, const ReqView& r) {
  return r.n > 0 && (long long)r.n * p.c.G <= p.narrow_rows;
}
template <int ROWS>
__device__ __forceinline__ int pw_row_tiles(const PwParams& p, const ReqView& r) { return (r.n * p.c.G + ROWS - 1) / ROWS; }
template <int ROWS, int KT>
__device__ __forceinline__ int pw_head_units(const PwParams& p, const ReqView& r) {
  int u = 0;
  const int nrt = pw_row_tiles<ROWS>(p, r);
  for (int rt = 0; rt < nrt; ++rt) u += pw_range<ROWS, KT>(p, r, rt).tiles;
  return u;
}

template <int ROWS, int KT>
struct PwCursor {
  int b, h, rt, nrt, tile;
  ReqView r;
  PwRange k;
  __device__ __forceinline__ void next(const PwParams& p) {
    if (++tile < k.tiles) return;
    tile = 0;
    if (++rt == nrt) {
      rt = 0;
      if (++h == p.c.cache.kv_heads) {
        h = 0;
        do { ++b; if (b >= p.c.B) return; r = attn_request(p.c, b); } while (!pw_mine(p, r));
        nrt = pw_row_tiles<ROWS>(p, r);
      }
    }
    k = pw_range<ROWS, KT>(p, r, rt);
  }
};

// An item that the shares of a CTA cut.
struct PwCut { int valid, b, h, rt, first_cta, last_cta; long long first_unit; int tiles; };

template <int D, int MT>
__global__ void __launch_bounds__(PW_THREADS, 1)
paged_warp_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ PwParams p) {
  using Sh = PwShape<D, MT>;
  constexpr int ROWS = Sh::ROWS, KT = Sh::KT, HALVES = D / 64, NT = KT / 8;
  using Cursor = PwCursor<ROWS, KT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[PW_WARPS * PW_STAGES];
  __shared__ long long s_scan[PW_WARPS];
  __shared__ int s_start_b[PW_WARPS];
  __shared__ long long s_start_u[PW_WARPS];
  __shared__ PwCut s_cut[PW_WARPS + 1];
  __shared__ int s_ready[PW_WARPS + 1];
  const AttnCall& c = p.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t ring = base + warp * (PW_STAGES * Sh::STAGE);
  const uint32_t sq = base + PW_WARPS * PW_STAGES * Sh::STAGE + warp * Sh::Q_BYTES;
  const uint32_t full = smem_u32(s_full + warp * PW_STAGES);

  // the tcgen05 kernel of the same call reads nothing of this one's and may start as SMs become free
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (lane == 0) {
    for (int s = 0; s < PW_STAGES; ++s) mbar_init(full + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_cut[warp + 1].valid = 0;
    if (warp == 0) s_cut[0].valid = 0;
  }

  // ---- the line: units before each request, all units, the shares -----------------------------------------------------
  const int per = (c.B + PW_THREADS - 1) / PW_THREADS;
  const int b_lo = min(tid * per, c.B), b_hi = min(b_lo + per, c.B);
  long long mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const ReqView r = attn_request(c, b);
    if (pw_mine(p, r)) mine += (long long)pw_head_units<ROWS, KT>(p, r) * c.cache.kv_heads;
  }
  long long incl = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < PW_WARPS; ++w) {
    if (w < warp) incl += s_scan[w];
    total += s_scan[w];
  }
  const long long shares = min((long long)gridDim.x * PW_WARPS, max(1LL, total / p.min_units));
  auto share_begin = [&](long long g) { return total * g / shares; };
  const long long g0 = (long long)blockIdx.x * PW_WARPS;
  if (total == 0 || g0 >= shares) return;
  for (int w = 0; w < PW_WARPS; ++w) {
    if (g0 + w >= shares) break;
    const long long u0 = share_begin(g0 + w);
    if (incl - mine <= u0 && u0 < incl) {   // one thread of the CTA: the request that holds unit u0
      long long u = incl - mine;
      int b = b_lo;
      for (;; ++b) {
        const ReqView r = attn_request(c, b);
        if (!pw_mine(p, r)) continue;
        const long long n = (long long)pw_head_units<ROWS, KT>(p, r) * c.cache.kv_heads;
        if (u0 < u + n) break;
        u += n;
      }
      s_start_b[w] = b;
      s_start_u[w] = u0 - u;
    }
  }
  __syncthreads();
  const long long g = g0 + warp;
  const long long u0 = g < shares ? share_begin(g) : 0, u1 = g < shares ? share_begin(g + 1) : 0;
  const int units = (int)(u1 - u0);

  bool ok = true;
  int odd_pages = 0;
  if (units > 0) {
    Cursor ld;
    ld.b = s_start_b[warp];
    ld.r = attn_request(c, ld.b);
    ld.nrt = pw_row_tiles<ROWS>(p, ld.r);
    {
      const int hu = pw_head_units<ROWS, KT>(p, ld.r);
      ld.h = (int)(s_start_u[warp] / hu);
      int rest = (int)(s_start_u[warp] - (long long)ld.h * hu);
      ld.rt = 0;
      ld.k = pw_range<ROWS, KT>(p, ld.r, 0);
      while (rest >= ld.k.tiles) { rest -= ld.k.tiles; ++ld.rt; ld.k = pw_range<ROWS, KT>(p, ld.r, ld.rt); }
      ld.tile = rest;
    }
    Cursor cu = ld;

    // ---- loads: lane i issues box i: (K or V, half of the head, run of keys) ------------------------------------------
    const int runs = KT / p.box_keys;                 // boxes along the keys
    const int n_boxes = 2 * HALVES * runs;            // at most 32
    const int my_run = lane / (2 * HALVES), my_half = (lane >> 1) % HALVES, my_kv = lane & 1;
    const uint32_t my_dst = (uint32_t)(my_kv * Sh::KV_BYTES + my_half * (KT * 128) + my_run * p.box_keys * 128);
    auto lookup = [&](int& entry) -> int {            // page of this lane's box; past the cache: zeros
      const int key = ld.k.lo + ld.tile * KT + my_run * p.box_keys;
      entry = 0;
      if (lane >= n_boxes || key >= ld.k.hi) return c.cache.n_pages;
      const int j = fast_div(key, c.cache.page_size, p.div_page);
      entry = key - j * c.cache.page_size;
      return __ldg(c.table + (long long)ld.b * c.width + j);
    };
    int issued = 0, entry, page = lookup(entry), st_ld = 0;
    auto issue = [&](uint32_t dep) {
      if (page < 0 || page > c.cache.n_pages) { odd_pages = 1; page = c.cache.n_pages; }
      const bool past = page == c.cache.n_pages && ld.k.lo + ld.tile * KT + my_run * p.box_keys < ld.k.hi;
      if (lane < n_boxes && past) odd_pages = 1;
      if (lane == 0) mbar_arrive_expect_tx(full + 8 * st_ld, Sh::STAGE);
      __syncwarp();
      if (lane < n_boxes)
        tma_load_4d(ring + st_ld * Sh::STAGE + my_dst + dep, my_kv ? &tm_v : &tm_k, full + 8 * st_ld, my_half * 64, entry, ld.h, page);
      if (++st_ld == PW_STAGES) st_ld = 0;
      if (++issued < units) { ld.next(p); page = lookup(entry); }
    };
    for (int s = 0; s < PW_STAGES && issued < units; ++s) issue(0);

    // ldmatrix offsets of this lane: row and swizzled chunk pair i of a 128-byte span, for K (as it lies) and V (transposed)
    uint32_t xk[4], xv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rk = (lane & 7) + ((lane >> 4) << 3), rv = lane & 15;
      xk[i] = (uint32_t)(rk * 128 + (((2 * i + ((lane >> 3) & 1)) ^ (rk & 7)) << 4));
      xv[i] = (uint32_t)(rv * 128 + (((2 * i + (lane >> 4)) ^ (rv & 7)) << 4));
    }
    float o[MT][D / 8][4], m[MT][2], l[MT][2];
    uint32_t qf[MT == 1 ? D / 16 : 1][4];
    int r0 = 0, hi[MT][2], lo[MT][2];
    int stage = 0;
    uint32_t ph = 0;
    bool first_segment = true;

    for (int it = 0; it < units; ++it) {
      if (it == 0 || cu.tile == 0) {
        r0 = cu.rt * ROWS;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {                 // this lane's rows: the keys they see
            const int gr = r0 + t * 16 + (lane >> 2) + 8 * i, tok = fast_div(gr, c.G, p.div_group);
            const int pos = cu.r.kv - cu.r.n + min(tok, cu.r.n - 1);
            hi[t][i] = attn_hi(c, cu.r.kv, pos);
            lo[t][i] = attn_lo(c, pos);
            if (MT == 1) {
              const uint32_t* q = reinterpret_cast<const uint32_t*>(c.q + (long long)(cu.r.t0 + tok) * c.q_ts +
                                                                    (long long)(cu.h * c.G + gr - tok * c.G) * c.q_hs) + (lane & 3);
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                qf[MT == 1 ? k : 0][i] = tok < cu.r.n ? __ldg(q + 8 * k) : 0u;
                qf[MT == 1 ? k : 0][2 + i] = tok < cu.r.n ? __ldg(q + 8 * k + 4) : 0u;
              }
            }
            m[t][i] = -INFINITY;
            l[t][i] = 0.f;
          }
        if (MT > 1) {
          __syncwarp();
          for (int i = lane; i < ROWS * (D / 8); i += 32) {
            const int row = i / (D / 8), ch = i % (D / 8), gr = r0 + row, tok = fast_div(gr, c.G, p.div_group);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (tok < cu.r.n)
              v = __ldg(reinterpret_cast<const uint4*>(c.q + (long long)(cu.r.t0 + tok) * c.q_ts + (long long)(cu.h * c.G + gr - tok * c.G) * c.q_hs) + ch);
            st_shared_v4(sq + (uint32_t)(row * D * 2 + ((ch ^ (row & 7)) << 4)), v.x, v.y, v.z, v.w);
          }
          __syncwarp();
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int n = 0; n < D / 8; ++n) o[t][n][0] = o[t][n][1] = o[t][n][2] = o[t][n][3] = 0.f;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * stage, ph, c.status, p.wait_limit))) { ok = false; break; }
      const uint32_t sk = ring + stage * Sh::STAGE, sv = sk + Sh::KV_BYTES;

      // scores: fragment n covers keys 8 n .. 8 n + 7 (lane: rows lane / 4 and + 8, keys 2 (lane % 4) + {0, 1})
      float s[MT][NT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) s[t][n][0] = s[t][n][1] = s[t][n][2] = s[t][n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t qa[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          if (MT == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) qa[t][e] = qf[MT == 1 ? k : 0][e];
          } else {
            const int row = t * 16 + (lane & 15), ch = 2 * k + (lane >> 4);
            frag_ldm4(qa[t], sq + (uint32_t)(row * D * 2 + ((ch ^ (row & 7)) << 4)));
          }
        }
#pragma unroll
        for (int n2 = 0; n2 < NT / 2; ++n2) {
          uint32_t kf[4];
          frag_ldm4(kf, sk + xk[k & 3] + (uint32_t)((k >> 2) * (KT * 128) + n2 * 2048));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            frag_mma(s[t][2 * n2], qa[t], kf[0], kf[1]);
            frag_mma(s[t][2 * n2 + 1], qa[t], kf[2], kf[3]);
          }
        }
      }
      const int k0 = cu.k.lo + cu.tile * KT;
      const bool partial = k0 + KT > cu.k.all_hi || k0 < cu.k.all_lo;
      bool odd = false;                                    // a NaN or infinity in V of a tile with masked keys
      if (partial) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = k0 + n * 8 + 2 * (lane & 3) + (e & 1);
              if (j >= hi[t][e >> 1] || j < lo[t][e >> 1]) s[t][n][e] = -INFINITY;
            }
        // 0 * NaN must not reach rows that do not see a key: V of keys that no row sees becomes zero, other NaNs and infinities
        // are taken out and given back below
#pragma unroll 1
        for (int i = lane; i < Sh::KV_BYTES / 16; i += 32) {
          const int key = k0 + (i >> 3) % KT;
          uint32_t w[4];
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(sv + 16 * i) : "memory");
          bool hit = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            hit |= bf16x2_odd(w[e]);
            w[e] = key >= cu.k.hi ? 0u : bf16x2_clean(w[e]);
          }
          if (key >= cu.k.hi || hit) st_shared_v4(sv + 16 * i, w[0], w[1], w[2], w[3]);
          odd |= hit && key < cu.k.hi;
        }
        odd = __any_sync(0xffffffffu, odd);
        fence_async_proxy();                               // before the slot's next copy
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = s[t][0][2 * i];
#pragma unroll
          for (int n = 0; n < NT; ++n) x = fmaxf(x, fmaxf(s[t][n][2 * i], s[t][n][2 * i + 1]));
          x = fmaxf(m[t][i], x * p.scale2);
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          const float b_ = x == -INFINITY ? 0.f : x;       // nothing seen yet: all weights are 2^-inf = 0
          f[i] = fast_exp2(m[t][i] - b_);
          m[t][i] = x;
          float sum = 0.f;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            s[t][n][2 * i] = fast_exp2(fmaf(s[t][n][2 * i], p.scale2, -b_));
            s[t][n][2 * i + 1] = fast_exp2(fmaf(s[t][n][2 * i + 1], p.scale2, -b_));
            sum += s[t][n][2 * i] + s[t][n][2 * i + 1];
          }
          l[t][i] = l[t][i] * f[i] + sum;                  // this lane's part; joined over the quad at the end
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
          for (int n = 0; n < D / 8; ++n) { o[t][n][0] *= f[0]; o[t][n][1] *= f[0]; o[t][n][2] *= f[1]; o[t][n][3] *= f[1]; }
        }
      }
#pragma unroll
      for (int k = 0; k < KT / 16; ++k) {
        uint32_t a[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          a[t][0] = pack_bf16x2(s[t][2 * k][0], s[t][2 * k][1]);
          a[t][1] = pack_bf16x2(s[t][2 * k][2], s[t][2 * k][3]);
          a[t][2] = pack_bf16x2(s[t][2 * k + 1][0], s[t][2 * k + 1][1]);
          a[t][3] = pack_bf16x2(s[t][2 * k + 1][2], s[t][2 * k + 1][3]);
        }
#pragma unroll
        for (int n2 = 0; n2 < D / 16; ++n2) {
          uint32_t vf[4];
          frag_ldm4t(vf, sv + xv[n2 & 3] + (uint32_t)((n2 >> 2) * (KT * 128) + k * 2048));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            frag_mma(o[t][2 * n2], a[t], vf[0], vf[1]);
            frag_mma(o[t][2 * n2 + 1], a[t], vf[2], vf[3]);
          }
        }
      }
      if (odd) {
        // rare: the values that were taken out, read again, for the rows that see them
        for (int j = max(k0, 0); j < min(k0 + KT, cu.k.hi); ++j) {
          const int x = fast_div(j, c.cache.page_size, p.div_page), pg = __ldg(c.table + (long long)cu.b * c.width + x);
          if (pg < 0 || pg >= c.cache.n_pages) continue;
          const __nv_bfloat16* v = c.cache.v + (long long)pg * c.cache.ps + (long long)(j - x * c.cache.page_size) * c.cache.ts +
                                   (long long)cu.h * c.cache.hs + 2 * (lane & 3);
#pragma unroll
          for (int n = 0; n < D / 8; ++n) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(v + 8 * n);
            if (!bf16x2_odd(w)) continue;
            const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                if (j >= hi[t][i] || j < lo[t][i]) continue;
                if ((w & 0x7f80u) == 0x7f80u) o[t][n][2 * i] += v0;
                if ((w & 0x7f800000u) == 0x7f800000u) o[t][n][2 * i + 1] += v1;
              }
          }
        }
      }
      // The slot is free when every lane's fragments have been read.  Each was an operand of an MMA whose result is in o, so
      // the copy's address is made to depend on all of o: it cannot be issued while a load is still on its way.
      if (issued < units) {
        uint32_t dep = 0;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) dep |= __float_as_uint(o[0][n][0]);
        __syncwarp();
        issue(dep & p.zero);
      }
      if (++stage == PW_STAGES) { stage = 0; ph ^= 1u; }

      // ---- end of an item, or of this share's part of it --------------------------------------------------------------
      if (cu.tile + 1 == cu.k.tiles || it + 1 == units) {
        const long long item_first = u0 + it - cu.tile;
        const bool whole = item_first >= u0 && item_first + cu.k.tiles <= u1;
        const long long slot = 2 * g + (first_segment ? 0 : 1);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float sum = l[t][i];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            const int row = t * 16 + (lane >> 2) + 8 * i, gr = r0 + row, tok = fast_div(gr, c.G, p.div_group);
            if (tok >= cu.r.n) continue;
            if (whole) {
              const int head = cu.h * c.G + gr - tok * c.G;
              const float inv = sum == 0.f ? 0.f : 1.f / sum;
              __nv_bfloat16* out = c.out + (long long)(cu.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + 2 * (lane & 3);
#pragma unroll
              for (int n = 0; n < D / 8; ++n)
                *reinterpret_cast<uint32_t*>(out + 8 * n) = pack_bf16x2(o[t][n][2 * i] * inv, o[t][n][2 * i + 1] * inv);
              if (c.lse && (lane & 3) == 0)
                c.lse[(long long)(cu.r.t0 + tok) * c.H + head] = sum == 0.f ? -INFINITY : (m[t][i] + log2f(sum)) * PW_LN2;
            } else {
              float* d = p.part_o + (slot * ROWS + row) * D + 2 * (lane & 3);
#pragma unroll
              for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(d + 8 * n) = make_float2(o[t][n][2 * i], o[t][n][2 * i + 1]);
              if ((lane & 3) == 0) *reinterpret_cast<float2*>(p.part_ml + (slot * ROWS + row) * 2) = make_float2(m[t][i], sum);
            }
          }
        if (!whole && lane == 0) {
          // of the warps of a CTA, the first that holds a part announces the item
          const bool opens = item_first >= u0, enters = warp == 0 && first_segment && item_first < u0;
          if (opens || enters) {
            PwCut& x = s_cut[enters ? 0 : warp + 1];
            x.valid = 1; x.b = cu.b; x.h = cu.h; x.rt = cu.rt; x.first_unit = item_first; x.tiles = cu.k.tiles;
          }
        }
        first_segment = false;
      }
      cu.next(p);
    }
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      for (int j = max(0, issued - PW_STAGES); j < issued; ++j)
        mbar_wait(full + 8 * (j % PW_STAGES), (uint32_t)(j / PW_STAGES) & 1u, c.status, p.wait_limit);
    }
    if (__any_sync(0xffffffffu, odd_pages) && lane == 0) atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
  }

  // ---- joins ------------------------------------------------------------------------------------------------------------
  __threadfence();
  __syncthreads();
  auto share_of = [&](long long u) {
    long long x = u * shares / total;
    while (share_begin(x + 1) <= u) ++x;
    while (share_begin(x) > u) --x;
    return x;
  };
  if (tid <= PW_WARPS) {
    PwCut& x = s_cut[tid];
    int ready = 0;
    if (x.valid) {
      x.first_cta = (int)(share_of(x.first_unit) / PW_WARPS);
      x.last_cta = (int)(share_of(x.first_unit + x.tiles - 1) / PW_WARPS);
      // at most one item leaves a CTA's shares at their end: the counter of the CTA it starts in is its own
      ready = x.first_cta == x.last_cta || atomicAdd(p.counters + x.first_cta, 1u) == (uint32_t)(x.last_cta - x.first_cta);
    }
    s_ready[tid] = ready;
  }
  __syncthreads();
  __threadfence();
  constexpr int LANES = D / 4;                            // lanes per row (16 or 32), four columns each
  for (int w = 0; w <= PW_WARPS; ++w) {
    if (!s_ready[w]) continue;
    const PwCut x = s_cut[w];
    const ReqView r = attn_request(c, x.b);
    const long long first = share_of(x.first_unit), last = share_of(x.first_unit + x.tiles - 1);
    const long long slot0 = 2 * first + (share_begin(first) == x.first_unit ? 0 : 1);
    const int r0 = x.rt * ROWS, rows = min(ROWS, r.n * c.G - r0), col = (tid % LANES) * 4;
    for (int row = tid / LANES; row < rows; row += PW_THREADS / LANES) {
      const int gr = r0 + row, tok = fast_div(gr, c.G, p.div_group), head = x.h * c.G + gr - tok * c.G;
      // one pass: the running maximum moves along with the parts
      float M = -INFINITY, L = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (long long q = first; q <= last; ++q) {
        const long long at = (q == first ? slot0 : 2 * q) * ROWS + row;
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + at * 2));
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * D + col));
        const float mn = fmaxf(M, ml.x), b_ = mn == -INFINITY ? 0.f : mn;
        const float fa = fast_exp2(M - b_), fb = fast_exp2(ml.x - b_);
        M = mn;
        L = L * fa + ml.y * fb;
        acc.x = acc.x * fa + v.x * fb; acc.y = acc.y * fa + v.y * fb;
        acc.z = acc.z * fa + v.z * fb; acc.w = acc.w * fa + v.w * fb;
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
      *reinterpret_cast<uint2*>(c.out + (long long)(r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + col) =
          make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
      if (c.lse && col == 0) c.lse[(long long)(r.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * PW_LN2;
    }
  }
}

template <int D, int MT>
int pw_launch(PwParams p, const CUtensorMap& tk, const CUtensorMap& tv, char* scratch, cudaStream_t st) {
  using Sh = PwShape<D, MT>;
  static std::atomic<bool> attr_set[64];
  int dev = 0, sms = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  auto kernel = paged_warp_kernel<D, MT>;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
    attr_set[dev].store(true, std::memory_order_release);
  }
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int grid = std::min(sms, kPagedMaxSms);
  p.counters = reinterpret_cast<uint32_t*>(scratch);
  p.part_ml = reinterpret_cast<float*>(scratch + kPagedCounterBytes);
  p.part_o = p.part_ml + (size_t)2 * kPagedMaxSms * PW_WARPS * Sh::ROWS * 2;
  kernel<<<grid, PW_THREADS, Sh::SMEM, st>>>(tk, tv, p);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

}  // namespace

static_assert(PW_WARPS <= kPagedMaxPerSm, "the scratch of paged_attn.cu holds this kernel's parts too");

bool paged_warp_supported(const AttnCall& c) {
  if ((c.D != 64 && c.D != 128) || !(c.scale > 0.f)) return false;
  const int kt = c.D == 64 ? 64 : 32, pg = c.cache.page_size;
  // a tile is whole boxes of one page each; at most 32 boxes, one per lane
  return pg % 8 == 0 && (pg <= kt ? kt % pg == 0 : pg % kt == 0);
}

int launch_paged_warp(const AttnCall& c, int narrow_rows, char* scratch, cudaStream_t st) {
  PwParams p{};
  p.c = c;
  p.scale2 = c.scale * 1.4426950408889634f;
  p.narrow_rows = narrow_rows;
  p.min_units = 2;
  p.box_keys = std::min(c.cache.page_size, c.D == 64 ? 64 : 32);
  p.div_page = fast_div_magic((uint32_t)c.cache.page_size);
  p.div_group = fast_div_magic((uint32_t)c.G);
  p.wait_limit = wait_limit_cycles();
  CUtensorMap tk, tv;
  int rc = make_cache_maps(c, p.box_keys, &tk, &tv);
  if (rc) return rc;
  // Row tiles of 16 or 32 rows.  The host knows rows only on average: G per new token, tokens / requests new tokens.
  const bool one = ((c.T + c.B - 1) / c.B) * c.G <= 16;
  if (c.D == 64) return one ? pw_launch<64, 1>(p, tk, tv, scratch, st) : pw_launch<64, 2>(p, tk, tv, scratch, st);
  return one ? pw_launch<128, 1>(p, tk, tv, scratch, st) : pw_launch<128, 2>(p, tk, tv, scratch, st);
}

}  // namespace qb
