// Attention over the paged cache for many rows per key head (chunks of new tokens): both products on tcgen05.
//
// Mathematics: the running softmax of paged_attn.cu, for tiles of 128 rows x 128 keys.  A row tile holds 128 / G whole
// tokens of one request, row = token * G + query head in its group, so shared keys are loaded once for the group.
//   S = Q K^T          tcgen05.mma, operands in shared memory, S (fp32) in tensor memory
//   P = 2^(S c - m)    one thread per row; bf16 P goes back to tensor memory, over S
//   O += P V           tcgen05.mma, A = P from tensor memory, V as an MN-major B operand, O (fp32) in tensor memory
// m moves only when a row's maximum has grown by more than 2^8 (weights up to 2^8 are as exact as weights up to 1, and
// l uses the same m); then O is scaled in tensor memory by the row's thread.  That is safe without a further wait: the
// commit that announces S of tile j covers P V of tile j - 1, and P V of tile j waits for this thread.
//
// Roles (one CTA per SM, 384 threads): warps 0-3 and 4-7 are the softmax of two row tiles that share every K and V stage
// -- while one tile's softmax runs, the tensor core works for the other --, warp 8 loads (TMA), warp 9 issues the MMAs,
// warps 10-11 clean V where a tile has keys that some row does not see: keys past the request's end become zeros and NaNs
// or infinities are taken out (0 * NaN would reach every row); rows that do see such a value get it back at the end.
//
// Work: items = (request, key head, pair of row tiles), cut into key tiles.  With at least four items per SM whole items
// are dealt out, in an order that lets CTAs read the same key head at the same time (below); with fewer the line of
// all key tiles is cut into equal shares, one per CTA, and the CTA that finishes a cut item last joins the parts in
// share order (the rule of paged_attn.cu).
//
// What bounds it: S of both row tiles reads 8 KB of shared memory per 64 tensor cycles, the full rate, and the exponentials
// take as many cycles as the products (16 per cycle and SM).
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "paged_join.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"
#include "tc_small.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int TA_THREADS = 384;
constexpr int TA_TILE = 128;            // rows per row tile, keys per key tile
constexpr float TA_LN2 = 0.69314718055994530942f;
constexpr float TA_SLACK = 8.0f;        // how far (in powers of two) a row's maximum may run ahead of m

template <int D>
struct TaShape {
  static constexpr int STAGES = D == 64 ? 6 : 4;            // K and V tiles take turns; even, so V keeps to odd stages
  static constexpr int TILE_BYTES = TA_TILE * D * 2;        // one Q, K or V tile
  static constexpr int BARS = 2 * STAGES + STAGES + 12;     // full, empty, clean; s, p, o_full, o_free, q_full, q_empty x 2
  static constexpr int LIST_BYTES = kWideMaxRequests * 16;
  static constexpr int SMEM = (2 + STAGES) * TILE_BYTES + LIST_BYTES + BARS * 8 + 64 + 1024;
};

struct TaParams {
  AttnCall c;
  JoinCall join;          // what paged_warp.cu has left to join
  float scale2;
  int narrow_rows;        // requests with at most so many rows belong to paged_attn.cu
  int tokens_per_tile;    // 128 / G
  int box_keys;           // keys per TMA box: min(page_size, 128)
  long long wait_limit;
  uint32_t* counters;     // [2 * grid], zeroed
  float* part_o;          // [2 * grid][2 row tiles][D / 4][128 rows][4]
  float* part_ml;         // [2 * grid][2][128][2]
};

__device__ __forceinline__ float ta_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One stretch of key tiles [ja, jb) of an item.
struct TaSeg {
  ReqView r;
  int b, h, tok0;          // request, key head, first token of the pair
  int lo;                  // first key of tile 0, a multiple of 128
  int nt[2];               // key tiles that each row tile sees
  int ja, jb, tiles;       // this stretch, and all tiles of the item
  long long first_unit;    // of the item in the line
  __device__ __forceinline__ int end(int t) const { return min(jb, nt[t]); }
  __device__ __forceinline__ int last() const { return max(end(0), end(1)); }
};

__device__ __forceinline__ int ta_pair_tiles(const TaParams& p, const ReqView& r, int q, int* nt, int* lo) {
  const int tpt = p.tokens_per_tile, p0 = r.kv - r.n;
  *lo = min(attn_lo(p.c, p0 + 2 * q * tpt), r.kv) & ~(TA_TILE - 1);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int i0 = (2 * q + t) * tpt, cnt = min(r.n - i0, tpt);
    nt[t] = cnt > 0 ? max(0, (attn_hi(p.c, r.kv, p0 + i0 + cnt - 1) - *lo + TA_TILE - 1) / TA_TILE) : 0;
  }
  return max(1, max(nt[0], nt[1]));
}
__device__ __forceinline__ int ta_pairs(const TaParams& p, const ReqView& r) {
  return (r.n + 2 * p.tokens_per_tile - 1) / (2 * p.tokens_per_tile);
}

// The list of this kernel's requests (shared memory) and this CTA's part of their work.
struct TaWalk {
  const int* req;            // [n]
  const int* items;          // [n] inclusive sums
  const long long* units;    // [n] inclusive sums
  int n;
  bool whole;                // whole items are dealt out
  long long u, u1, total, shares;
  int k;

  __device__ __forceinline__ bool next(const TaParams& p, TaSeg& s) {
    int wi, q;
    const int hkv = p.c.cache.kv_heads;
    if (whole) {
      // rounds of gridDim.x items, every second one backwards: with the longest items first the shares come out even
      const int g = gridDim.x;
      const long long i = (long long)k * g + ((k & 1) ? g - 1 - (int)blockIdx.x : (int)blockIdx.x);
      ++k;
      if (i >= items[n - 1]) return false;
      wi = find(items, (int)i);
      const int local = (int)i - (wi ? items[wi - 1] : 0);
      s.b = req[wi];
      s.r = attn_request(p.c, s.b);
      const int np = ta_pairs(p, s.r);
      // Pairs with the most keys first.  While the request's keys fit the L2 (126 MB) the key heads run fastest, which sorts
      // items by length; beyond that all pairs of a key head come one after another, so that the CTAs in flight
      // stream the keys of few heads.
      if ((long long)s.r.kv * hkv * p.c.D * 4 <= 96000000LL) { q = np - 1 - local / hkv; s.h = local % hkv; }
      else { s.h = local / np; q = np - 1 - local % np; }
      s.tiles = ta_pair_tiles(p, s.r, q, s.nt, &s.lo);
      s.ja = 0; s.jb = s.tiles; s.first_unit = 0;
    } else {
      if (u >= u1) return false;
      int a = 0, e = n;
      while (a < e) { const int m = (a + e) >> 1; if (units[m] > u) e = m; else a = m + 1; }
      wi = a;
      const long long base = wi ? units[wi - 1] : 0;
      const long long hu = (units[wi] - base) / hkv;
      s.b = req[wi];
      s.r = attn_request(p.c, s.b);
      s.h = (int)((u - base) / hu);
      long long rest = u - base - s.h * hu;
      q = 0;
      s.tiles = ta_pair_tiles(p, s.r, 0, s.nt, &s.lo);
      while (rest >= s.tiles) { rest -= s.tiles; ++q; s.tiles = ta_pair_tiles(p, s.r, q, s.nt, &s.lo); }
      s.ja = (int)rest;
      s.jb = (int)min((long long)s.tiles, rest + (u1 - u));
      s.first_unit = u - rest;
      u += s.jb - s.ja;
    }
    s.tok0 = 2 * q * p.tokens_per_tile;
    return true;
  }
  __device__ __forceinline__ int find(const int* sums, int x) const {
    int a = 0, e = n;
    while (a < e) { const int m = (a + e) >> 1; if (sums[m] > x) e = m; else a = m + 1; }
    return a;
  }
};

// whether some row of the row tiles that take part in tile j does not see some of its keys
__device__ __forceinline__ bool ta_partial(const TaParams& p, const TaSeg& s, int t, int j) {
  const int i0 = s.tok0 + t * p.tokens_per_tile, i1 = min(s.r.n, i0 + p.tokens_per_tile) - 1, p0 = s.r.kv - s.r.n;
  const int k0 = s.lo + j * TA_TILE;
  return k0 + TA_TILE > attn_hi(p.c, s.r.kv, p0 + i0) || k0 < attn_lo(p.c, p0 + i1);
}

template <int D>
__global__ void __launch_bounds__(TA_THREADS, 1)
tc_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TaParams p) {
  using Sh = TaShape<D>;
  constexpr int STAGES = Sh::STAGES, TB = Sh::TILE_BYTES, HALVES = D / 64;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_g = smem_raw + (base - raw);
  const uint32_t sQ = base, sKV = base + 2 * TB, bars = sKV + STAGES * TB;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (STAGES + s); };
  auto clean = [&](int s) { return bars + 8u * (2 * STAGES + s); };
  auto pairbar = [&](int which, int t) { return bars + 8u * (3 * STAGES + 2 * which + t); };
  enum { S_FULL = 0, P_READY = 1, O_FULL = 2, O_FREE = 3, Q_FULL = 4, Q_EMPTY = 5 };
  const uint32_t tmem_slot = bars + 8u * (3 * STAGES + 12);
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(base_g + (tmem_slot - base));
  uint8_t* list = base_g + (2 + STAGES) * TB + Sh::BARS * 8 + 64;
  long long* l_units = reinterpret_cast<long long*>(list);
  int* l_req = reinterpret_cast<int*>(list + kWideMaxRequests * 8);
  int* l_items = l_req + kWideMaxRequests;
  __shared__ int s_n;
  __shared__ int s_warp_n[TA_THREADS / 32], s_warp_i[TA_THREADS / 32];
  __shared__ long long s_warp_u[TA_THREADS / 32];
  __shared__ int s_odd[8];         // segment number + 1 where a value was taken out of V
  __shared__ int s_join[2];
  __shared__ JoinShared s_list;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const AttnCall& c = p.c;
  const int hkv = c.cache.kv_heads;

  // ---- the list: requests of this kernel in order, with running sums of items and key tiles ---------------------------
  {
    int n_before = 0, i_before = 0;
    long long u_before = 0;
    for (int b0 = 0; b0 < c.B; b0 += TA_THREADS) {
      const int b = b0 + tid;
      int take = 0, items = 0;
      long long units = 0;
      if (b < c.B) {
        const ReqView r = attn_request(c, b);
        if ((long long)r.n * c.G > p.narrow_rows) {
          take = 1;
          const int np = ta_pairs(p, r);
          items = np * hkv;
          int nt[2], lo;
          for (int q = 0; q < np; ++q) units += ta_pair_tiles(p, r, q, nt, &lo);
          units *= hkv;
        }
      }
      int ni = take, ii = items;
      long long ui = units;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, ni, d), z = __shfl_up_sync(0xffffffffu, ii, d);
        const long long w = __shfl_up_sync(0xffffffffu, ui, d);
        if (lane >= d) { ni += y; ii += z; ui += w; }
      }
      if (lane == 31) { s_warp_n[warp] = ni; s_warp_i[warp] = ii; s_warp_u[warp] = ui; }
      __syncthreads();
      int n_all = n_before, i_all = i_before;
      long long u_all = u_before;
#pragma unroll
      for (int w = 0; w < TA_THREADS / 32; ++w) {
        if (w < warp) { ni += s_warp_n[w]; ii += s_warp_i[w]; ui += s_warp_u[w]; }
        n_all += s_warp_n[w]; i_all += s_warp_i[w]; u_all += s_warp_u[w];
      }
      if (take) {
        l_req[n_before + ni - 1] = b;
        l_items[n_before + ni - 1] = i_before + ii;
        l_units[n_before + ni - 1] = u_before + ui;
      }
      n_before = n_all; i_before = i_all; u_before = u_all;
      __syncthreads();
    }
    if (tid == 0) s_n = n_before;
    if (tid < 8) s_odd[tid] = 0;
  }
  __syncthreads();
  TaWalk walk;
  walk.n = s_n;
  walk.req = l_req; walk.items = l_items; walk.units = l_units;
  walk.k = 0; walk.u = walk.u1 = 0; walk.total = walk.shares = 1; walk.whole = true;
  bool some = walk.n > 0;
  if (some) {
    walk.whole = l_items[walk.n - 1] >= 4 * (int)gridDim.x;
    walk.total = l_units[walk.n - 1];
    walk.shares = min((long long)gridDim.x, walk.total);
    if (!walk.whole) {
      if ((long long)blockIdx.x >= walk.shares) some = false;
      else {
        walk.u = walk.total * blockIdx.x / walk.shares;
        walk.u1 = walk.total * (blockIdx.x + 1) / walk.shares;
      }
    }
  }
  if (!some) {
    asm volatile("griddepcontrol.wait;" ::: "memory");     // the kernel in front has ended
    join_all<D, TA_THREADS>(c, p.join, &s_list);
    return;
  }

  if (tid == 0) {
    // K and V take turns, so V lies in the odd stages; those are released by the cleaning warps too, which keeps their
    // count of the stage's turns in step (a parity wait cannot tell turns apart that are two or more behind)
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), s & 1 ? 3 : 1); mbar_init(clean(s), 64); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(pairbar(S_FULL, t), 1); mbar_init(pairbar(P_READY, t), 128);
      mbar_init(pairbar(O_FULL, t), 1); mbar_init(pairbar(O_FREE, t), 128);
      mbar_init(pairbar(Q_FULL, t), 1); mbar_init(pairbar(Q_EMPTY, t), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot_g;
  const uint32_t tS = tmem, tO = tmem + 256;    // S (and P): 2 x 128 columns, O: 2 x D columns

  TaSeg sg;
  if (warp == 8) {
    // ------------------------------------------------------------------------------------------------ loads (TMA)
    const int boxes = TA_TILE / p.box_keys;
    const uint32_t box_bytes = (uint32_t)p.box_keys * 128u;
    const uint32_t q_bytes = (uint32_t)(p.tokens_per_tile * c.G) * D * 2;
    uint32_t it = 0, uq[2] = {0, 0};
    bool ok = true;
    while (ok && walk.next(p, sg)) {
      const int e = sg.last();
      if (sg.ja >= e) continue;
      for (int j = sg.ja; j < e && ok; ++j) {
        // lane i < boxes: page of the tile's i-th box; one past the cache (a box of zeros) behind the request's keys
        int page = c.cache.n_pages, entry = 0;
        const int key = sg.lo + j * TA_TILE + lane * p.box_keys;
        if (lane < boxes && key < sg.r.kv) {
          page = __ldg(c.table + (long long)sg.b * c.width + key / c.cache.page_size);
          entry = key % c.cache.page_size;
          if (page < 0 || page >= c.cache.n_pages) {
            atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
            page = c.cache.n_pages;
          }
        }
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          const int s = it % STAGES;
          if (!__all_sync(0xffffffffu, mbar_wait(empty(s), ((it / STAGES) & 1u) ^ 1u, c.status, p.wait_limit))) { ok = false; break; }
          if (lane == 0) mbar_arrive_expect_tx(full(s), TB);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t dst = sKV + s * TB + lane * box_bytes;
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf)
              tma_load_4d(dst + hf * (TA_TILE * 128), kv ? &tm_v : &tm_k, full(s), hf * 64, entry, sg.h, page);
          }
          ++it;
          if (kv == 0 && j == sg.ja) {
            for (int t = 0; t < 2 && ok; ++t) {
              if (sg.ja >= sg.end(t)) continue;
              if (!__all_sync(0xffffffffu, mbar_wait(pairbar(Q_EMPTY, t), (uq[t] & 1u) ^ 1u, c.status, p.wait_limit))) { ok = false; break; }
              ++uq[t];
              if (lane == 0) {
                mbar_arrive_expect_tx(pairbar(Q_FULL, t), q_bytes);
                for (int hf = 0; hf < HALVES; ++hf)
                  tma_load_3d(sQ + t * TB + hf * (TA_TILE * 128), &tm_q, pairbar(Q_FULL, t), hf * 64, sg.h * c.G,
                              sg.r.t0 + sg.tok0 + t * p.tokens_per_tile);
              }
              __syncwarp();
            }
            if (!ok) break;
          }
        }
      }
    }
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      const uint32_t lo = it > (uint32_t)STAGES ? it - STAGES : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(full(j % STAGES), (j / STAGES) & 1u, c.status, p.wait_limit);
      for (int t = 0; t < 2; ++t)
        if (uq[t]) mbar_wait(pairbar(Q_FULL, t), (uq[t] - 1) & 1u, c.status, p.wait_limit);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TA_TILE >> 3) << 17) | ((uint32_t)(TA_TILE >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(TA_TILE >> 4) << 24);
      uint32_t it = 0, ns[2] = {0, 0}, nseg[2] = {0, 0}, clean_ph = 0;
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !mbar_wait(bar, parity, c.status, p.wait_limit)) ok = false;
        return ok;
      };
      auto scores = [&](int t, int stage) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (uint32_t)(k >> 2) * (TA_TILE * 128) + (uint32_t)(k & 3) * 32;
          tc_mma(tS + t * 128, smem_desc(sQ + t * TB + off, 16, 1024), smem_desc(sKV + stage * TB + off, 16, 1024), idesc_s, k ? 1u : 0u);
        }
        tc_commit(pairbar(S_FULL, t));
      };
      while (ok && walk.next(p, sg)) {
        const int e = sg.last(), e0[2] = {sg.end(0), sg.end(1)};
        if (sg.ja >= e) continue;
        const uint32_t it0 = it;
        auto stage_of = [&](uint32_t i) { return (int)(i % STAGES); };
        auto phase_of = [&](uint32_t i) { return (i / STAGES) & 1u; };
        if (!wait(full(stage_of(it0)), phase_of(it0))) break;
        tc_fence_after();
        for (int t = 0; t < 2; ++t) {
          if (sg.ja >= e0[t]) continue;
          if (!wait(pairbar(Q_FULL, t), nseg[t] & 1u)) break;
          tc_fence_after();
          scores(t, stage_of(it0));
          if (sg.ja + 1 >= e0[t]) tc_commit(pairbar(Q_EMPTY, t));
        }
        if (!ok) break;
        tc_commit(empty(stage_of(it0)));
        for (int j = sg.ja; j < e && ok; ++j) {
          const uint32_t iv = it0 + 2 * (uint32_t)(j - sg.ja) + 1, ik = iv + 1;   // V of tile j, K of tile j + 1
          bool v_seen = false, k_seen = false;
          const bool dirty = (j < e0[0] && ta_partial(p, sg, 0, j)) || (j < e0[1] && ta_partial(p, sg, 1, j));
          for (int t = 0; t < 2; ++t) {
            if (j >= e0[t]) continue;
            if (!v_seen) {
              if (!wait(full(stage_of(iv)), phase_of(iv))) break;
              if (dirty) {
                const int s = stage_of(iv);
                if (!wait(clean(s), (clean_ph >> s) & 1u)) break;
                clean_ph ^= 1u << s;
              }
              v_seen = true;
            }
            if (!wait(pairbar(P_READY, t), ns[t] & 1u)) break;
            ++ns[t];
            if (j == sg.ja && !wait(pairbar(O_FREE, t), (nseg[t] & 1u) ^ 1u)) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < TA_TILE / 16; ++k)
              tc_mma_ta(tO + t * D, tS + t * 128 + k * 8, smem_desc(sKV + stage_of(iv) * TB + k * 2048, TA_TILE * 128, 1024), idesc_o,
                        (j > sg.ja || k) ? 1u : 0u);
            if (j + 1 == e0[t]) { tc_commit(pairbar(O_FULL, t)); ++nseg[t]; }
            else {
              if (!k_seen) {
                if (!wait(full(stage_of(ik)), phase_of(ik))) break;
                tc_fence_after();
                k_seen = true;
              }
              scores(t, stage_of(ik));
              if (j + 2 >= e0[t]) tc_commit(pairbar(Q_EMPTY, t));
            }
          }
          if (!ok) break;
          tc_commit(empty(stage_of(iv)));
          if (j + 1 < e) tc_commit(empty(stage_of(ik)));
        }
        it = it0 + 2 * (uint32_t)(e - sg.ja);
      }
    }
  } else if (warp >= 10) {
    // ------------------------------------------------------------------------------------------------ V cleaning
    const int ct = tid - 320;
    uint32_t it = 0;
    int seg = 0;
    bool ok = true;
    for (; ok && walk.next(p, sg); ++seg) {
      const int e = sg.last();
      const int p0 = sg.r.kv - sg.r.n;
      // keys from here on are seen by no row of the pair
      const int stop = attn_hi(c, sg.r.kv, p0 + min(sg.r.n, sg.tok0 + 2 * p.tokens_per_tile) - 1);
      for (int j = sg.ja; j < e; ++j, it += 2) {
        const uint32_t iv = it + 1;
        const int s = iv % STAGES;
        if (!__all_sync(0xffffffffu, mbar_wait(full(s), (iv / STAGES) & 1u, c.status, p.wait_limit))) { ok = false; break; }
        if (!((j < sg.end(0) && ta_partial(p, sg, 0, j)) || (j < sg.end(1) && ta_partial(p, sg, 1, j)))) {
          if (lane == 0) mbar_arrive(empty(s));
          continue;
        }
        const int k0 = sg.lo + j * TA_TILE;
        bool odd = false;
        uint8_t* v = base_g + (2 + s) * TB;
        for (int i = ct; i < TB / 16; i += 64) {
          uint4* w = reinterpret_cast<uint4*>(v + i * 16);
          const int key = k0 + ((i >> 3) & (TA_TILE - 1));        // [half][128 keys][128 bytes]
          if (key >= stop) { *w = make_uint4(0, 0, 0, 0); continue; }
          uint4 x = *w;
          uint32_t* y = reinterpret_cast<uint32_t*>(&x);
          bool hit = false;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if ((y[q] & 0x7f80u) == 0x7f80u) { y[q] &= 0xffff0000u; hit = true; }
            if ((y[q] & 0x7f800000u) == 0x7f800000u) { y[q] &= 0x0000ffffu; hit = true; }
          }
          if (hit) { *w = x; odd = true; }
        }
        if (odd) s_odd[seg & 7] = seg + 1;
        fence_async_proxy();
        mbar_arrive(clean(s));
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ softmax, output
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tSr = tS + t * 128 + lanes, tOr = tO + t * D + lanes;
    const int tok_in = row / c.G, head_in = row - tok_in * c.G;
    uint32_t ns = 0, nseg = 0;
    int seg = 0;
    bool ok = true;
    for (; ok && walk.next(p, sg); ++seg) {
      const int e = sg.end(t), p0 = sg.r.kv - sg.r.n;
      const int tok = sg.tok0 + t * p.tokens_per_tile + tok_in;
      const bool real = tok_in < p.tokens_per_tile && tok < sg.r.n;
      const int hi = real ? attn_hi(c, sg.r.kv, p0 + tok) : sg.r.kv, lo = real ? attn_lo(c, p0 + tok) : 0;
      float m = -INFINITY, l = 0.f;
      for (int j = sg.ja; j < e; ++j) {
        if (!mbar_wait(pairbar(S_FULL, t), ns & 1u, c.status, p.wait_limit)) { ok = false; break; }
        ++ns;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_ld32_start(tSr + q * 32, s + q * 32);
        tc_ld_wait();
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_ready32(s + q * 32);
        if (ta_partial(p, sg, t, j)) {
          const int k0 = sg.lo + j * TA_TILE, h_ = hi - k0, l_ = lo - k0;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i >= h_ || i < l_) s[i] = 0xff800000u;
        }
        float mx[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) mx[q] = __uint_as_float(s[q]);
#pragma unroll
        for (int i = 4; i < 128; i += 8) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            mx[q] = fmaxf(mx[q], __uint_as_float(s[i + q]));
            if (i + 4 + q < 128) mx[q] = fmaxf(mx[q], __uint_as_float(s[i + 4 + q]));
          }
        }
        const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale2;
        const bool grow = mt > m + TA_SLACK;
        if (__any_sync(0xffffffffu, grow)) {
          const float mn = grow ? mt : m;
          const float f = m == mn ? 1.f : ta_exp2(m - mn);          // m = -infinity: 0
          m = mn;
          l *= f;
          if (j > sg.ja) {
#pragma unroll 1
            for (int q = 0; q < D / 32; ++q) {
              uint32_t o[32];
              tc_ld32(tOr + q * 32, o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tc_st32(tOr + q * 32, o);
            }
          }
        }
        const float base = m == -INFINITY ? 0.f : m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float a = ta_exp2(fmaf(__uint_as_float(s[q * 64 + 2 * i]), p.scale2, -base));
            const float b = ta_exp2(fmaf(__uint_as_float(s[q * 64 + 2 * i + 1]), p.scale2, -base));
            sum[2 * (i & 1)] += a;
            sum[2 * (i & 1) + 1] += b;
            w[i] = pack_bf16x2(a, b);
          }
          tc_st32(tSr + q * 32, w);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tc_st_wait();
        tc_fence_before();
        mbar_arrive(pairbar(P_READY, t));
      }
      if (!ok) break;
      const bool worked = sg.ja < e;
      if (worked) {
        if (!mbar_wait(pairbar(O_FULL, t), nseg & 1u, c.status, p.wait_limit)) { ok = false; break; }
        ++nseg;
        tc_fence_after();
      }
      const bool whole = sg.ja == 0 && sg.jb == sg.tiles;
      const bool odd = s_odd[seg & 7] == seg + 1;
      const int head = sg.h * c.G + head_in;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      int first = 0, last = 0, slot = 0;
      if (!whole) {
        auto share_of = [&](long long u) {
          long long x = u * walk.shares / walk.total;
          while (walk.total * (x + 1) / walk.shares <= u) ++x;
          while (walk.total * x / walk.shares > u) --x;
          return (int)x;
        };
        first = share_of(sg.first_unit);
        last = share_of(sg.first_unit + sg.tiles - 1);
        // a share's first stretch has slot 0, its last slot 1
        slot = 2 * (int)blockIdx.x + (walk.total * blockIdx.x / walk.shares == sg.first_unit + sg.ja ? 0 : 1);
      }
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (worked) {
          tc_ld32(tOr + q * 32, o);
          if (q == D / 32 - 1) { tc_fence_before(); mbar_arrive(pairbar(O_FREE, t)); }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0;
        }
        if (odd && real) {
          // rare: values that were taken out of V go to the rows that see their key
          for (int j = sg.ja; j < sg.last(); ++j) {
            if (!((j < sg.end(0) && ta_partial(p, sg, 0, j)) || (j < sg.end(1) && ta_partial(p, sg, 1, j)))) continue;
            const int k0 = sg.lo + j * TA_TILE;
            for (int key = max(k0, lo); key < min(k0 + TA_TILE, hi); ++key) {
              const int page = __ldg(c.table + (long long)sg.b * c.width + key / c.cache.page_size);
              if (page < 0 || page >= c.cache.n_pages) continue;
              const __nv_bfloat16* v = c.cache.v + (long long)page * c.cache.ps + (long long)(key % c.cache.page_size) * c.cache.ts +
                                       (long long)sg.h * c.cache.hs + q * 32;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float x = __bfloat162float(v[i]);
                if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
              }
            }
          }
        }
        if (whole) {
          if (real) {
            uint4* out = reinterpret_cast<uint4*>(c.out + (long long)(sg.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + q * 32);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t w[4];
#pragma unroll
              for (int x = 0; x < 4; ++x)
                w[x] = pack_bf16x2(__uint_as_float(o[i * 8 + 2 * x]) * inv, __uint_as_float(o[i * 8 + 2 * x + 1]) * inv);
              out[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        } else {
          float4* dst = reinterpret_cast<float4*>(p.part_o + (long long)(slot * 2 + t) * D * 128);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            dst[(q * 8 + i) * 128 + row] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                       __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
        }
      }
      if (whole) {
        if (real && c.lse) c.lse[(long long)(sg.r.t0 + tok) * c.H + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * TA_LN2;
        continue;
      }
      reinterpret_cast<float2*>(p.part_ml)[(slot * 2 + t) * 128 + row] = make_float2(m, l);
      __threadfence();
      asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
      if (row == 0) s_join[t] = atomicAdd(p.counters + 2 * first + t, 1u) == (uint32_t)(last - first);
      asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
      if (s_join[t]) {
        __threadfence();
        // the first share's part of the item is its last stretch, unless that share begins with the item
        const int slot0 = 2 * first + (walk.total * first / walk.shares == sg.first_unit ? 0 : 1);
        auto part = [&](int x) { return ((x == first ? slot0 : 2 * x) * 2 + t); };
        float M = -INFINITY;
        for (int x = first; x <= last; ++x) M = fmaxf(M, __ldcg(reinterpret_cast<const float2*>(p.part_ml) + part(x) * 128 + row).x);
        const float mb = M == -INFINITY ? 0.f : M;
        float L = 0.f;
        for (int x = first; x <= last; ++x) {
          const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml) + part(x) * 128 + row);
          L += ml.y * ta_exp2(ml.x - mb);
        }
        const float iv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll 1
        for (int q = 0; q < D / 8; ++q) {
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
          for (int x = first; x <= last; ++x) {
            const float g = ta_exp2(__ldcg(reinterpret_cast<const float2*>(p.part_ml) + part(x) * 128 + row).x - mb);
            const float4* src = reinterpret_cast<const float4*>(p.part_o + (long long)part(x) * D * 128);
            const float4 u = __ldcg(src + (2 * q) * 128 + row), v = __ldcg(src + (2 * q + 1) * 128 + row);
            a.x += u.x * g; a.y += u.y * g; a.z += u.z * g; a.w += u.w * g;
            b.x += v.x * g; b.y += v.y * g; b.z += v.z * g; b.w += v.w * g;
          }
          if (real)
            *reinterpret_cast<uint4*>(c.out + (long long)(sg.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + q * 8) =
                make_uint4(pack_bf16x2(a.x * iv, a.y * iv), pack_bf16x2(a.z * iv, a.w * iv), pack_bf16x2(b.x * iv, b.y * iv),
                           pack_bf16x2(b.z * iv, b.w * iv));
        }
        if (real && c.lse) c.lse[(long long)(sg.r.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * TA_LN2;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");       // the kernel in front has ended
  join_all<D, TA_THREADS>(c, p.join, &s_list);
}

template <int D>
int ta_launch(const TaParams& p0, char* counters, char* scratch, cudaStream_t st) {
  using Sh = TaShape<D>;
  static std::atomic<bool> attr_set[64];
  int dev = 0, sms = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  auto kernel = tc_attention_kernel<D>;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
    attr_set[dev].store(true, std::memory_order_release);
  }
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  TaParams p = p0;
  const AttnCall& c = p.c;
  p.counters = reinterpret_cast<uint32_t*>(counters);
  p.part_ml = reinterpret_cast<float*>(scratch);
  p.part_o = p.part_ml + (size_t)2 * kPagedMaxSms * 2 * 128 * 2;

  // a dimension of one entry may come with any stride: give the map one it accepts
  auto pitch = [](int64_t n, int64_t stride, int64_t other) { return (uint64_t)(n > 1 ? stride : other) * 2; };
  CUtensorMap tq, tk, tv;
  {
    const uint64_t dims[3] = {(uint64_t)D, (uint64_t)c.H, (uint64_t)c.T};
    const uint64_t pt[2] = {pitch(c.H, c.q_hs, D), pitch(c.T, c.q_ts, D)};
    const uint32_t box[3] = {64, (uint32_t)c.G, (uint32_t)p.tokens_per_tile};
    const int rc = make_tensor_map_nd(&tq, 3, c.q, dims, pt, box);
    if (rc) return rc;
  }
  const int rc = make_cache_maps(c, p.box_keys, &tk, &tv);
  if (rc) return rc;

  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min(sms, kPagedMaxSms));
  cfg.blockDim = dim3(TA_THREADS);
  cfg.dynamicSmemBytes = Sh::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, kernel, tq, tk, tv, p));
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

}  // namespace

// Boxes of 64 elements of a head x `box_keys` entries of a page.
int make_cache_maps(const AttnCall& c, int box_keys, void* tm_k, void* tm_v) {
  // a dimension of one entry may come with any stride: give the map one it accepts
  auto pitch = [&](int64_t n, int64_t stride) { return (uint64_t)(n > 1 ? stride : c.D) * 2; };
  const uint64_t dims[4] = {(uint64_t)c.D, (uint64_t)c.cache.page_size, (uint64_t)c.cache.kv_heads, (uint64_t)c.cache.n_pages};
  const uint64_t pt[3] = {pitch(c.cache.page_size, c.cache.ts), pitch(c.cache.kv_heads, c.cache.hs), pitch(c.cache.n_pages, c.cache.ps)};
  const uint32_t box[4] = {64, (uint32_t)box_keys, 1, 1};
  const int rc = make_tensor_map_nd(tm_k, 4, c.cache.k, dims, pt, box);
  return rc ? rc : make_tensor_map_nd(tm_v, 4, c.cache.v, dims, pt, box);
}

bool tc_attention_supported(const AttnCall& c) {
  if (c.D != 64 && c.D != 128) return false;
  if (c.G > TA_TILE || !(c.scale > 0.f) || c.B > kWideMaxRequests) return false;
  const int pg = c.cache.page_size;
  return pg % 8 == 0 && (pg <= TA_TILE ? TA_TILE % pg == 0 : pg % TA_TILE == 0);
}

size_t tc_attention_scratch_bytes(int head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  return (size_t)2 * kPagedMaxSms * 2 * 128 * (head_dim + 2) * 4;
}

int launch_tc_attention(const AttnCall& c, int narrow_rows, const JoinCall& join, char* counters, char* scratch, cudaStream_t st) {
  TaParams p{};
  p.c = c;
  p.join = join;
  p.scale2 = c.scale * 1.4426950408889634f;
  p.narrow_rows = narrow_rows;
  p.tokens_per_tile = TA_TILE / c.G;
  p.box_keys = std::min(c.cache.page_size, TA_TILE);
  p.wait_limit = wait_limit_cycles();
  return c.D == 64 ? ta_launch<64>(p, counters, scratch, st) : ta_launch<128>(p, counters, scratch, st);
}

}  // namespace qb
