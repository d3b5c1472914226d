// Attention over the paged cache for many rows per key head (chunks of new tokens): both products on tcgen05.
//
// Mathematics: the running softmax of paged_attn.cu, for tiles of 128 rows x 128 keys.  A row tile holds 128 / G whole
// tokens of one request, row = token * G + query head in its group, so shared keys are loaded once for the group.
//   S = Q K^T          tcgen05.mma, operands in shared memory, S (fp32) in tensor memory
//   P = 2^(S c - m)    one thread per row; bf16 P goes back to tensor memory, over S
//   O += P V           tcgen05.mma, A = P from tensor memory, V as an MN-major B operand, O (fp32) in tensor memory
// m need not be the maximum: weights of 2^10 are as exact as weights of 1 (both have the same 8 and 24 bits), so m is a row's
// maximum over its first tile and moves only when a tile's sum of weights shows that the scores have outgrown it (by more, values
// of a size that bf16 still holds would overflow O); then O is scaled in tensor memory by the row's thread.  That is safe without
// a further wait: the commit that announces S of tile j covers P V of tile j - 1, and P V of tile j waits for this thread.
//
// Roles (one CTA per SM, 384 threads): warps 0-3 and 4-7 are the softmax of two row tiles that share every K and V stage
// -- while one tile's softmax runs, the tensor core works for the other --, warp 8 loads (TMA), warp 9 issues the MMAs,
// warps 10-11 clean V where a tile has keys that some row does not see: keys past the request's end become zeros and NaNs
// or infinities are taken out (0 * NaN would reach every row); rows that do see such a value get it back at the end.
//
// Work: items = (request, key head, pair of row tiles), each a run of key tiles.  Whole items are dealt out, longest first, to
// whichever CTA is free, where that ends about as early as equal shares would (the rule stands at its place below);
// else the line of all key tiles is cut into equal shares, up to three per CTA, and a kernel behind this one joins the parts of cut
// items (paged_join.cuh).
//
// What bounds it: neither unit, but the chain of a row tile.  A key tile of both row tiles takes about 4000 cycles (4096 tokens behind 28k,
// 1.64 GHz), of which the products of both are 2 x 1053 (128 x 128 x 128 measured alone: Q K^T 531 cycles, P V 522 of 512) and the
// exponentials as much (16 per cycle and SM): the tensor pipe and the special-function unit are active 56 % of the time each.  Since
// P lies over S, the next S of a row tile waits for P V, P V for the softmax and the softmax for S: what is left of the 4000 cycles after
// its own products, about 3000, a row tile spends in its softmax and the handovers, and the other row tile's products fill only a part.
// Measured: 4096 tokens behind 28k, 40 heads, D 128: 2.42 to 2.49 ms, 1012 to 1040 TFLOP/s (0.60 to 0.62 of the measured bf16 rate;
// the clock falls to 1.64 GHz under it); 4 requests of 512 tokens behind 3584, 8 key heads of 4: 138 to 159 us, 812 to 934 TFLOP/s.
//
// P is bf16, as the other operand is; m, l and O are fp32.  With fp32 weights the error against 64 bits is 0.0017 of the result (its
// own rounding to bf16), with these 0.0023.
// Built and slower: two warps that issue MMAs, one per row tile (391 -> 427 us at 4096 tokens over 6k keys); 16 softmax warps,
// two per row quadrant, that swap maxima (358 -> 411); 1/8 to 3/8 of the exponentials by a polynomial (358 -> 363 to 401).
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

constexpr int TA_THREADS = 384;
constexpr int TA_TILE = 128;            // rows per row tile, keys per key tile
constexpr float TA_LN2 = 0.69314718055994530942f;
constexpr long long TA_L2_BYTES = 96000000;
// Key tiles that the cuts of a share cost.  Measured with 2 / 6 / 12: 1021 fresh tokens, 32 heads 40.7 / 34.5 / 34.5 us; 200 tokens behind 500,
// 8 heads 23.1 / 30.3 / 30.3; 400 behind 2000, 2048 fresh over shared keys, 8 x 300 fresh and 4 x 512 behind 3584 the same with all.
constexpr int TA_CUT = 6;
constexpr int TA_SEGS = 4;              // segments handed out ahead
constexpr float TA_OUTGROWN = 1024.0f;  // a tile's sum of weights that asks for a new m (at most 128 with m the maximum)

template <int D>
struct TaShape {
  static constexpr int STAGES = D == 64 ? 6 : 4;            // K and V tiles take turns; even, so V keeps to odd stages
  static constexpr int TILE_BYTES = TA_TILE * D * 2;        // one Q, K or V tile
  static constexpr int BARS = 3 * STAGES + 12 + 3 * TA_SEGS;       // full, empty, clean; six for each row tile; the segments' three
  static constexpr int LIST_BYTES = kWideMaxRequests * 12;
  static constexpr int SMEM = (2 + STAGES) * TILE_BYTES + LIST_BYTES + BARS * 8 + 64 + 1024;
};

struct TaParams {
  AttnCall c;
  float scale2;
  int narrow_rows;        // requests with at most so many rows belong to paged_warp.cu
  int tokens_per_tile;    // 128 / G
  int box_keys;           // keys per TMA box: min(page_size, 128)
  long long wait_limit;
  uint32_t div_page;
  uint32_t* counters;     // zeroed; [0]: items dealt out, [1], [2]: JoinCall::wide_counts
  JoinCut* cuts;          // JoinCall::wide_cuts
  float* part_o;          // [2 * shares][2 row tiles][D / 4][128 rows][4]
  float* part_ml;         // [2 * shares][2][128][2]
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two fp32 values in a 64-bit register
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ uint64_t pack2u(uint32_t a, uint32_t b) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ float lo2(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float hi2(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
// One stretch of key tiles [ja, jb) of an item, as the loading warp hands it to the others.
struct TaSeg {
  int valid;               // 0: no more
  ReqView r;
  int b, h, tok0;          // request, key head, first token of the pair
  int lo;                  // first key of tile 0, a multiple of 128
  int seen;                // first key that some row of the pair sees
  int solo;                // there is only the first row tile: both softmax groups work for it, on every other key tile each
  int nt[2];               // key tiles that each row tile sees
  int full_lo[2], full_hi[2];   // tiles in this range have only keys that every row of the row tile sees
  int stop;                // keys from here on are seen by no row of the pair
  int ja, jb;
  int whole;               // the stretch is the item
  int slot, slot0, first, last;   // where not: its place for partial results, that of the item's first part, shares first .. last
  __device__ __forceinline__ int end(int t) const { return min(jb, nt[t]); }
  __device__ __forceinline__ int last_tile() const { return max(end(0), end(1)); }
  __device__ __forceinline__ bool partial(int t, int j) const { return j < full_lo[t] || j >= full_hi[t]; }
  // whether V of tile j has to be cleaned
  __device__ __forceinline__ bool dirty(int j) const { return (j < end(0) && partial(0, j)) || (j < end(1) && partial(1, j)); }
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
  const int* units;          // [n] inclusive sums of key tiles
  int n;
  bool dealt;                // whole items are dealt out one by one
  int share, shares, each, extra, u, u1;

  __device__ __forceinline__ int find(const int* sums, int x) const {
    int a = 0, e = n;
    while (a < e) { const int m = (a + e) >> 1; if (sums[m] > x) e = m; else a = m + 1; }
    return a;
  }
  // the first total % shares shares have one tile more
  __device__ __forceinline__ int begin(int s) const { return s * each + min(s, extra); }
  __device__ __forceinline__ int share_of(int x) const {
    const int cut = extra * (each + 1);
    return x < cut ? x / (each + 1) : extra + (x - cut) / each;
  }
  // called by all lanes of the loading warp
  __device__ __forceinline__ bool next(const TaParams& p, TaSeg& s) {
    const int hkv = p.c.cache.kv_heads;
    int wi, q, tiles, first_unit = 0;
    if (dealt) {
      int i = 0;
      if ((threadIdx.x & 31) == 0) i = (int)atomicAdd(p.counters, 1u);
      i = __shfl_sync(0xffffffffu, i, 0);
      if (i >= items[n - 1]) return false;
      wi = find(items, i);
      const int local = i - (wi ? items[wi - 1] : 0);
      s.b = req[wi];
      s.r = attn_request(p.c, s.b);
      q = ta_pairs(p, s.r) - 1 - local / hkv;        // the longest first: the last ones to be dealt out are short
      s.h = local % hkv;
      tiles = ta_pair_tiles(p, s.r, q, s.nt, &s.lo);
      s.ja = 0; s.jb = tiles;
    } else {
      while (u >= u1) {
        share += gridDim.x;
        if (share >= shares) return false;
        u = begin(share); u1 = begin(share + 1);
      }
      wi = find(units, u);
      const int base = wi ? units[wi - 1] : 0, hu = (units[wi] - base) / hkv;
      s.b = req[wi];
      s.r = attn_request(p.c, s.b);
      s.h = (u - base) / hu;
      int rest = u - base - s.h * hu;
      q = 0;
      tiles = ta_pair_tiles(p, s.r, 0, s.nt, &s.lo);
      while (rest >= tiles) { rest -= tiles; ++q; tiles = ta_pair_tiles(p, s.r, q, s.nt, &s.lo); }
      s.ja = rest;
      s.jb = min(tiles, rest + (u1 - u));
      first_unit = u - rest;
      s.slot = 2 * share + (begin(share) == u ? 0 : 1);   // a share's first stretch, or its last
      u += s.jb - s.ja;
    }
    s.valid = 1;
    s.whole = s.ja == 0 && s.jb == tiles;
    if (!s.whole) {
      s.first = share_of(first_unit);
      s.last = share_of(first_unit + tiles - 1);
      s.slot0 = 2 * s.first + (begin(s.first) == first_unit ? 0 : 1);
    }
    s.tok0 = 2 * q * p.tokens_per_tile;
    s.solo = s.tok0 + p.tokens_per_tile >= s.r.n;
    const int p0 = s.r.kv - s.r.n;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i0 = s.tok0 + t * p.tokens_per_tile, i1 = min(s.r.n, i0 + p.tokens_per_tile) - 1;
      s.full_hi[t] = max(0, attn_hi(p.c, s.r.kv, p0 + i0) - s.lo) / TA_TILE;
      s.full_lo[t] = (max(0, attn_lo(p.c, p0 + i1) - s.lo) + TA_TILE - 1) / TA_TILE;
    }
    s.seen = attn_lo(p.c, p0 + s.tok0);
    s.stop = attn_hi(p.c, s.r.kv, p0 + min(s.r.n, s.tok0 + 2 * p.tokens_per_tile) - 1);
    return true;
  }
};

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
  auto seg_full = [&](int i) { return bars + 8u * (3 * STAGES + 12 + (i & (TA_SEGS - 1))); };
  auto seg_empty = [&](int i) { return bars + 8u * (3 * STAGES + 12 + TA_SEGS + (i & (TA_SEGS - 1))); };
  auto mail = [&](int i) { return bars + 8u * (3 * STAGES + 12 + 2 * TA_SEGS + (i & (TA_SEGS - 1))); };
  const uint32_t tmem_slot = bars + 8u * Sh::BARS;
  volatile uint32_t* tmem_slot_g = reinterpret_cast<volatile uint32_t*>(base_g + (tmem_slot - base));
  uint8_t* list = base_g + (2 + STAGES) * TB + Sh::BARS * 8 + 64;
  int* l_units = reinterpret_cast<int*>(list);
  int* l_req = l_units + kWideMaxRequests;
  int* l_items = l_req + kWideMaxRequests;
  __shared__ int s_n, s_over;
  __shared__ unsigned long long s_kv;              // keys of this kernel's requests
  __shared__ int s_most, s_least;                  // key tiles of its longest and shortest item
  __shared__ int s_key[TA_THREADS];

  __shared__ int s_warp_n[TA_THREADS / 32], s_warp_i[TA_THREADS / 32];
  __shared__ long long s_warp_u[TA_THREADS / 32];
  __shared__ int s_odd[8];         // segment number + 1 where a value was taken out of V
  __shared__ TaSeg s_seg[TA_SEGS];
  __shared__ float2 s_mail[TA_SEGS][TA_TILE];     // (m, l) of the second softmax group where both work for one row tile

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");     // the join kernel, where it comes after this one
  const AttnCall& c = p.c;
  const int hkv = c.cache.kv_heads;

  // ---- the list: requests of this kernel in order, with running sums of items and key tiles ---------------------------
  {
    int n_before = 0, i_before = 0;
    long long u_before = 0;
    if (tid == 0) { s_kv = 0; s_most = 0; s_least = 0x7fffffff; }
    __syncthreads();
    for (int b0 = 0; b0 < c.B; b0 += TA_THREADS) {
      const int b = b0 + tid;
      int take = 0, items = 0;
      long long units = 0;
      if (b < c.B) {
        const ReqView r = attn_request(c, b);
        if ((long long)r.n * c.G > p.narrow_rows) {
          take = 1;
          atomicAdd(&s_kv, (unsigned long long)r.kv);
          const int np = ta_pairs(p, r);
          items = np * hkv;
          int nt[2], lo;
          int most = 0, least = 0x7fffffff;
          for (int q = 0; q < np; ++q) {
            const int u = ta_pair_tiles(p, r, q, nt, &lo);
            units += u; most = max(most, u); least = min(least, u);
          }
          units *= hkv;
          atomicMax(&s_most, most);
          atomicMin(&s_least, least);
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
        l_units[n_before + ni - 1] = (int)min(u_before + ui, 0x7fffffffLL);
      }
      n_before = n_all; i_before = i_all; u_before = u_all;
      __syncthreads();
    }
    if (tid == 0) { s_n = n_before; s_over = u_before > 0x7fffffffLL; }
    if (tid < 8) s_odd[tid] = 0;
  }
  __syncthreads();
  TaWalk walk;
  walk.n = s_n;
  walk.req = l_req; walk.items = l_items; walk.units = l_units;
  bool some = walk.n > 0;
  if (some && s_over) {     // 2^31 key tiles and more: the lengths cannot be meant
    if (tid == 0) atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
    some = false;
  }
  if (some) {
    const int total = l_units[walk.n - 1];
    const int grid = (int)gridDim.x;
    // Whole items are dealt out, the long ones first, where that ends about as early as equal shares of the line of all key
    // tiles would: the last items to be dealt are the shortest, half of one is lost on average, while a share's borders
    // cut two items, which costs about six key tiles (parts written, read and joined).  And only with all keys and values
    // in the L2 (126 MB), since it works on all key heads at once.  Shares are taken in up to three rounds: the CTAs of a
    // round work on a contiguous part of the line, so that fewer key heads are streamed at a time.
    const long long bytes = (long long)s_kv * hkv * D * 4;
    const int mean = total / grid;
    walk.dealt = max(s_most, mean + (l_items[walk.n - 1] > grid ? s_least / 2 : 0)) <= mean + TA_CUT && bytes <= TA_L2_BYTES;
    const int rounds = (int)min(min((long long)kWideRounds, bytes / TA_L2_BYTES + 1), max(1LL, (long long)total / (256LL * grid)));
    walk.shares = min(grid * rounds, total);
    walk.each = total / walk.shares;
    walk.extra = total - walk.each * walk.shares;
    walk.share = (int)blockIdx.x;
    walk.u = walk.u1 = 0;
    if (!walk.dealt) {
      some = walk.share < walk.shares;
      if (some) { walk.u = walk.begin(walk.share); walk.u1 = walk.begin(walk.share + 1); }
    }
  }
  if (some && walk.dealt && walk.n > 1 && walk.n <= TA_THREADS) {
    // requests with the longest items first (in any order the result is the same)
    int b = 0, items = 0, units = 0, key = 0;
    if (tid < walk.n) {
      b = l_req[tid];
      items = l_items[tid] - (tid ? l_items[tid - 1] : 0);
      units = l_units[tid] - (tid ? l_units[tid - 1] : 0);
      const ReqView r = attn_request(c, b);
      int nt[2], lo;
      key = ta_pair_tiles(p, r, ta_pairs(p, r) - 1, nt, &lo);
      s_key[tid] = key;
    }
    __syncthreads();
    int rank = 0, i_before = 0, u_before = 0;
    if (tid < walk.n) {
      for (int i = 0; i < walk.n; ++i) {
        const bool first = s_key[i] > key || (s_key[i] == key && i < tid);
        rank += first;
        if (first) {
          i_before += l_items[i] - (i ? l_items[i - 1] : 0);
          u_before += l_units[i] - (i ? l_units[i - 1] : 0);
        }
      }
    }
    __syncthreads();
    if (tid < walk.n) { l_req[rank] = b; l_items[rank] = i_before + items; l_units[rank] = u_before + units; }
    __syncthreads();
  }
  if (!some) {
    // nothing may follow this grid in the stream before the kernels in front of it have ended
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }

  if (tid == 0) {
    // K and V take turns, so V lies in the odd stages; those are released by the cleaning warps too, which keeps their
    // count of the stage's turns in step (a parity wait cannot tell turns apart that are two or more behind)
    for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), s & 1 ? 3 : 1); mbar_init(clean(s), 64); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(pairbar(S_FULL, t), 1); mbar_init(pairbar(P_READY, t), 4);
      mbar_init(pairbar(O_FULL, t), 1); mbar_init(pairbar(O_FREE, t), 4);
      mbar_init(pairbar(Q_FULL, t), 1); mbar_init(pairbar(Q_EMPTY, t), 1);
    }
    // readers of a segment: the MMA thread, the two cleaning warps, the eight softmax warps
    for (int i = 0; i < TA_SEGS; ++i) { mbar_init(seg_full(i), 1); mbar_init(seg_empty(i), 11); mbar_init(mail(i), 4); }
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

  // The next segment, for every role but the loads; `n` counts them.  false: there is none, or a wait has run out.
  auto take = [&](TaSeg& sg, int n, bool& ok) {
    ok = mbar_wait(seg_full(n), (uint32_t)(n / TA_SEGS) & 1u, c.status, p.wait_limit);
    if (!ok) return false;
    sg = s_seg[n & (TA_SEGS - 1)];
    return sg.valid != 0;
  };
  // registers: 384 threads x 168 at launch = 128 x 88 + 256 x 208
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (warp == 8) {
    // ------------------------------------------------------------------------------------------------ loads (TMA)
    const int boxes = TA_TILE / p.box_keys;
    const uint32_t box_bytes = (uint32_t)p.box_keys * 128u;
    const uint32_t q_bytes = (uint32_t)(p.tokens_per_tile * c.G) * D * 2;
    uint32_t it = 0, uq0 = 0, uq1 = 0;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity, c.status, p.wait_limit));
      return ok;
    };
    TaSeg sg;
    for (int n = 0;; ++n) {
      const bool more = walk.next(p, sg);
      if (!wait(seg_empty(n), ((uint32_t)(n / TA_SEGS) & 1u) ^ 1u)) break;
      if (lane == 0) {
        sg.valid = more;
        s_seg[n & (TA_SEGS - 1)] = sg;
        mbar_arrive(seg_full(n));
      }
      if (!more) break;
      const int e = sg.last_tile();
      for (int j = sg.ja; j < e && ok; ++j) {
        // lane i < boxes: page of the tile's i-th box.  A box of keys that no row of the pair sees is filled with zeros (one page past
        // the cache) and its page not looked up: those in front of a window may have been given back
        int page = c.cache.n_pages, entry = 0;
        const int key = sg.lo + j * TA_TILE + lane * p.box_keys;
        if (lane < boxes && key < sg.stop && key + p.box_keys > sg.seen) {
          const int x = fast_div(key, c.cache.page_size, p.div_page);
          page = __ldg(c.table + (long long)sg.b * c.width + x);
          entry = key - x * c.cache.page_size;
          if (page < 0 || page >= c.cache.n_pages) {
            atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
            page = c.cache.n_pages;
          }
        }
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++it) {
          const int s = it % STAGES;
          if (!wait(empty(s), ((it / STAGES) & 1u) ^ 1u)) break;
          if (lane == 0) mbar_arrive_expect_tx(full(s), TB);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t dst = sKV + s * TB + lane * box_bytes;
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf)
              tma_load_4d(dst + hf * (TA_TILE * 128), kv ? &tm_v : &tm_k, full(s), hf * 64, entry, sg.h, page);
          }
          if (kv == 0 && j == sg.ja) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              uint32_t& uq = t ? uq1 : uq0;
              if (sg.ja >= sg.end(t) || !wait(pairbar(Q_EMPTY, t), (uq & 1u) ^ 1u)) continue;
              ++uq;
              if (lane == 0) {
                mbar_arrive_expect_tx(pairbar(Q_FULL, t), q_bytes);
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
                  tma_load_3d(sQ + t * TB + hf * (TA_TILE * 128), &tm_q, pairbar(Q_FULL, t), hf * 64, sg.h * c.G,
                              sg.r.t0 + sg.tok0 + t * p.tokens_per_tile);
              }
              __syncwarp();
            }
            if (!ok) { ++it; break; }
          }
        }
      }
      if (!ok) break;
    }
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      const uint32_t lo = it > (uint32_t)STAGES ? it - STAGES : 0;
      for (uint32_t j = lo; j < it; ++j) mbar_wait(full(j % STAGES), (j / STAGES) & 1u, c.status, p.wait_limit);
      if (uq0) mbar_wait(pairbar(Q_FULL, 0), (uq0 - 1) & 1u, c.status, p.wait_limit);
      if (uq1) mbar_wait(pairbar(Q_FULL, 1), (uq1 - 1) & 1u, c.status, p.wait_limit);
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------------------------------------------ MMA issuer
    // The whole warp walks the loop on values that are the same in every lane, and one elected lane issues: the operands
    // of an MMA then lie in uniform registers, and an issue takes 12 cycles instead of 60 (one lane's private loop), less
    // than the MMA's 64.
    {
      auto uni = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
      uint32_t leader;
      asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(leader));
      const uint32_t uQ = uni((int)sQ), uKV = uni((int)sKV), ub = uni((int)bars), uT = uni((int)tmem);
      auto ufull = [&](int i) { return ub + 8u * i; };
      auto uempty = [&](int i) { return ub + 8u * (STAGES + i); };
      auto uclean = [&](int i) { return ub + 8u * (2 * STAGES + i); };
      auto upair = [&](int which, int t) { return ub + 8u * (3 * STAGES + 2 * which + t); };
      const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TA_TILE >> 3) << 17) | ((uint32_t)(TA_TILE >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(TA_TILE >> 4) << 24);
      const uint64_t dq = smem_desc(0, 16, 1024) | ((uQ & 0x3FFFFu) >> 4), dk = smem_desc(0, 16, 1024) | ((uKV & 0x3FFFFu) >> 4),
                     dv = smem_desc(0, TA_TILE * 128, 1024) | ((uKV & 0x3FFFFu) >> 4);
      uint32_t ns0 = 0, ns1 = 0, nseg0 = 0, nseg1 = 0, nq1 = 0, clean_ph = 0, full_ph = 0;   // phases of the ring's stages, a bit each
      int sk = 0;                                             // stage of the next K tile; V's is the one behind it
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        ok = __all_sync(0xffffffffu, ok && mbar_wait(bar, parity, c.status, p.wait_limit));
        return ok;
      };
      auto wait_full = [&](int s) {
        const bool w = wait(ufull(s), (full_ph >> s) & 1u);
        full_ph ^= 1u << s;
        return w;
      };
      auto scores = [&](int t, int qt, int stage) {            // S of t, from row tile qt and the K of a stage
        const uint64_t a = dq + (uint32_t)qt * (TB >> 4), b = dk + (uint32_t)stage * (TB >> 4);
        if (leader) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = ((uint32_t)(k >> 2) * (TA_TILE * 128) + (uint32_t)(k & 3) * 32) >> 4;
            tc_mma(uT + t * 128, a + off, b + off, idesc_s, k ? 1u : 0u);
          }
          tc_commit(upair(S_FULL, t));
        }
      };
      auto commit = [&](uint32_t bar) { if (leader) tc_commit(bar); };
      for (int n = 0;; ++n) {
        if (!wait(seg_full(n), (uint32_t)(n / TA_SEGS) & 1u)) break;
        const TaSeg& sg = s_seg[n & (TA_SEGS - 1)];
        const int valid = uni(sg.valid), ja = uni(sg.ja), e0 = uni(sg.end(0)), e1 = uni(sg.end(1)), fl0 = uni(sg.full_lo[0]),
                  fl1 = uni(sg.full_lo[1]), fh0 = uni(sg.full_hi[0]), fh1 = uni(sg.full_hi[1]), e = max(e0, e1), solo = uni(sg.solo);
        __syncwarp();
        if (lane == 0) mbar_arrive(seg_empty(n));
        if (!valid) break;
        if (ja >= e) continue;
        if (solo) {
          // one row tile: S and O of t = 0 and 1 are those of even and odd key tiles, so that the products of one go with the
          // exponentials of the other here too.  K of tile j + 2 is asked for behind P V of tile j.
          auto ring = [&](int s, int by) { return s + by >= STAGES ? s + by - STAGES : s + by; };
          if (!wait_full(sk) || !wait(upair(Q_FULL, 0), nseg0 & 1u)) break;
          tc_fence_after();
          scores(0, 0, sk);
          commit(uempty(sk));
          if (ja + 1 < e) {
            const int s1 = ring(sk, 2);
            if (!wait_full(s1)) break;
            tc_fence_after();
            scores(1, 0, s1);
            commit(uempty(s1));
          }
          if (ja + 2 >= e) commit(upair(Q_EMPTY, 0));
          for (int j0 = ja; j0 < e && ok; j0 += 2) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int j = j0 + t, sv = sk + 1, s2 = ring(sk, 4 % STAGES);
              uint32_t &ns = t ? ns1 : ns0, &nseg = t ? nseg1 : nseg0;
              if (j >= e || !ok || !wait_full(sv)) continue;
              if (j < fl0 || j >= fh0) {
                if (!wait(uclean(sv), (clean_ph >> sv) & 1u)) continue;
                clean_ph ^= 1u << sv;
              }
              if (j0 == ja && !wait(upair(O_FREE, t), (nseg & 1u) ^ 1u)) continue;
              if (!wait(upair(P_READY, t), ns & 1u)) continue;
              ++ns;
              tc_fence_after();
              const uint64_t bv = dv + (uint32_t)sv * (TB >> 4);
              if (leader) {
#pragma unroll
                for (int k = 0; k < TA_TILE / 16; ++k)
                  tc_mma_ta(uT + 256 + t * D, uT + t * 128 + k * 8, bv + (uint32_t)k * 128u, idesc_o, (j0 > ja || k) ? 1u : 0u);
              }
              commit(uempty(sv));
              if (j + 2 >= e) { commit(upair(O_FULL, t)); ++nseg; }
              else {
                if (!wait_full(s2)) continue;
                tc_fence_after();
                scores(t, 0, s2);
                commit(uempty(s2));
                if (j + 3 >= e) commit(upair(Q_EMPTY, 0));
              }
              sk = ring(sk, 2);
            }
          }
          if (!ok) break;
          continue;
        }
        if (!wait_full(sk)) break;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int et = t ? e1 : e0;
          if (ja >= et || !wait(upair(Q_FULL, t), (t ? nq1 : nseg0) & 1u)) continue;
          if (t) ++nq1;
          tc_fence_after();
          scores(t, t, sk);
          if (ja + 1 >= et) commit(upair(Q_EMPTY, t));
        }
        if (!ok) break;
        commit(uempty(sk));
        for (int j = ja; j < e; ++j) {
          // The issuer is at most a few MMAs ahead of the tensor pipe: what it waits for here, the pipe soon waits for too.
          const int sv = sk + 1;                              // V of tile j
          sk = sv + 1 == STAGES ? 0 : sv + 1;                 // K of tile j + 1
          if (!wait_full(sv)) break;
          if ((j < e0 && (j < fl0 || j >= fh0)) || (j < e1 && (j < fl1 || j >= fh1))) {
            if (!wait(uclean(sv), (clean_ph >> sv) & 1u)) break;
            clean_ph ^= 1u << sv;
          }
          bool k_seen = false;
          const uint64_t bv = dv + (uint32_t)sv * (TB >> 4);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int et = t ? e1 : e0;
            uint32_t &ns = t ? ns1 : ns0, &nseg = t ? nseg1 : nseg0;
            if (j >= et || !ok) continue;
            if (j == ja && !wait(upair(O_FREE, t), (nseg & 1u) ^ 1u)) continue;
            if (!wait(upair(P_READY, t), ns & 1u)) continue;
            ++ns;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int k = 0; k < TA_TILE / 16; ++k)
                tc_mma_ta(uT + 256 + t * D, uT + t * 128 + k * 8, bv + (uint32_t)k * 128u, idesc_o, (j > ja || k) ? 1u : 0u);
            }
            if (j + 1 == et) { commit(upair(O_FULL, t)); ++nseg; }
            else {
              if (!k_seen) {
                if (!wait_full(sk)) continue;
                tc_fence_after();
                k_seen = true;
              }
              scores(t, t, sk);
              if (j + 2 >= et) commit(upair(Q_EMPTY, t));
            }
          }
          if (!ok) break;
          commit(uempty(sv));
          if (j + 1 < e) commit(uempty(sk));
        }
        if (!ok) break;
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ V cleaning
    const int ct = tid - 320;
    uint32_t it = 0;
    bool ok = true;
    TaSeg sg;
    for (int n = 0; ok; ++n) {
      if (!__all_sync(0xffffffffu, take(sg, n, ok))) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(n));
      const int e = sg.last_tile();
      for (int j = sg.ja; j < e; ++j, it += 2) {
        const uint32_t iv = it + 1;
        const int s = iv % STAGES;
        if (!__all_sync(0xffffffffu, mbar_wait(full(s), (iv / STAGES) & 1u, c.status, p.wait_limit))) { ok = false; break; }
        if (!sg.dirty(j)) {
          if (lane == 0) mbar_arrive(empty(s));
          continue;
        }
        const int k0 = sg.lo + j * TA_TILE;
        bool odd = false;
        uint8_t* v = base_g + (2 + s) * TB;
        for (int i = ct; i < TB / 16; i += 64) {
          uint4* w = reinterpret_cast<uint4*>(v + i * 16);
          const int key = k0 + ((i >> 3) & (TA_TILE - 1));        // [half][128 keys][128 bytes]
          if (key >= sg.stop) { *w = make_uint4(0, 0, 0, 0); continue; }
          uint4 x = *w;
          if (bf16x2_odd(x.x) || bf16x2_odd(x.y) || bf16x2_odd(x.z) || bf16x2_odd(x.w)) {
            *w = make_uint4(bf16x2_clean(x.x), bf16x2_clean(x.y), bf16x2_clean(x.z), bf16x2_clean(x.w));
            odd = true;
          }
        }
        if (odd) s_odd[n & 7] = n + 1;
        fence_async_proxy();
        mbar_arrive(clean(s));
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
      }
    }
  }
  } else {
    // ------------------------------------------------------------------------------------------------ softmax, output
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tSr = tS + t * 128 + lanes, tOr = tO + t * D + lanes;
    const int tok_in = row / c.G, head_in = row - tok_in * c.G;
    uint32_t ns = 0, nseg = 0, nseg1 = 0;     // nseg1: nseg of the second group, for the first
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {     // one answer for the warp
      ok = __all_sync(0xffffffffu, ok && mbar_wait(bar, parity, c.status, p.wait_limit));
      return ok;
    };
    for (int n = 0; ok; ++n) {
      // the segment is read where it lies: only what the key loop needs stays in registers
      if (!wait(seg_full(n), (uint32_t)(n / TA_SEGS) & 1u)) break;
      const TaSeg& sg = s_seg[n & (TA_SEGS - 1)];
      if (!sg.valid) break;
      const bool solo = sg.solo;
      const int rt = solo ? 0 : t, e = sg.end(rt), step = solo ? 2 : 1, p0 = sg.r.kv - sg.r.n;
      const int tok = sg.tok0 + rt * p.tokens_per_tile + tok_in;
      const bool real = tok_in < p.tokens_per_tile && tok < sg.r.n;
      const int hi = real ? attn_hi(c, sg.r.kv, p0 + tok) : sg.r.kv, lo = real ? attn_lo(c, p0 + tok) : 0;
      const int full_lo = rt ? sg.full_lo[1] : sg.full_lo[0], full_hi = rt ? sg.full_hi[1] : sg.full_hi[0], seg_lo = sg.lo;
      const int ja = sg.ja + (solo ? t : 0);
      float m = real ? -INFINITY : 0.f, l = 0.f;       // rows that are none need no maximum
      for (int j = ja; j < e; j += step) {
        if (!wait(pairbar(S_FULL, t), ns & 1u)) break;
        ++ns;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_ld32_start(tSr + q * 32, s + q * 32);
        tc_ld_wait();
#pragma unroll
        for (int q = 0; q < 4; ++q) tc_ready32(s + q * 32);
        if (__any_sync(0xffffffffu, j < full_lo || j >= full_hi)) {      // (a vote: the selects are to be branched around)
          const int k0 = seg_lo + j * TA_TILE, h_ = hi - k0, l_ = lo - k0;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i >= h_ || i < l_) s[i] = 0xff800000u;
        }
        // The weights are taken with the m there is; only where a row has none yet, or where its sum shows that the scores
        // have outgrown m, the maximum is looked for and the tile done again with it.  That saves a pass over the scores of almost every tile.
        float sum = 0.f;
#pragma unroll 1
        for (int pass = __any_sync(0xffffffffu, m == -INFINITY) ? 1 : 0; pass < 2; ++pass) {
          if (__builtin_expect(pass == 1, 0)) {
            float mx[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) mx[q] = max3(__uint_as_float(s[q]), __uint_as_float(s[4 + q]), __uint_as_float(s[8 + q]));
#pragma unroll
            for (int i = 12; i + 8 <= 128; i += 8) {
#pragma unroll
              for (int q = 0; q < 4; ++q) mx[q] = max3(mx[q], __uint_as_float(s[i + q]), __uint_as_float(s[i + 4 + q]));
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) mx[q] = fmaxf(mx[q], __uint_as_float(s[124 + q]));
            const float mt = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * p.scale2;
            const float mn = fmaxf(m, mt);
            const float f = m == mn ? 1.f : fast_exp2(m - mn);        // m = -infinity: 0
            m = mn;
            l *= f;
            if (j > ja) {
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
          const uint64_t scale2x2 = pack2(p.scale2, p.scale2), base2 = pack2(-base, -base);
          uint64_t sum2[2] = {0, 0};
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const uint64_t x = fma2(pack2u(s[q * 64 + 2 * i], s[q * 64 + 2 * i + 1]), scale2x2, base2);
              const float ea = fast_exp2(lo2(x)), eb = fast_exp2(hi2(x));
              sum2[i & 1] = add2(sum2[i & 1], pack2(ea, eb));
              w[i] = pack_bf16x2(ea, eb);
            }
            tc_st32(tSr + q * 32, w);
          }
          sum2[0] = add2(sum2[0], sum2[1]);
          sum = lo2(sum2[0]) + hi2(sum2[0]);
          // rows that are none do not vote: what they hold is other requests' queries, or what an earlier kernel left in shared memory
          if (!__any_sync(0xffffffffu, real && !(sum < TA_OUTGROWN))) break;
        }
        l += sum;
        tc_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pairbar(P_READY, t));
      }
      if (!ok) break;
      const bool worked = ja < e;
      if (t == 1) {
        // a letter for every segment, so that the letters' barriers keep step with the segments
        if (solo) s_mail[n & (TA_SEGS - 1)][row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(mail(n));
        if (solo) {                                  // the first group does the rest
          nseg += worked;
          if (lane == 0) mbar_arrive(seg_empty(n));
          continue;
        }
      }
      if (worked) {
        if (!wait(pairbar(O_FULL, t), nseg & 1u)) break;
        ++nseg;
        tc_fence_after();
      }
      const bool worked1 = t == 0 && (solo ? ja + 1 < e : sg.ja < sg.end(1)), both = solo && worked1;
      float f0 = 1.f, f1 = 0.f;
      if (both) {
        // (the letter comes first: behind it O_FULL of t = 1 cannot be two turns behind)
        if (!wait(mail(n), (uint32_t)(n / TA_SEGS) & 1u) || !wait(pairbar(O_FULL, 1), nseg1 & 1u)) break;
        tc_fence_after();
        const float2 ml = s_mail[n & (TA_SEGS - 1)][row];
        const float M = fmaxf(m, ml.x), b = M == -INFINITY ? 0.f : M;
        f0 = fast_exp2(m - b);
        f1 = fast_exp2(ml.x - b);
        l = l * f0 + ml.y * f1;
        m = M;
      }
      nseg1 += worked1;
      const bool odd = s_odd[n & 7] == n + 1;
      const int head = sg.h * c.G + head_in;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (worked) {
          tc_ld32(tOr + q * 32, o);
          if (both) {
            uint32_t o1[32];
            tc_ld32(tOr + D + q * 32, o1);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
          }
          if (q == D / 32 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(pairbar(O_FREE, t));
              if (both) mbar_arrive(pairbar(O_FREE, 1));
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0;
        }
        if (odd && real) {
          // rare: values that were taken out of V go to the rows that see their key
          for (int j = sg.ja; j < sg.last_tile(); ++j) {
            if (!sg.dirty(j)) continue;
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
        if (sg.whole) {
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
          float4* dst = reinterpret_cast<float4*>(p.part_o + (long long)(sg.slot * 2 + t) * D * 128);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            dst[(q * 8 + i) * 128 + row] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                       __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
        }
      }
      if (sg.whole) {
        if (real && c.lse) c.lse[(long long)(sg.r.t0 + tok) * c.H + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * TA_LN2;
        __syncwarp();
        if (lane == 0) mbar_arrive(seg_empty(n));
        continue;
      }
      reinterpret_cast<float2*>(p.part_ml)[(sg.slot * 2 + t) * 128 + row] = make_float2(m, l);
      // the second of the shares that cut the item tells the join kernel about this row tile of it
      if (row == 0 && (sg.slot >> 1) == sg.first + 1 && real) {
        const int parts = sg.last - sg.first + 1;
        const bool many = parts > kJoinWideShort;
        const int at = (int)atomicAdd(p.counters + (many ? 2 : 1), 1u);
        p.cuts[many ? 2 * kWideMaxShares - 1 - at : at] =
            JoinCut{sg.slot0, sg.first, parts, sg.r.t0 + tok, 0, min(p.tokens_per_tile, sg.r.n - tok) * c.G, sg.h, t};
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(n));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");       // as above
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
  p.part_o = p.part_ml + (size_t)2 * kWideMaxShares * 2 * 128 * 2;
  p.cuts = reinterpret_cast<JoinCut*>(p.part_o + (size_t)2 * kWideMaxShares * 2 * 128 * D);

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
  return (size_t)2 * kWideMaxShares * 2 * 128 * (head_dim + 2) * 4 + (size_t)2 * kWideMaxShares * sizeof(JoinCut);
}

void tc_attention_join(int head_dim, char* counters, char* scratch, JoinCall* j) {
  j->wide_counts = reinterpret_cast<uint32_t*>(counters) + 1;
  j->wide_ml = reinterpret_cast<float*>(scratch);
  j->wide_o = j->wide_ml + (size_t)2 * kWideMaxShares * 2 * 128 * 2;
  j->wide_cuts = reinterpret_cast<const JoinCut*>(j->wide_o + (size_t)2 * kWideMaxShares * 2 * 128 * head_dim);
}

int launch_tc_attention(const AttnCall& c, int narrow_rows, char* counters, char* scratch, cudaStream_t st) {
  TaParams p{};
  p.c = c;
  p.scale2 = c.scale * 1.4426950408889634f;
  p.narrow_rows = narrow_rows;
  p.tokens_per_tile = TA_TILE / c.G;
  p.box_keys = std::min(c.cache.page_size, TA_TILE);
  p.div_page = fast_div_magic((uint32_t)c.cache.page_size);
  p.wait_limit = wait_limit_cycles();
  return c.D == 64 ? ta_launch<64>(p, counters, scratch, st) : ta_launch<128>(p, counters, scratch, st);
}

}  // namespace qb
