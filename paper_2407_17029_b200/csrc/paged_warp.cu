// Attention over the paged cache for few rows per key head (decoding, drafted tokens): the form that streams the cache
// with TMA.  Head sizes 64 and 128, pages that fit its tiles; paged_attn.cu takes the rest.
//
// Mathematics as in paged_attn.cu: a running softmax in base 2 over row tiles of 16 rows (tokens x query heads that share
// a key head); partial triples (maximum, sum, weighted values) over disjoint keys join in any grouping.
//
// What bounds it: the cache's bytes, so each warp is made to need little else.  The key tiles of all (request, row tile) pairs
// are put in one line, alike for every key head, and the line is cut into parts; a share is one part for one key head, and
// the heads of a part are neighbouring shares, so that warps which run at the same time read the same pages (with each head's
// tiles in a row instead, 6 requests x 40 heads x 15k keys took 309 us, now 293).  Every warp starts with one share and then
// takes the next one that nobody has taken, the later ones shorter: SMs do not get equal parts of a saturated memory (with
// one equal share per warp the slowest CTA of a 1 GB call ended 20 % after the median).  A warp streams its shares through a
// ring of its own -- lane i issues box i of a tile as the ring's slot becomes free, across the borders of items and shares,
// and nothing waits for another warp -- and does both products for the whole tile with the maximum that there is; a new one is
// looked for only where a sum shows that the scores have outgrown it.  In flight per SM: 8 warps x 3 slots x 8 KB.
//
// An item cut by a share's border leaves partial triples in the workspace, which a second kernel joins (paged_join.cuh); joined
// by whichever warp came last, the joins of a call fell to the few warps that ended last, one row after the other: 5 to
// 65 us at the end of a 45 to 180 us call.  Calls of very few rows have a form without either (CLUSTER): one cluster of CTAs
// per item, joined through the cluster's shared memory.
//
// Measured, D 128, on several cards: 64 requests of 30 to 8100 keys, 8 key heads of 4 query heads, 1.07 GB: 186 to 193 us = 5.5 to
// 5.7 TB/s, of which the join kernel about 8; 6 requests of 15k keys, 40 heads, 1.87 GB: 286 to 295 us = 6.3 to 6.5 TB/s, the
// rate of a copy.
//
// The weights are rounded to bf16 for their product with V, as mma.sync wants them; m, l, o and the parts are fp32.  With fp32 weights
// the error against 64 bits is 0.0017 of the result (its own rounding to bf16), with these 0.0023.
//
// Entries behind a request's keys: whole pages are asked for at a page number past the cache, which TMA fills with zeros;
// the rest of the last page is masked (scores set to -infinity, V set to zero in shared memory).
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include "paged_join.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"
#include "tc_small.cuh"

namespace qb {
using namespace ptx;
namespace {

constexpr int PW_WARPS = 8, PW_THREADS = PW_WARPS * 32;
constexpr int PW_MAX_LEVELS = kPagedLevels;
// Key tiles of the shortest shares: with short ones the last warps end together, with long ones there are fewer joins.  Measured with
// 4 / 11 / 24: 64 requests of 30 to 8100 keys 191 / 194 / 196 us, 6 of 15k keys 281 / 282 / 286; 200 of up to 1000 keys 99 / 99 / 97, 24 of
// up to 2000 keys with 32 key heads 77.5 / 76 / 76, 16 requests of 12 to 28 rows 67 / 61 / 61.
constexpr int PW_FINE = 11;
constexpr float PW_OUTGROWN = 1024.0f;   // a lane's sum of a tile's weights that asks for a new maximum
constexpr float PW_LN2 = 0.69314718055994530942f;

template <int D>
struct PwShape {
  static constexpr int ROWS = 16;
  static constexpr int KT = D == 64 ? 32 : 16;            // keys per tile: 8 KB of K and V
  static constexpr int STAGES = 3;
  static constexpr int KV_BYTES = KT * D * 2;
  static constexpr int STAGE = 2 * KV_BYTES;
  static constexpr int SMEM = PW_WARPS * STAGES * STAGE + 1024;
};

struct PwParams {
  AttnCall c;
  float scale2;              // scale * log2 e
  int narrow_rows;           // requests with more rows than this belong to the tcgen05 kernel
  int box_keys;              // keys per TMA box: min(page_size, KT)
  uint32_t div_page, div_group;
  uint32_t zero;             // 0, but not to the compiler
  long long wait_limit;
  uint32_t* counters;        // [0]: shares taken; [1 ... 3]: JoinCall::counts.  Zeroed
  JoinCut* cuts;             // JoinCall::cuts
  float* part_o;             // [2 * shares][ROWS][D]
  float* part_ml;            // [2 * shares][ROWS][2]
};

// Keys [first, hi) that some row of a row tile sees, in `tiles` tiles from lo on, which is first rounded down; [all_lo, all_hi): those
// that every row sees.
struct PwRange { int lo, hi, tiles, first, all_lo, all_hi; };
template <int ROWS, int KT>
__device__ __forceinline__ PwRange pw_range(const PwParams& p, const ReqView& r, int rt) {
  const AttnCall& c = p.c;
  const int i0 = fast_div(rt * ROWS, c.G, p.div_group), i1 = min(r.n - 1, fast_div(rt * ROWS + ROWS - 1, c.G, p.div_group));
  const int p0 = r.kv - r.n;
  PwRange k;
  k.hi = attn_hi(c, r.kv, p0 + i1);
  k.first = min(attn_lo(c, p0 + i0), k.hi);
  k.lo = k.first & ~(KT - 1);
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

struct PwReq { int t0, n, kv; };     // a request as the scan saw it

template <int ROWS, int KT>
struct PwCursor {
  int b, h, rt, nrt, tile;
  ReqView r;
  PwRange k;
  // known: the requests of the scan, in shared memory; nullptr where there are too many
  __device__ __forceinline__ void next(const PwParams& p, const PwReq* known) {
    if (++tile < k.tiles) return;
    tile = 0;
    if (++rt == nrt) {
      rt = 0;
      do {
        if (++b >= p.c.B) return;
        r = known ? ReqView{known[b].t0, known[b].n, known[b].kv} : attn_request(p.c, b);
      } while (!pw_mine(p, r));
      nrt = pw_row_tiles<ROWS>(p, r);
    }
    k = pw_range<ROWS, KT>(p, r, rt);
  }
};

// The line of all key tiles of one key head (they are alike for all) and its shares: share g is part g / kv_heads of the line
// for key head g % kv_heads.  All arrays in shared memory.
template <int ROWS, int KT>
struct PwLine {
  const PwReq* known;        // the requests, where there is one for each thread; else nullptr
  const int* units;          // [threads] inclusive sums of tiles over each thread's `per` requests
  const int *base, *each;    // [levels + 1], [levels]: first tile of a level, tiles of its shares
  int per, per_level, levels, total, extra;   // parts per level; of the last level, the first `extra` parts have one tile more

  // part x of the line begins at; tile u belongs to part
  __device__ __forceinline__ int begin(int x) const {
    if (x >= per_level * levels) return total;
    const int k = x / per_level, i = x - k * per_level;
    return base[k] + i * each[k] + (k + 1 == levels ? min(i, extra) : 0);
  }
  __device__ __forceinline__ int part_of(int u) const {
    int k = 0;
    while (k + 1 < levels && u >= base[k + 1]) ++k;
    const int v = u - base[k], n = each[k];
    if (k + 1 < levels) return k * per_level + v / n;
    const int cut = extra * (n + 1);
    return k * per_level + (v < cut ? v / (n + 1) : extra + (v - cut) / n);
  }
  // the cursor of tile u: a search over the threads' sums, a walk over that thread's requests
  __device__ __forceinline__ void locate(const PwParams& p, PwCursor<ROWS, KT>& at, int u) const {
    const AttnCall& c = p.c;
    int a = 0, e = PW_THREADS;
    while (a < e) { const int x = (a + e) >> 1; if (units[x] > u) e = x; else a = x + 1; }
    int rest = u - (a ? units[a - 1] : 0);
    if (known) {
      at.b = a;
      at.r = ReqView{known[a].t0, known[a].n, known[a].kv};
    } else {
      for (at.b = a * per;; ++at.b) {
        at.r = attn_request(c, at.b);
        if (!pw_mine(p, at.r)) continue;
        const int hu = pw_head_units<ROWS, KT>(p, at.r);
        if (rest < hu) break;
        rest -= hu;
      }
    }
    int left = rest;
    at.nrt = pw_row_tiles<ROWS>(p, at.r);
    at.rt = 0;
    at.k = pw_range<ROWS, KT>(p, at.r, 0);
    while (left >= at.k.tiles) { left -= at.k.tiles; ++at.rt; at.k = pw_range<ROWS, KT>(p, at.r, at.rt); }
    at.tile = left;
  }
};

template <int D>
__global__ void __launch_bounds__(kJoinThreads, 2) paged_join_kernel(const __grid_constant__ AttnCall c, const __grid_constant__ JoinCall j) {
  __shared__ JoinShared<D> sh;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");       // the parts are written
  join_all<D>(c, j, &sh);
  join_wide_all<D>(c, j, &sh);
}

// status word and counters
__global__ void __launch_bounds__(256) attention_reset_kernel(uint4* ws, int n) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) ws[i] = make_uint4(0, 0, 0, 0);
}

template <int D, bool CLUSTER>
__global__ void __launch_bounds__(PW_THREADS, 1)
paged_warp_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ PwParams p) {
  using Sh = PwShape<D>;
  constexpr int ROWS = Sh::ROWS, KT = Sh::KT, HALVES = D / 64, NT = KT / 8, PW_STAGES = Sh::STAGES;
  using Cursor = PwCursor<ROWS, KT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[PW_WARPS * PW_STAGES];
  __shared__ long long s_scan[PW_WARPS];
  __shared__ int s_units[PW_THREADS], s_base[PW_MAX_LEVELS + 1], s_each[PW_MAX_LEVELS];
  __shared__ PwReq s_req[PW_THREADS];
  __shared__ float2 s_ml[PW_WARPS + 1][16];    // CLUSTER: (m, l) of each warp's and of the CTA's part
  __shared__ Cursor s_next[PW_WARPS];          // where the next share of each warp begins
  const AttnCall& c = p.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t ring = base + warp * (PW_STAGES * Sh::STAGE);
  const uint32_t full = smem_u32(s_full + warp * PW_STAGES);

  if (lane == 0) {
    for (int s = 0; s < PW_STAGES; ++s) mbar_init(full + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }

  PwLine<ROWS, KT> line{};           // not CLUSTER: the shares
  int shares = 0, first_taken = 0;   // all shares; those that the warps begin with
  int g = 0, u0, u1, g_next = 0;     // the share being computed, its tiles [u0, u1); lane 0: the share after it
  Cursor ld;
  if constexpr (CLUSTER) {
    // one item per cluster, its tiles in equal parts for the cluster's warps: no line, no workspace, nothing to prepare
    const int cs = (int)cluster_ctas(), item = (int)blockIdx.x / cs;
    ld.h = item % c.cache.kv_heads;
    ld.b = item / c.cache.kv_heads % c.B;
    ld.rt = item / c.cache.kv_heads / c.B;       // last, so that the row tiles that requests do not have come after all others
    ld.r = attn_request(c, ld.b);
    ld.nrt = pw_row_tiles<ROWS>(p, ld.r);
    if (ld.rt >= ld.nrt) {           // the whole cluster; but no grid ends before the one in front of it
      asm volatile("griddepcontrol.wait;" ::: "memory");
      return;
    }
    ld.k = pw_range<ROWS, KT>(p, ld.r, ld.rt);
    const int parts = cs * PW_WARPS, me = (int)cluster_ctarank() * PW_WARPS + warp;
    u0 = (int)((long long)ld.k.tiles * me / parts);
    u1 = (int)((long long)ld.k.tiles * (me + 1) / parts);
    ld.tile = u0;
  } else {
    // ---- the line: units before each request, all units, the shares -----------------------------------------------------
    const int per = (c.B + PW_THREADS - 1) / PW_THREADS;
    const int b_lo = min(tid * per, c.B), b_hi = min(b_lo + per, c.B);
    long long mine = 0;
    for (int b = b_lo; b < b_hi; ++b) {
      const ReqView r = attn_request(c, b);
      const int hu = pw_mine(p, r) ? pw_head_units<ROWS, KT>(p, r) : 0;
      mine += hu;
      if (per == 1) s_req[b] = PwReq{r.t0, r.n, r.kv};
    }
    const PwReq* known = per == 1 ? s_req : nullptr;
    long long incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long total_ = 0;
#pragma unroll
    for (int w = 0; w < PW_WARPS; ++w) {
      if (w < warp) incl += s_scan[w];
      total_ += s_scan[w];
    }
    s_units[tid] = (int)min(incl, 0x7fffffffLL);
    // From here on this kernel writes what the reset kernel clears; and the kernel behind it, which reads nothing that this
    // one writes before it has waited for its end, may start as SMs become free.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (total_ == 0) return;
    if (total_ > 0x7fffffffLL) {   // 2^31 tiles are 10^13 bytes of keys and values and more: the lengths cannot be meant
      if (tid == 0) atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);
      return;
    }
    const int total = (int)total_;
    // Shares: level k hands every warp one share; the levels' parts of the line are 1/2, 1/4, ... with the last two equal, so
    // the shares that are taken late are short.  A share has more tiles than the ring has slots (then at most one share's
    // beginning is in the ring besides the current one).
    const int heads = c.cache.kv_heads;
    const int per_level = min(max(1, (int)gridDim.x * PW_WARPS / heads), max(1, total / (PW_STAGES + 1)));
    int levels = 1;
    while (levels < PW_MAX_LEVELS && (total >> (levels + 1)) / per_level >= PW_FINE) ++levels;
    if (tid == 0) {
      int at = 0;
      for (int k = 0; k < levels; ++k) {
        s_base[k] = at;
        s_each[k] = (k + 1 < levels ? total >> (k + 1) : total - at) / per_level;
        at += s_each[k] * per_level;
      }
      s_base[levels] = total;
    }
    __syncthreads();
    // of the last level, the first `extra` shares have one tile more
    const int extra = total - s_base[levels - 1] - s_each[levels - 1] * per_level;
    line.known = known; line.units = s_units; line.base = s_base; line.each = s_each; line.per = per;
    line.per_level = per_level; line.levels = levels; line.total = total; line.extra = extra;
    first_taken = per_level * heads;
    shares = first_taken * levels;
    g = (int)blockIdx.x * PW_WARPS + warp;
    if (g >= first_taken) {            // a warp too many for the first level
      if (lane == 0) g = levels > 1 ? (int)atomicAdd(p.counters, 1u) + first_taken : shares;
      g = __shfl_sync(0xffffffffu, g, 0);
      if (g >= shares) return;
    }
    u0 = line.begin(g / heads);
    u1 = line.begin(g / heads + 1);
    g_next = shares;
    if (lane == 0 && levels > 1) g_next = (int)atomicAdd(p.counters, 1u) + first_taken;
    line.locate(p, ld, u0);
    ld.h = g % heads;
  }
  const PwReq* known = line.known;

  bool ok = true;
  int odd_pages = 0;
  {
    Cursor cu = ld;
    int ld_left = u1 - u0;            // tiles of the share being loaded that are not issued yet
    int ld_next_g = -1;               // the share being loaded, where that is the one after g; `shares` or more: none left

    // ---- loads: lane i issues box i: (K or V, half of the head, run of keys) ------------------------------------------
    const int runs = KT / p.box_keys;                 // boxes along the keys
    const int n_boxes = 2 * HALVES * runs;            // at most 32
    const int my_run = lane / (2 * HALVES), my_half = (lane >> 1) % HALVES, my_kv = lane & 1;
    const uint32_t my_dst = (uint32_t)(my_kv * Sh::KV_BYTES + my_half * (KT * 128) + my_run * p.box_keys * 128);
    // page of this lane's box.  A box of keys that no row sees is filled with zeros (entry -1) and its page not looked up: the page
    // behind the request's keys is not there yet, the one in front of a window may have been given back.
    auto lookup = [&](int& entry) -> int {
      const int key = ld.k.lo + ld.tile * KT + my_run * p.box_keys;
      entry = -1;
      if (lane >= n_boxes || key >= ld.k.hi || key + p.box_keys <= ld.k.first) return 0;
      const int j = fast_div(key, c.cache.page_size, p.div_page);
      entry = key - j * c.cache.page_size;
      return __ldg(c.table + (long long)ld.b * c.width + j);
    };
    uint32_t issued = 0, done = 0;
    int entry = -1, page = ld_left > 0 ? lookup(entry) : 0, st_ld = 0;
    auto issue = [&](uint32_t dep) {
      const bool none = entry < 0, odd_page = !none && (page < 0 || page >= c.cache.n_pages);
      odd_pages |= odd_page;
      if (none || odd_page) { page = c.cache.n_pages; entry = 0; }     // past the cache: zeros
      if (lane == 0) mbar_arrive_expect_tx(full + 8 * st_ld, Sh::STAGE);
      __syncwarp();
      if (lane < n_boxes)
        tma_load_4d(ring + st_ld * Sh::STAGE + my_dst + dep, my_kv ? &tm_v : &tm_k, full + 8 * st_ld, my_half * 64, entry, ld.h, page);
      if (++st_ld == PW_STAGES) st_ld = 0;
      ++issued;
      if (--ld_left > 0) ld.next(p, known);
      else {
        ld_next_g = __shfl_sync(0xffffffffu, g_next, 0);
        if (ld_next_g >= shares) return;                       // ld_left stays 0: nothing more to issue
        const int x = ld_next_g / c.cache.kv_heads, b0 = line.begin(x);
        line.locate(p, ld, b0);
        ld.h = ld_next_g - x * c.cache.kv_heads;
        ld_left = line.begin(x + 1) - b0;
        if (lane == 0) {
          s_next[warp] = ld;
          g_next = (int)atomicAdd(p.counters, 1u) + first_taken;
        }
        __syncwarp();
      }
      page = lookup(entry);
    };
    for (int s = 0; s < PW_STAGES && ld_left > 0; ++s) issue(0);
    if constexpr (CLUSTER) asm volatile("griddepcontrol.wait;" ::: "memory");   // the status word is cleared

    // ldmatrix offsets of this lane: row and swizzled chunk pair i of a 128-byte span, for K (as it lies) and V (transposed)
    uint32_t xk[4], xv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rk = (lane & 7) + ((lane >> 4) << 3), rv = lane & 15;
      xk[i] = (uint32_t)(rk * 128 + (((2 * i + ((lane >> 3) & 1)) ^ (rk & 7)) << 4));
      xv[i] = (uint32_t)(rv * 128 + (((2 * i + (lane >> 4)) ^ (rv & 7)) << 4));
    }
    float o[D / 8][4], m[2], l[2];
    uint32_t qf[D / 16][4];
    int r0 = 0, hi[2], lo[2];
    int stage = 0;
    uint32_t ph = 0;
    bool first_segment = true, fresh = true;     // of the share; of the item
    int u = u0;                                  // the tile being computed

    if (CLUSTER && u0 == u1) {                    // more warps than tiles
      m[0] = m[1] = -INFINITY;
      l[0] = l[1] = 0.f;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    } else while (true) {
      if (fresh) {
        fresh = false;
        if (!CLUSTER && first_segment && cu.tile > 0 && lane == 0) {
          // this share begins inside an item: the first share that does tells the join kernel about it
          const int item_first = u0 - cu.tile, part = g / c.cache.kv_heads - 1, first = g - c.cache.kv_heads;
          if (line.begin(part) <= item_first) {
            const int n = line.part_of(item_first + cu.k.tiles - 1) - part + 1;
            // its first part is the first share's last segment (slot 1) unless that share begins with the item; the others' first (slot 0)
            const bool many = n > kJoinShort;
            const int at = (int)atomicAdd(p.counters + (many ? 2 : 1), 1u);
            atomicMax(p.counters + 3, (uint32_t)min(ROWS, cu.r.n * c.G - cu.rt * ROWS));
            p.cuts[many ? kPagedMaxShares - 1 - at : at] = JoinCut{2 * first + (line.begin(part) == item_first ? 0 : 1), first, n, cu.r.t0, cu.rt * ROWS,
                              min(ROWS, cu.r.n * c.G - cu.rt * ROWS), cu.h, 0};
          }
        }
        r0 = cu.rt * ROWS;
#pragma unroll
        for (int i = 0; i < 2; ++i) {                 // this lane's rows: the keys they see
          const int gr = r0 + (lane >> 2) + 8 * i, tok = fast_div(gr, c.G, p.div_group);
          const int pos = cu.r.kv - cu.r.n + min(tok, cu.r.n - 1);
          hi[i] = attn_hi(c, cu.r.kv, pos);
          lo[i] = attn_lo(c, pos);
          const uint32_t* q = reinterpret_cast<const uint32_t*>(c.q + (long long)(cu.r.t0 + tok) * c.q_ts +
                                                                (long long)(cu.h * c.G + gr - tok * c.G) * c.q_hs) + (lane & 3);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            qf[k][i] = tok < cu.r.n ? __ldg(q + 8 * k) : 0u;
            qf[k][2 + i] = tok < cu.r.n ? __ldg(q + 8 * k + 4) : 0u;
          }
          m[i] = tok < cu.r.n ? -INFINITY : 0.f;      // rows that are none need no maximum
          l[i] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * stage, ph, c.status, p.wait_limit))) { ok = false; break; }
      const uint32_t sk = ring + stage * Sh::STAGE, sv = sk + Sh::KV_BYTES;

      const int k0 = cu.k.lo + cu.tile * KT;
      const bool partial = k0 + KT > cu.k.all_hi || k0 < cu.k.all_lo;
      bool odd = false;                                    // a NaN or infinity in V of a tile with masked keys
      if (partial) {
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
        __syncwarp();                                      // every lane's fragments hold what other lanes have cleaned (a vote orders no memory)
      }

      // scores: fragment n covers keys 8 n .. 8 n + 7 (lane: rows lane / 4 and + 8, keys 2 (lane % 4) + {0, 1}); with few
      // fragments, even and odd steps of the contraction are summed apart, so that an MMA does not wait for the one before
      constexpr int SPLIT = NT < 4 ? 2 : 1;
      float s[NT][4], s2[SPLIT == 2 ? NT : 1][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
        if (SPLIT == 2) s2[n][0] = s2[n][1] = s2[n][2] = s2[n][3] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
#pragma unroll
        for (int n2 = 0; n2 < NT / 2; ++n2) {
          uint32_t kf[4];
          frag_ldm4(kf, sk + xk[k & 3] + (uint32_t)((k >> 2) * (KT * 128) + n2 * 2048));
          if (SPLIT == 2 && (k & 1)) {
            frag_mma(s2[SPLIT == 2 ? 2 * n2 : 0], qf[k], kf[0], kf[1]);
            frag_mma(s2[SPLIT == 2 ? 2 * n2 + 1 : 0], qf[k], kf[2], kf[3]);
          } else {
            frag_mma(s[2 * n2], qf[k], kf[0], kf[1]);
            frag_mma(s[2 * n2 + 1], qf[k], kf[2], kf[3]);
          }
        }
      }
      // V's fragments are on their way during the softmax
      uint32_t vf[KT / 16][D / 16][4];
#pragma unroll
      for (int k = 0; k < KT / 16; ++k)
#pragma unroll
        for (int n2 = 0; n2 < D / 16; ++n2) frag_ldm4t(vf[k][n2], sv + xv[n2 & 3] + (uint32_t)((n2 >> 2) * (KT * 128) + k * 2048));
      if (SPLIT == 2) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][e] += s2[SPLIT == 2 ? n : 0][e];
      }
      if (partial) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = k0 + n * 8 + 2 * (lane & 3) + (e & 1);
            if (j >= hi[e >> 1] || j < lo[e >> 1]) s[n][e] = -INFINITY;
          }
      }
      // Weights with the m there is; only where a row has none yet, or where a sum shows that the scores have outgrown m, the
      // maximum is looked for and they are done again.  Weights of 2^10 are as exact as weights of 1; but what o can hold shrinks by
      // that factor (with 2^40 here, values of 2^90 overflowed).
      float w[NT][4], sum[2];
      bool again = __any_sync(0xffffffffu, m[0] == -INFINITY || m[1] == -INFINITY);
#pragma unroll 1
      for (;;) {
        if (again) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = s[0][2 * i];
#pragma unroll
            for (int n = 0; n < NT; ++n) x = fmaxf(x, fmaxf(s[n][2 * i], s[n][2 * i + 1]));
            x = fmaxf(m[i], x * p.scale2);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            f[i] = m[i] == x ? 1.f : fast_exp2(m[i] - x);
            m[i] = x;
            l[i] *= f[i];
          }
#pragma unroll
          for (int n = 0; n < D / 8; ++n) { o[n][0] *= f[0]; o[n][1] *= f[0]; o[n][2] *= f[1]; o[n][3] *= f[1]; }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float b = m[i] == -INFINITY ? 0.f : m[i];      // nothing seen yet: all weights are 2^-inf = 0
          sum[i] = 0.f;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            w[n][2 * i] = fast_exp2(fmaf(s[n][2 * i], p.scale2, -b));
            w[n][2 * i + 1] = fast_exp2(fmaf(s[n][2 * i + 1], p.scale2, -b));
            sum[i] += w[n][2 * i] + w[n][2 * i + 1];
          }
        }
        if (again || !__any_sync(0xffffffffu, !(sum[0] < PW_OUTGROWN) || !(sum[1] < PW_OUTGROWN))) break;
        again = true;
      }
      l[0] += sum[0];                                          // this lane's part; joined over the quad at the end
      l[1] += sum[1];
#pragma unroll
      for (int k = 0; k < KT / 16; ++k) {
        uint32_t a[4];
        a[0] = pack_bf16x2(w[2 * k][0], w[2 * k][1]);
        a[1] = pack_bf16x2(w[2 * k][2], w[2 * k][3]);
        a[2] = pack_bf16x2(w[2 * k + 1][0], w[2 * k + 1][1]);
        a[3] = pack_bf16x2(w[2 * k + 1][2], w[2 * k + 1][3]);
#pragma unroll
        for (int n2 = 0; n2 < D / 16; ++n2) {
          frag_mma(o[2 * n2], a, vf[k][n2][0], vf[k][n2][1]);
          frag_mma(o[2 * n2 + 1], a, vf[k][n2][2], vf[k][n2][3]);
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
            for (int i = 0; i < 2; ++i) {
              if (j >= hi[i] || j < lo[i]) continue;
              if ((w & 0x7f80u) == 0x7f80u) o[n][2 * i] += v0;
              if ((w & 0x7f800000u) == 0x7f800000u) o[n][2 * i + 1] += v1;
            }
          }
        }
      }
      // The slot is free when every lane's fragments have been read.  Each was an operand of an MMA whose result is in o, so
      // the copy's address is made to depend on all of o: it cannot be issued while a load is still on its way.
      ++done;
      if (ld_left > 0) {
        uint32_t dep = 0;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) dep |= __float_as_uint(o[n][0]);
        __syncwarp();
        issue(dep & p.zero);
      }
      if (++stage == PW_STAGES) { stage = 0; ph ^= 1u; }

      // ---- end of an item, or of this share's part of it --------------------------------------------------------------
      if (CLUSTER && u + 1 == u1) break;
      if (!CLUSTER && (cu.tile + 1 == cu.k.tiles || u + 1 == u1)) {
        const int item_first = u - cu.tile;
        const bool whole = item_first >= u0 && item_first + cu.k.tiles <= u1;
        const long long slot = 2 * g + (first_segment ? 0 : 1);   // of partial results
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float sum = l[i];
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          const int row = (lane >> 2) + 8 * i, gr = r0 + row, tok = fast_div(gr, c.G, p.div_group);
          if (tok >= cu.r.n) continue;
          if (whole) {
            const int head = cu.h * c.G + gr - tok * c.G;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            __nv_bfloat16* out = c.out + (long long)(cu.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + 2 * (lane & 3);
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
              *reinterpret_cast<uint32_t*>(out + 8 * n) = pack_bf16x2(o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
            if (c.lse && (lane & 3) == 0)
              c.lse[(long long)(cu.r.t0 + tok) * c.H + head] = sum == 0.f ? -INFINITY : (m[i] + log2f(sum)) * PW_LN2;
          } else {
            float* d = p.part_o + (slot * ROWS + row) * D + 2 * (lane & 3);
#pragma unroll
            for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(d + 8 * n) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            if ((lane & 3) == 0) *reinterpret_cast<float2*>(p.part_ml + (slot * ROWS + row) * 2) = make_float2(m[i], sum);
          }
        }
        first_segment = false;
        fresh = true;
      }
      if (++u < u1) { cu.next(p, known); continue; }
      // the next share: its tiles are on their way already
      if (ld_next_g < 0 || ld_next_g >= shares) break;
      g = ld_next_g;
      ld_next_g = -1;
      u = u0 = line.begin(g / c.cache.kv_heads);
      u1 = line.begin(g / c.cache.kv_heads + 1);
      cu = s_next[warp];
      first_segment = fresh = true;
    }
    if (!ok) {   // give copies already in flight a bounded chance to land before the CTA exits
      for (uint32_t j = done; j < issued; ++j) mbar_wait(full + 8 * (j % PW_STAGES), (j / PW_STAGES) & 1u, c.status, p.wait_limit);
    }
    if (__any_sync(0xffffffffu, odd_pages) && lane == 0) atomicExch(c.status, (int)QBLORA_ERR_INVALID_ARG);

    if constexpr (CLUSTER) {
      // ---- the warps' parts become the CTA's in its shared memory, the CTAs' the item's through the cluster's ------------
      static_assert(16 * D * 4 <= Sh::STAGE, "a warp's part fits a slot of its ring, the CTA's the next slot of the first ring");
      const int r0 = cu.rt * ROWS, rows = min(ROWS, cu.r.n * c.G - r0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = l[i];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const int row = (lane >> 2) + 8 * i;
        float* d = reinterpret_cast<float*>(smem_raw + (ring - raw)) + row * D + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(d + 8 * n) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
        if ((lane & 3) == 0) s_ml[warp][row] = make_float2(m[i], sum);
      }
      __syncthreads();
      constexpr int LANES = D / 4;
      const uint32_t cta_part = base + Sh::STAGE;
      for (int i = tid; i < rows * LANES; i += PW_THREADS) {
        const int row = i / LANES, col = i % LANES;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < PW_WARPS; ++w) M = fmaxf(M, s_ml[w][row].x);
        const float b = M == -INFINITY ? 0.f : M;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < PW_WARPS; ++w) {
          const float2 ml = s_ml[w][row];
          const float f = fast_exp2(ml.x - b);
          const float4 v = *reinterpret_cast<const float4*>(smem_raw + (base - raw) + w * (PW_STAGES * Sh::STAGE) + (row * D + 4 * col) * 4);
          L += ml.y * f;
          acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
        }
        *reinterpret_cast<float4*>(smem_raw + (cta_part - raw) + (row * D + 4 * col) * 4) = acc;
        if (col == 0) s_ml[PW_WARPS][row] = make_float2(M, L);
      }
      cluster_sync_all();
      const int cs = (int)cluster_ctas(), rank = (int)cluster_ctarank();
      const uint32_t cta_ml = smem_u32(&s_ml[PW_WARPS][0]);
      for (int i = tid; i < rows * LANES; i += PW_THREADS) {
        const int row = i / LANES, col = i % LANES;
        if (row % cs != rank) continue;
        float M = -INFINITY, L = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int x = 0; x < cs; ++x) {
          const float2 ml = ld_cluster2(map_to_cta(cta_ml + 8 * row, x));
          const float4 v = ld_cluster4(map_to_cta(cta_part + (row * D + 4 * col) * 4, x));
          const float mn = fmaxf(M, ml.x), b = mn == -INFINITY ? 0.f : mn, fa = fast_exp2(M - b), fb = fast_exp2(ml.x - b);
          M = mn;
          L = L * fa + ml.y * fb;
          acc.x = acc.x * fa + v.x * fb; acc.y = acc.y * fa + v.y * fb;
          acc.z = acc.z * fa + v.z * fb; acc.w = acc.w * fa + v.w * fb;
        }
        const int gr = r0 + row, tok = fast_div(gr, c.G, p.div_group), head = cu.h * c.G + gr - tok * c.G;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        *reinterpret_cast<uint2*>(c.out + (long long)(cu.r.t0 + tok) * c.o_ts + (long long)head * c.o_hs + 4 * col) =
            make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        if (c.lse && col == 0) c.lse[(long long)(cu.r.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * PW_LN2;
      }
      cluster_sync_all();              // no CTA leaves while another reads its part
    }
  }
}

// CTAs of the line: one per SM; 0 without a device
int pw_ctas() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return std::min(sms, kPagedMaxSms);
}

// where the workspace holds what
template <int D>
void pw_workspace(PwParams* p, char* counters, char* scratch) {
  constexpr int ROWS = PwShape<D>::ROWS;
  p->counters = reinterpret_cast<uint32_t*>(counters);
  p->part_ml = reinterpret_cast<float*>(scratch);
  p->part_o = p->part_ml + (size_t)2 * kPagedMaxShares * ROWS * 2;
  p->cuts = reinterpret_cast<JoinCut*>(p->part_o + (size_t)2 * kPagedMaxShares * ROWS * D);
}

template <int D>
int pw_launch(PwParams p, const CUtensorMap& tk, const CUtensorMap& tv, char* counters, char* scratch, cudaStream_t st) {
  using Sh = PwShape<D>;
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  auto kernel = paged_warp_kernel<D, false>;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
    attr_set[dev].store(true, std::memory_order_release);
  }
  pw_workspace<D>(&p, counters, scratch);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)pw_ctas());
  cfg.blockDim = dim3(PW_THREADS);
  cfg.dynamicSmemBytes = Sh::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, kernel, tk, tv, p));
  count_launch();
  return QBLORA_OK;
}

template <int D>
int pw_launch_join(const AttnCall& c, char* counters, char* scratch, char* wide_counters, char* wide_scratch, cudaStream_t st) {
  int dev = 0, sms = 0;
  QB_CUDA(cudaGetDevice(&dev));
  QB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  PwParams p{};
  pw_workspace<D>(&p, counters, scratch);
  JoinCall j{p.counters + 1, p.cuts, p.part_o, p.part_ml, PwShape<D>::ROWS, fast_div_magic((uint32_t)c.G)};
  tc_attention_join(D, wide_counters, wide_scratch, &j);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * sms));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  QB_CUDA(cudaLaunchKernelEx(&cfg, paged_join_kernel<D>, c, j));
  count_launch();
  return QBLORA_OK;
}

// Clusters of `1 << i` CTAs that the device holds at once, for i = 0 ... 4; 0 where it does not take that size.
struct PwResident { int n[5]; };

template <int D>
int pw_resident(const PwResident** out) {
  using Sh = PwShape<D>;
  static PwResident table[64];
  static std::atomic<bool> ready[64];
  static std::mutex once;
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  if (!ready[dev].load(std::memory_order_acquire)) {
    std::lock_guard<std::mutex> hold(once);
    auto kernel = paged_warp_kernel<D, true>;
    QB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
    const bool wide = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    for (int i = 0; i < 5; ++i) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(1u << i);
      cfg.blockDim = dim3(PW_THREADS);
      cfg.dynamicSmemBytes = Sh::SMEM;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim = {1u << i, 1, 1};
      cfg.attrs = attr; cfg.numAttrs = 1;
      int n = 0;
      if ((i == 4 && !wide) || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) n = 0;
      table[dev].n[i] = n;
    }
    (void)cudaGetLastError();
    ready[dev].store(true, std::memory_order_release);
  }
  *out = &table[dev];
  return QBLORA_OK;
}

// No request has more rows than the call.
int pw_row_tiles_bound(const AttnCall& c) { return (int)((c.T * c.G + 15) / 16); }

// CTAs per cluster; 0: not this form.  The largest size with which all items are resident at once (a second wave costs more
// than the split gains: 16 items of 513 keys, clusters of 4 11.1 us, of 8 15.3 us).  Then the lengths, which the host does not
// know, are bounded by the table's width, because a cluster's item has only its own SMs and the line has them all.  Measured
// (D 128, line / cluster):
//   one request: 8 heads, 2 keys 15.7 / 10.3 us, 513 14.9 / 10.3, 8192 34 / 18.5, 32768 62 / 43;  2 heads, 32768 86 / 28;
//                16 heads (clusters of 4), 8192 30 / 26.6, 32768 68 / 76;
//   several, which may be uneven -- all keys in one of them at worst: 4 x 8 heads (clusters of 4), 8192 41 / 33, worst 34 / 27;
//                at 32768 115 / 98, worst 62 / 75;  8 x 8 heads (2), 2048 22.5 / 18.5;  8 x 16 heads (1), 2048 36 / 31.
int pw_cluster_size(const AttnCall& c, const PwResident& r) {
  const int64_t tiles = std::min<int64_t>((int64_t)c.B * pw_row_tiles_bound(c), c.B + c.T * c.G / 16);   // of all requests, at most
  const int64_t items = tiles * c.cache.kv_heads, keys = (int64_t)c.width * c.cache.page_size;
  for (int i = 4; i >= 0; --i)
    if (items <= r.n[i]) return keys <= ((c.B == 1 ? 4096LL : 2048LL) << i) ? 1 << i : 0;
  return 0;
}

template <int D>
int pw_launch_cluster(const PwParams& p, const CUtensorMap& tk, const CUtensorMap& tv, int cs, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.c.B * p.c.cache.kv_heads * pw_row_tiles_bound(p.c) * cs));
  cfg.blockDim = dim3(PW_THREADS);
  cfg.dynamicSmemBytes = PwShape<D>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)cs, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  QB_CUDA(cudaLaunchKernelEx(&cfg, paged_warp_kernel<D, true>, tk, tv, p));
  count_launch();
  return QBLORA_OK;
}

int pw_params(const AttnCall& c, PwParams* p, CUtensorMap* tk, CUtensorMap* tv) {
  p->c = c;
  p->scale2 = c.scale * 1.4426950408889634f;
  p->box_keys = std::min(c.cache.page_size, c.D == 64 ? 32 : 16);
  p->div_page = fast_div_magic((uint32_t)c.cache.page_size);
  p->div_group = fast_div_magic((uint32_t)c.G);
  p->wait_limit = wait_limit_cycles();
  return make_cache_maps(c, p->box_keys, tk, tv);
}

}  // namespace

static_assert(PW_WARPS == kPagedWarps, "shares per SM");

int launch_attention_reset(void* ws, size_t bytes, cudaStream_t st) {
  const int n = (int)(bytes / 16);
  static_assert(kAttnResetBytes % 16 == 0, "whole words");
  attention_reset_kernel<<<(n + 255) / 256, 256, 0, st>>>(static_cast<uint4*>(ws), n);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

bool paged_warp_supported(const AttnCall& c) {
  if ((c.D != 64 && c.D != 128) || !(c.scale > 0.f)) return false;
  // every warp of the line begins with one share of the first level, which has at least one share for each key head: with more
  // key heads than warps nobody would take the last ones
  if (c.cache.kv_heads > pw_ctas() * kPagedWarps) return false;
  const int kt = c.D == 64 ? 32 : 16, pg = c.cache.page_size;
  // a tile is whole boxes of one page each; at most 32 boxes, one per lane
  return pg % 8 == 0 && (pg <= kt ? kt % pg == 0 : pg % kt == 0);
}

int launch_paged_warp(const AttnCall& c, int narrow_rows, char* counters, char* scratch, cudaStream_t st) {
  PwParams p{};
  CUtensorMap tk, tv;
  const int rc = pw_params(c, &p, &tk, &tv);
  if (rc) return rc;
  p.narrow_rows = narrow_rows;
  return c.D == 64 ? pw_launch<64>(p, tk, tv, counters, scratch, st) : pw_launch<128>(p, tk, tv, counters, scratch, st);
}

int launch_paged_join(const AttnCall& c, char* counters, char* scratch, char* wide_counters, char* wide_scratch, cudaStream_t st) {
  return c.D == 64 ? pw_launch_join<64>(c, counters, scratch, wide_counters, wide_scratch, st)
                   : pw_launch_join<128>(c, counters, scratch, wide_counters, wide_scratch, st);
}

int paged_cluster_size(const AttnCall& c, int* size) {
  *size = 0;
  if (!paged_warp_supported(c) || c.T * c.G > 32) return QBLORA_OK;
  const PwResident* r = nullptr;
  const int rc = c.D == 64 ? pw_resident<64>(&r) : pw_resident<128>(&r);
  if (rc) return rc;
  *size = pw_cluster_size(c, *r);
  return QBLORA_OK;
}

int launch_paged_cluster(const AttnCall& c, int size, cudaStream_t st) {
  PwParams p{};
  CUtensorMap tk, tv;
  const int rc = pw_params(c, &p, &tk, &tv);
  if (rc) return rc;
  return c.D == 64 ? pw_launch_cluster<64>(p, tk, tv, size, st) : pw_launch_cluster<128>(p, tk, tv, size, st);
}

}  // namespace qb
