// The tiles of rows that a plan gives every adapter, found by each CTA for itself.
#pragma once
#include "adapters.cuh"

namespace qb {

// ---- adapters' rows: where they lie in the workspace, and their tiles ------------------------------------------------------------
inline size_t ag_table_bytes(int n) { return (size_t)2 * (n + 1) * 4; }
struct AgGroups {
  const uint32_t* pad;      // [n + 1] first row of each adapter in the workspace, multiples of 16
  const uint32_t* tile;     // [n + 1] tiles in front of it
  int kept;                 // adapters whose rows lie in the workspace: all, for a plan whose offsets rise
};
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }   // both below 2^31

// by the whole CTA; s: 2 (n + 1) words of shared memory
// tn: rows of a tile
template <int NT>
__device__ __forceinline__ AgGroups ag_groups(const AdaptersCall& c, uint32_t* s, uint32_t rows_there, int tn) {
  __shared__ uint32_t s_part[2][NT / 32];
  __shared__ int s_kept;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = c.k.n;
  uint32_t *pad = s, *tile = s + n + 1;
  const int per = (n + NT - 1) / NT, lo = min(tid * per, n), hi = min(lo + per, n);
  uint32_t mine = 0, tiles = 0;
  for (int a = lo; a < hi; ++a) {
    const uint32_t rows = (uint32_t)max(plan_start(c, a + 1) - plan_start(c, a), 0);
    const uint32_t p = (min(rows, 0x7ffffff0u) + 15u) & ~15u, t = (rows + tn - 1) / tn;
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

// Values as parts: a number in fp32 as the sum of bf16 numbers, each the rounding of what the ones before leave.
__device__ __forceinline__ float ag_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float ag_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace qb
