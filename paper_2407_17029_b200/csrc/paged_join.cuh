// Joining of partial attention results: items (row tiles of one request and key head) whose keys several warps of
// paged_warp.cu or several CTAs of tc_attn.cu have worked on.
//
// A part is (m, l, o) per row: running maximum in base 2, sum of weights, sum of weighted values, over some of the item's keys.
// With M = max m_i:  l = sum l_i 2^(m_i - M),  o = sum o_i 2^(m_i - M),  out = o / l,  lse = (M + log2 l) ln 2.
// Parts are taken in a fixed order, so results do not depend on timing (the order of the lists of cut items does, and has no
// influence on them).  Nothing here waits for another CTA: all parts are there when the kernel starts.
//
// What bounds it is latency: a row's parts are a few KB that lie in L2.  So a row of a short item is one warp's, with 16 parts in
// flight, rows go evenly over all warps of the device, and only an item of more than kJoinShort parts takes a CTA per row.  Of
// tc_attn.cu's row tiles a warp takes 32 rows x 32 columns, a lane per row, as its parts lie.  (Joined in tc_attn.cu by the CTA that
// came last, two or three parts of 128 x 128 took 14 us at the end of a call; here about 3, all of them side by side.)
#pragma once
#include "mma_frag.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"

namespace qb {

struct JoinAcc { float M, L; float4 o; };

// Parts a, a + step, ... below x.n of one row: this lane's 4 columns.
template <int D, int PB>
__device__ __forceinline__ JoinAcc join_parts(const AttnCall& c, const JoinCall& j, const JoinCut& x, int row, int col, int a, int step) {
  JoinAcc r{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  for (int i0 = a; i0 < x.n; i0 += PB * step) {
    float2 ml[PB];
    float4 v[PB];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      const int k = i0 + i * step;
      if (k < x.n) {
        const long long at = (long long)(k == 0 ? x.slot0 : 2 * (x.first + k * c.cache.kv_heads)) * j.rows_per_slot + row;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(j.part_ml + at * 2));
        v[i] = __ldcg(reinterpret_cast<const float4*>(j.part_o + at * D + col));
      }
    }
    float mn = r.M;
#pragma unroll
    for (int i = 0; i < PB; ++i) mn = fmaxf(mn, ml[i].x);
    const float b = mn == -INFINITY ? 0.f : mn, f = fast_exp2(r.M - b);
    r.M = mn;
    r.L *= f; r.o.x *= f; r.o.y *= f; r.o.z *= f; r.o.w *= f;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const float g = fast_exp2(ml[i].x - b);
      r.L += ml[i].y * g;
      r.o.x += v[i].x * g; r.o.y += v[i].y * g; r.o.z += v[i].z * g; r.o.w += v[i].w * g;
    }
  }
  return r;
}

__device__ __forceinline__ void join_store(const AttnCall& c, const JoinCall& j, const JoinCut& x, int row, int col, const JoinAcc& r) {
  const int gr = x.r0 + row, tok = fast_div(gr, c.G, j.div_group), head = x.h * c.G + gr - tok * c.G;
  const float inv = r.L == 0.f ? 0.f : 1.f / r.L;
  *reinterpret_cast<uint2*>(c.out + (long long)(x.t0 + tok) * c.o_ts + (long long)head * c.o_hs + col) =
      make_uint2(ptx::pack_bf16x2(r.o.x * inv, r.o.y * inv), ptx::pack_bf16x2(r.o.z * inv, r.o.w * inv));
  if (c.lse && col == 0)
    c.lse[(long long)(x.t0 + tok) * c.H + head] = r.L == 0.f ? -INFINITY : (r.M + log2f(r.L)) * 0.69314718055994530942f;
}

// All cut items.  Called by all threads of the CTA.
template <int D>
struct JoinShared { float2 ml[kJoinThreads]; float4 o[8 * kJoinThreads]; };

struct JoinWideAcc { float M, L; float4 o[8]; };
// Parts a, a + step, ... below x.n of one row: 32 columns.
template <int D>
__device__ __forceinline__ void join_wide_parts(const JoinCall& j, const JoinCut& x, int row, int cg, int a, int step, JoinWideAcc& r) {
  constexpr int PB = 2;
  r.M = -INFINITY;
  r.L = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) r.o[q] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = a; i0 < x.n; i0 += PB * step) {
    float2 ml[PB];
    float4 v[PB][8];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const int k = i0 + i * step;
      ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[i][q] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k < x.n) {
        const long long slot = (k == 0 ? 2LL * x.slot0 : 4LL * (x.first + k)) + x.tile;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(j.wide_ml) + slot * 128 + row);
        const float4* o = reinterpret_cast<const float4*>(j.wide_o) + (slot * (D / 4) + cg * 8) * 128 + row;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[i][q] = __ldcg(o + q * 128);
      }
    }
    float mn = r.M;
#pragma unroll
    for (int i = 0; i < PB; ++i) mn = fmaxf(mn, ml[i].x);
    const float b = mn == -INFINITY ? 0.f : mn, f = fast_exp2(r.M - b);
    r.M = mn;
    r.L *= f;
#pragma unroll
    for (int q = 0; q < 8; ++q) { r.o[q].x *= f; r.o[q].y *= f; r.o[q].z *= f; r.o[q].w *= f; }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const float g = fast_exp2(ml[i].x - b);
      r.L += ml[i].y * g;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        r.o[q].x += v[i][q].x * g; r.o[q].y += v[i][q].y * g; r.o[q].z += v[i][q].z * g; r.o[q].w += v[i][q].w * g;
      }
    }
  }
}
__device__ __forceinline__ void join_wide_store(const AttnCall& c, const JoinCall& j, const JoinCut& x, int row, int cg, const JoinWideAcc& r) {
  if (row >= x.rows) return;
  const int tok = fast_div(row, c.G, j.div_group), head = x.h * c.G + row - tok * c.G;
  const float inv = r.L == 0.f ? 0.f : 1.f / r.L;
  uint4* out = reinterpret_cast<uint4*>(c.out + (long long)(x.t0 + tok) * c.o_ts + (long long)head * c.o_hs + cg * 32);
#pragma unroll
  for (int q = 0; q < 4; ++q)
    out[q] = make_uint4(ptx::pack_bf16x2(r.o[2 * q].x * inv, r.o[2 * q].y * inv), ptx::pack_bf16x2(r.o[2 * q].z * inv, r.o[2 * q].w * inv),
                        ptx::pack_bf16x2(r.o[2 * q + 1].x * inv, r.o[2 * q + 1].y * inv), ptx::pack_bf16x2(r.o[2 * q + 1].z * inv, r.o[2 * q + 1].w * inv));
  if (c.lse && cg == 0)
    c.lse[(long long)(x.t0 + tok) * c.H + head] = r.L == 0.f ? -INFINITY : (r.M + log2f(r.L)) * 0.69314718055994530942f;
}
template <int D>
__device__ __forceinline__ void join_wide_all(const AttnCall& c, const JoinCall& j, JoinShared<D>* sh) {
  constexpr int COLS = D / 32, PIECES = 4 * COLS, WARPS = kJoinThreads / 32;     // a row tile's pieces of 32 rows x 32 columns
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_short = (int)__ldcg(j.wide_counts), n_long = (int)__ldcg(j.wide_counts + 1);
  for (int i = warp * gridDim.x + blockIdx.x; i < n_short * PIECES; i += WARPS * gridDim.x) {
    const int piece = i / n_short, cg = piece % COLS, r0 = piece / COLS * 32;
    const JoinCut x = j.wide_cuts[i - piece * n_short];
    if (r0 >= x.rows) continue;
    JoinWideAcc r;
    join_wide_parts<D>(j, x, r0 + lane, cg, 0, 1, r);
    join_wide_store(c, j, x, r0 + lane, cg, r);
  }
  for (int i = blockIdx.x; i < n_long * PIECES; i += gridDim.x) {
    const int piece = i / n_long, cg = piece % COLS, r0 = piece / COLS * 32;
    const JoinCut x = j.wide_cuts[2 * kWideMaxShares - 1 - (i - piece * n_long)];
    if (r0 >= x.rows) continue;                               // all threads of the CTA alike
    JoinWideAcc r;
    join_wide_parts<D>(j, x, r0 + lane, cg, warp, WARPS, r);
    sh->ml[tid] = make_float2(r.M, r.L);
#pragma unroll
    for (int q = 0; q < 8; ++q) sh->o[q * kJoinThreads + tid] = r.o[q];
    __syncthreads();
    if (warp == 0) {
      r.M = -INFINITY;
      for (int w = 0; w < WARPS; ++w) r.M = fmaxf(r.M, sh->ml[w * 32 + lane].x);
      const float b = r.M == -INFINITY ? 0.f : r.M;
      r.L = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) r.o[q] = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < WARPS; ++w) {
        const float2 ml = sh->ml[w * 32 + lane];
        const float f = fast_exp2(ml.x - b);
        r.L += ml.y * f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float4 v = sh->o[q * kJoinThreads + w * 32 + lane];
          r.o[q].x += v.x * f; r.o[q].y += v.y * f; r.o[q].z += v.z * f; r.o[q].w += v.w * f;
        }
      }
      join_wide_store(c, j, x, r0 + lane, cg, r);
    }
    __syncthreads();
  }
}

template <int D>
__device__ __forceinline__ void join_all(const AttnCall& c, const JoinCall& j, JoinShared<D>* sh) {
  constexpr int LANES = D / 4, GROUPS = kJoinThreads / LANES;    // lanes of a row; rows that a CTA works on side by side
  const int tid = threadIdx.x, grp = tid / LANES, lane = tid % LANES, col = 4 * lane;
  const int n_short = (int)__ldcg(j.counts), n_long = (int)__ldcg(j.counts + 1), rows = (int)__ldcg(j.counts + 2);
  for (long long i = (long long)grp * gridDim.x + blockIdx.x; i < (long long)n_short * rows; i += (long long)GROUPS * gridDim.x) {
    const int row = (int)(i / n_short);
    const JoinCut x = j.cuts[i - (long long)row * n_short];
    if (row < x.rows) join_store(c, j, x, row, col, join_parts<D, 16>(c, j, x, row, col, 0, 1));
  }
  for (long long i = blockIdx.x; i < (long long)n_long * rows; i += gridDim.x) {
    const int row = (int)(i / n_long);
    const JoinCut x = j.cuts[kPagedMaxShares - 1 - (i - (long long)row * n_long)];
    if (row >= x.rows) continue;                              // all threads of the CTA alike
    const JoinAcc a = join_parts<D, 8>(c, j, x, row, col, grp, GROUPS);
    sh->o[tid] = a.o;
    if (lane == 0) sh->ml[grp] = make_float2(a.M, a.L);
    __syncthreads();
    if (grp == 0) {
      JoinAcc r{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      for (int g = 0; g < GROUPS; ++g) r.M = fmaxf(r.M, sh->ml[g].x);
      const float b = r.M == -INFINITY ? 0.f : r.M;
      for (int g = 0; g < GROUPS; ++g) {
        const float f = fast_exp2(sh->ml[g].x - b);
        const float4 v = sh->o[g * LANES + lane];
        r.L += sh->ml[g].y * f;
        r.o.x += v.x * f; r.o.y += v.y * f; r.o.z += v.z * f; r.o.w += v.w * f;
      }
      join_store(c, j, x, row, col, r);
    }
    __syncthreads();
  }
}

}  // namespace qb
