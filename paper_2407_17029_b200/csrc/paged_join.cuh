// Joining of partial attention results: items (row tiles of one request and key head) whose keys several warps of
// paged_warp.cu have worked on.
//
// A part is (m, l, o) per row: running maximum in base 2, sum of weights, sum of weighted values, over some of the item's keys.
// With M = max m_i:  l = sum l_i 2^(m_i - M),  o = sum o_i 2^(m_i - M),  out = o / l,  lse = (M + log2 l) ln 2.
// Parts are taken in share order, so results do not depend on timing.
#pragma once
#include "mma_frag.cuh"
#include "serving.cuh"
#include "tc_ptx.cuh"

namespace qb {

// Rows rb .. (STEP = 128 / D of them, below r1) of one item by one warp, PB parts in flight, D / 4 lanes a row.
template <int D, int PB>
__device__ __forceinline__ void join_rows(const AttnCall& c, const JoinCall& j, const JoinCut& x, int rb, int r1) {
  constexpr int LANES = D / 4;
  const int lane = threadIdx.x & 31, col = (lane % LANES) * 4, row = rb + lane / LANES;
  if (row >= r1) return;
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < x.n; i0 += PB) {
    float2 ml[PB];
    float4 v[PB];
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      const int k = i0 + i;
      if (k < x.n) {
        const long long at = (long long)(k == 0 ? x.slot0 : 2 * (x.first + k)) * j.rows_per_slot + row;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(j.part_ml + at * 2));
        v[i] = __ldcg(reinterpret_cast<const float4*>(j.part_o + at * D + col));
      }
    }
    float mn = M;
#pragma unroll
    for (int i = 0; i < PB; ++i) mn = fmaxf(mn, ml[i].x);
    const float b = mn == -INFINITY ? 0.f : mn, f = fast_exp2(M - b);
    M = mn;
    L *= f; acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const float g = fast_exp2(ml[i].x - b);
      L += ml[i].y * g;
      acc.x += v[i].x * g; acc.y += v[i].y * g; acc.z += v[i].z * g; acc.w += v[i].w * g;
    }
  }
  const int gr = x.r0 + row, tok = fast_div(gr, c.G, j.div_group), head = x.h * c.G + gr - tok * c.G;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  *reinterpret_cast<uint2*>(c.out + (long long)(x.t0 + tok) * c.o_ts + (long long)head * c.o_hs + col) =
      make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv));
  if (c.lse && col == 0) c.lse[(long long)(x.t0 + tok) * c.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994530942f;
}

// All cut items, spread over the grid by share border and quarter of the rows (neighbouring CTAs get the quarters of one
// item); the pieces of a CTA go round its warps, so that they run side by side.  Called by all threads of the CTA.
constexpr int kJoinList = (4 * kPagedMaxShares + 63) / 64;
struct JoinShared { int n; short quarter[kJoinList]; JoinCut cut[kJoinList]; };
template <int D, int THREADS>
__device__ __forceinline__ void join_all(const AttnCall& c, const JoinCall& j, JoinShared* sh) {
  constexpr int STEP = 32 / (D / 4);
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) sh->n = 0;
  __syncthreads();
  for (int i = blockIdx.x + tid * gridDim.x; i < 4 * j.borders; i += THREADS * gridDim.x) {
    const int g = i >> 2;
    if (__ldcg(j.flags + g)) {
      const JoinCut x = j.cuts[g];
      const int rows = (x.rows + 3) / 4, r = (i & 3) * rows;        // this quarter's rows
      if (r < x.rows) {
        const int at = atomicAdd(&sh->n, 1);
        sh->cut[at] = x;
        sh->quarter[at] = (short)r;
      }
    }
  }
  __syncthreads();
  int next = warp;                                         // pieces until this warp's next one
  for (int i = 0; i < sh->n; ++i) {
    const JoinCut& x = sh->cut[i];
    const int r0 = sh->quarter[i], r1 = min(x.rows, r0 + (x.rows + 3) / 4);
    for (int rb = r0; rb < r1; rb += STEP) {
      if (next-- > 0) continue;
      next = THREADS / 32 - 1;
      join_rows<D, 8>(c, j, x, rb, r1);
    }
  }
}

}  // namespace qb
