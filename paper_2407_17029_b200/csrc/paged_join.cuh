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

// Rows rb .. of one item by one warp: RB rows x PB parts at a time in flight, D / 4 lanes a row.
template <int D, int RB, int PB>
__device__ __forceinline__ void join_rows(const AttnCall& c, const JoinCall& j, const JoinCut& x, int rb) {
  constexpr int LANES = D / 4, STEP = 32 / LANES;          // a warp has STEP rows at a time, RB deep
  const int lane = threadIdx.x & 31, col = (lane % LANES) * 4;
  {
    const int row0 = rb + lane / LANES;                    // this lane's rows: row0 + STEP r
    float M[RB], L[RB];
    float4 acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) { M[r] = -INFINITY; L[r] = 0.f; acc[r] = make_float4(0.f, 0.f, 0.f, 0.f); }
    for (int i0 = 0; i0 < x.n; i0 += PB) {
      float2 ml[RB][PB];
      float4 v[RB][PB];
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int i = 0; i < PB; ++i) {
          ml[r][i] = make_float2(-INFINITY, 0.f);
          v[r][i] = make_float4(0.f, 0.f, 0.f, 0.f);
          const int k = i0 + i, row = row0 + STEP * r;
          if (k < x.n && row < x.rows) {
            const long long at = (long long)(k == 0 ? x.slot0 : 2 * (x.first + k)) * j.rows_per_slot + row;
            ml[r][i] = __ldcg(reinterpret_cast<const float2*>(j.part_ml + at * 2));
            v[r][i] = __ldcg(reinterpret_cast<const float4*>(j.part_o + at * D + col));
          }
        }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float mn = M[r];
#pragma unroll
        for (int i = 0; i < PB; ++i) mn = fmaxf(mn, ml[r][i].x);
        const float b = mn == -INFINITY ? 0.f : mn, f = fast_exp2(M[r] - b);
        M[r] = mn;
        L[r] *= f; acc[r].x *= f; acc[r].y *= f; acc[r].z *= f; acc[r].w *= f;
#pragma unroll
        for (int i = 0; i < PB; ++i) {
          const float g = fast_exp2(ml[r][i].x - b);
          L[r] += ml[r][i].y * g;
          acc[r].x += v[r][i].x * g; acc[r].y += v[r][i].y * g; acc[r].z += v[r][i].z * g; acc[r].w += v[r][i].w * g;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int row = row0 + STEP * r;
      if (row >= x.rows) continue;
      const int gr = x.r0 + row, tok = fast_div(gr, c.G, j.div_group), head = x.h * c.G + gr - tok * c.G;
      const float inv = L[r] == 0.f ? 0.f : 1.f / L[r];
      *reinterpret_cast<uint2*>(c.out + (long long)(x.t0 + tok) * c.o_ts + (long long)head * c.o_hs + col) =
          make_uint2(ptx::pack_bf16x2(acc[r].x * inv, acc[r].y * inv), ptx::pack_bf16x2(acc[r].z * inv, acc[r].w * inv));
      if (c.lse && col == 0)
        c.lse[(long long)(x.t0 + tok) * c.H + head] = L[r] == 0.f ? -INFINITY : (M[r] + log2f(L[r])) * 0.69314718055994530942f;
    }
  }
}

// All cut items, spread over the grid by share border; pieces of two rows (one where there are many parts) of the CTA's items go
// round its warps, so that a CTA's joins run side by side.  Called by all threads of the CTA.
constexpr int kJoinList = (kPagedMaxShares + 63) / 64;
struct JoinShared { int n; JoinCut cut[kJoinList]; };
template <int D, int THREADS>
__device__ __forceinline__ void join_all(const AttnCall& c, const JoinCall& j, JoinShared* sh) {
  constexpr int STEP = 32 / (D / 4);
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) sh->n = 0;
  __syncthreads();
  for (int i = tid; i < kJoinList; i += THREADS) {
    const int g = blockIdx.x + i * gridDim.x;
    if (g < j.borders && __ldcg(j.flags + g)) sh->cut[atomicAdd(&sh->n, 1)] = j.cuts[g];
  }
  __syncthreads();
  int next = warp;                                         // pieces until this warp's next one
  for (int i = 0; i < sh->n; ++i) {
    const JoinCut& x = sh->cut[i];
    const int step = x.n <= 4 ? 2 * STEP : STEP;
    for (int rb = 0; rb < x.rows; rb += step) {
      if (next-- > 0) continue;
      next = THREADS / 32 - 1;
      if (x.n <= 4) join_rows<D, 2, 4>(c, j, x, rb);
      else join_rows<D, 1, 8>(c, j, x, rb);
    }
  }
}

}  // namespace qb
