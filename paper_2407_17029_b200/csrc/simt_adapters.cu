// Many adapters over one weight, general path: any sizes, strides and alignment, CUDA cores, fp32.  What the fast kernels
// are checked against, and what takes the sizes that they do not.
#include "adapters.cuh"

namespace qb {
namespace {

__device__ __forceinline__ float row_value(const RowsView& v, int64_t row, int col) {
  const int64_t i = row * v.stride + col;
  return v.dtype == QBLORA_F32 ? static_cast<const float*>(v.data)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(v.data)[i]);
}
__device__ __forceinline__ void row_add(const RowsView& v, int64_t row, int col, float x) {
  const int64_t i = row * v.stride + col;
  if (v.dtype == QBLORA_F32) static_cast<float*>(v.data)[i] += x;
  else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(v.data) + i;
    *p = __float2bfloat16_rn(__bfloat162float(*p) + x);
  }
}

struct Entry { int a, row; };            // of place j of the plan; a < 0: none
__device__ __forceinline__ Entry plan_entry(const AdaptersCall& c, int j) {
  Entry e{-1, -1};
  if (j < plan_start(c, 0) || j >= plan_start(c, c.k.n)) return e;
  int lo = 0, hi = c.k.n;                // start[lo] <= j < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (plan_start(c, mid) <= j) lo = mid; else hi = mid;
  }
  const int row = __ldg(c.rows + j);
  if (row >= 0 && row < c.T) { e.a = lo; e.row = row; }
  return e;
}

// small[j][i] = factor * sum over the lam neighbours of X[row_j][lam i ..]
__global__ void pool_kernel(const __grid_constant__ AdaptersCall c, RowsView x, int lam, int n_small, int mean, int scaled, float* out) {
  const int j = blockIdx.x;
  const Entry e = plan_entry(c, j);
  for (int i = threadIdx.x; i < n_small; i += blockDim.x) {
    float acc = 0.f;
    if (e.a >= 0) {
      for (int l = 0; l < lam; ++l) acc += row_value(x, e.row, i * lam + l);
      if (mean) acc /= (float)lam;
      if (scaled) acc *= __ldg(c.k.s + e.a);
    }
    out[(int64_t)j * n_small + i] = acc;
  }
}
// out[j][i] = sum_k in[j][k] W(k, i), W = A, B or a transpose: element (k, i) at k * sk + i * si of the adapter's slot.  Entries from the
// adapter's rank on are left out, on whichever side the rank is.
__global__ void product_kernel(const __grid_constant__ AdaptersCall c, const float* in, int K, const __nv_bfloat16* W, int64_t slot, int64_t sk,
                               int64_t si, int N, int rank_is_k, float* out) {
  const int j = blockIdx.x;
  const Entry e = plan_entry(c, j);
  const int r = e.a >= 0 ? bank_rank(c.k, e.a) : 0, kk = rank_is_k ? min(K, r) : K;
  for (int i = threadIdx.x + blockIdx.y * blockDim.x; i < N; i += blockDim.x * gridDim.y) {
    float acc = 0.f;
    if (e.a >= 0 && (rank_is_k || i < r)) {
      const __nv_bfloat16* w = W + (int64_t)e.a * slot + i * si;
      for (int k = 0; k < kk; ++k) acc = fmaf(in[(int64_t)j * K + k], __bfloat162float(w[k * sk]), acc);
    }
    out[(int64_t)j * N + i] = acc;
  }
}
// Y[row][o] += factor * sum_c u[j][c] W(c, o / lam)
__global__ void expand_kernel(const __grid_constant__ AdaptersCall c, RowsView y, const float* u, const __nv_bfloat16* W, int64_t slot, int64_t sk,
                              int64_t si, int N, int lam, int forward) {
  const int j = blockIdx.x;
  const Entry e = plan_entry(c, j);
  if (e.a < 0) return;
  const int r = bank_rank(c.k, e.a);
  for (int i = threadIdx.x + blockIdx.y * blockDim.x; i < N; i += blockDim.x * gridDim.y) {
    const __nv_bfloat16* w = W + (int64_t)e.a * slot + i * si;
    float acc = 0.f;
    for (int k = 0; k < r; ++k) acc = fmaf(u[(int64_t)j * c.k.r + k], __bfloat162float(w[k * sk]), acc);
    acc = forward ? acc * __ldg(c.k.s + e.a) : acc / (float)lam;
    for (int l = 0; l < lam; ++l) row_add(y, e.row, i * lam + l, acc);
  }
}
// out[a][i][k] = sum over the adapter's places j of left[j][i] right[j][k]; zero where the side of the rank is past the adapter's
__global__ void gradient_kernel(const __grid_constant__ AdaptersCall c, const float* left, int M, const float* right, int N, int rank_is_row,
                                float* out) {
  const int a = blockIdx.z, lo = plan_start(c, a), hi = plan_start(c, a + 1), r = bank_rank(c.k, a);
  for (int i = blockIdx.y; i < M; i += gridDim.y)
    for (int k = threadIdx.x + blockIdx.x * blockDim.x; k < N; k += blockDim.x * gridDim.x) {
      float acc = 0.f;
      if ((rank_is_row ? i : k) < r)
        for (int j = lo; j < hi; ++j) acc = fmaf(left[(int64_t)j * M + i], right[(int64_t)j * N + k], acc);
      out[((int64_t)a * M + i) * N + k] = acc;
    }
}

unsigned grid_rows(int n) { return (unsigned)(n > 1024 ? 1024 : n); }     // (the kernel goes on from there; a grid's y ends at 65535)
unsigned parts(int n, int per) { const int x = (n + per - 1) / per; return (unsigned)(x > 64 ? 64 : x); }

int launched() {
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

struct SimtScratch { float *x, *u, *dv, *du; };
SimtScratch scratch(const BankView& k, int64_t T, char* ws) {
  SimtScratch s;
  s.x = reinterpret_cast<float*>(ws + kStatusBytes);
  s.u = s.x + T * k.P;
  s.dv = s.u + T * k.r;
  s.du = s.dv + T * k.Q;
  return s;
}

}  // namespace

size_t simt_adapters_ws_bytes(const BankView& k, int64_t T, bool backward) {
  const size_t fwd = (size_t)T * (k.P + k.r), bwd = (size_t)T * (k.Q + k.r);
  return align_up(kStatusBytes + (fwd + (backward ? bwd : 0)) * 4, 256);
}

#define QB_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

int simt_adapters_fwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  QB_CUDA(cudaMemsetAsync(ws, 0, 16, st));       // status word
  const BankView& k = c.k;
  const SimtScratch s = scratch(k, c.T, ws);
  const unsigned T = (unsigned)c.T;
  pool_kernel<<<T, 256, 0, st>>>(c, c.X, k.l1, k.P, 1, 0, s.x);
  QB_TRY(launched());
  product_kernel<<<dim3(T, parts(k.r, 256)), 256, 0, st>>>(c, s.x, k.P, k.A, (int64_t)k.P * k.r, k.r, 1, k.r, 0, s.u);
  QB_TRY(launched());
  expand_kernel<<<dim3(T, parts(k.Q, 256)), 256, 0, st>>>(c, c.Y, s.u, k.B, (int64_t)k.r * k.Q, k.Q, 1, k.Q, k.l2, 1);
  return launched();
}

int simt_adapters_bwd(const AdaptersCall& c, char* ws, cudaStream_t st) {
  QB_CUDA(cudaMemsetAsync(ws, 0, 16, st));
  const BankView& k = c.k;
  const SimtScratch s = scratch(k, c.T, ws);
  const unsigned T = (unsigned)c.T;
  pool_kernel<<<T, 256, 0, st>>>(c, c.Y, k.l2, k.Q, 0, 1, s.dv);
  QB_TRY(launched());
  if (c.dX.data || c.dA) {
    product_kernel<<<dim3(T, parts(k.r, 256)), 256, 0, st>>>(c, s.dv, k.Q, k.B, (int64_t)k.r * k.Q, 1, k.Q, k.r, 0, s.du);
    QB_TRY(launched());
  }
  if (c.dX.data) {
    expand_kernel<<<dim3(T, parts(k.P, 256)), 256, 0, st>>>(c, c.dX, s.du, k.A, (int64_t)k.P * k.r, 1, k.r, k.P, k.l1, 0);
    QB_TRY(launched());
  }
  if (c.dA || c.dB) {
    pool_kernel<<<T, 256, 0, st>>>(c, c.X, k.l1, k.P, 1, 0, s.x);
    QB_TRY(launched());
  }
  if (c.dA) {
    gradient_kernel<<<dim3(parts(k.r, 256), grid_rows(k.P), (unsigned)k.n), 256, 0, st>>>(c, s.x, k.P, s.du, k.r, 0, c.dA);
    QB_TRY(launched());
  }
  if (c.dB) {
    product_kernel<<<dim3(T, parts(k.r, 256)), 256, 0, st>>>(c, s.x, k.P, k.A, (int64_t)k.P * k.r, k.r, 1, k.r, 0, s.u);
    QB_TRY(launched());
    gradient_kernel<<<dim3(parts(k.Q, 256), grid_rows(k.r), (unsigned)k.n), 256, 0, st>>>(c, s.u, k.r, s.dv, k.Q, 1, c.dB);
    QB_TRY(launched());
  }
  return QBLORA_OK;
}

}  // namespace qb
