// Shared declarations of the calls for many adapters over one weight: rows sorted by adapter, forward, backward
// (include/qblora.h, last part).
#pragma once
#include "common.cuh"

namespace qb {

constexpr int kPlanMaxAdapterRequests = 8192, kMaxAdapters = 4096;

struct AdapterPlanCall {
  const int *cu, *ids;
  int R, n, T;
  int *rows, *start;
};
int launch_adapter_plan(const AdapterPlanCall& c, cudaStream_t st);

struct BankView {
  int d_in, d_out, l1, l2, P, Q, n, r;
  const __nv_bfloat16 *A, *B;
  const float* s;
  const int* ranks;
};

// A matrix of rows in the caller's memory; bf16 or fp32.
struct RowsView { void* data; int64_t stride; int dtype; };

struct AdaptersCall {
  BankView k;
  const int *rows, *start;
  int T;
  RowsView X, Y;            // forward: Y in and out; backward: Y is dY
  RowsView dX;              // data == nullptr: not wanted, as dA and dB
  float *dA, *dB;
};

// Rank of adapter a that the kernels work with: a multiple of 16, or the slots' rank.  (Unsigned: the largest int32 rounded up passes 2^31.)
__device__ __forceinline__ int bank_rank(const BankView& k, int a) {
  return k.ranks ? (int)min(((uint32_t)max(__ldg(k.ranks + a), 0) + 15u) & ~15u, (uint32_t)k.r) : k.r;
}
// Entry i of the plan's offsets, forced into 0 .. T.
__device__ __forceinline__ int plan_start(const AdaptersCall& c, int i) { return min(max(__ldg(c.start + i), 0), c.T); }

// General path: any sizes, strides and alignment (simt_adapters.cu).
size_t simt_adapters_ws_bytes(const BankView& k, int64_t T, bool backward);
int simt_adapters_fwd(const AdaptersCall& c, char* ws, cudaStream_t st);
int simt_adapters_bwd(const AdaptersCall& c, char* ws, cudaStream_t st);

// Tensor cores (tc_adapters.cu): rank and Q multiples of 8, rows of multiples of 8 elements, 16-byte aligned.
bool tc_adapters_sizes_ok(const BankView& k, int64_t T);
bool tc_adapters_supported(const AdaptersCall& c);
size_t tc_adapters_ws_bytes(const BankView& k, int64_t T, bool backward);
int tc_adapters_fwd(const AdaptersCall& c, char* ws, cudaStream_t st);
int tc_adapters_bwd(const AdaptersCall& c, char* ws, cudaStream_t st);

// Few rows, forward (adapters_rows.cu): one launch, without workspace but the status word.
bool rows_adapters_supported(const AdaptersCall& c);
int rows_adapters_fwd(const AdaptersCall& c, int* status, cudaStream_t st);

}  // namespace qb
