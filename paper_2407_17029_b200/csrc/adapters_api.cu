// extern "C" entry points of the bank of adapters (include/qblora.h, last part): host-side argument checks and dispatch.
// No device memory is allocated here.
#include <algorithm>

#include "adapters.cuh"

namespace qb {
namespace {

bool bank_ok(const qblora_adapter_bank* b, bool need_ptrs, BankView* v) {
  if (!b || b->d_in < 1 || b->d_out < 1 || b->lambda_in < 1 || b->lambda_out < 1 || b->n_adapters < 1 || b->rank < 1) return false;
  if (b->d_in % b->lambda_in || b->d_out % b->lambda_out) return false;
  if (need_ptrs) {
    if (!b->A || !b->B || !b->scaling) return false;
    if (reinterpret_cast<uintptr_t>(b->A) % 2 || reinterpret_cast<uintptr_t>(b->B) % 2) return false;
    if (reinterpret_cast<uintptr_t>(b->scaling) % 4 || reinterpret_cast<uintptr_t>(b->ranks) % 4) return false;
  }
  *v = {b->d_in, b->d_out, b->lambda_in, b->lambda_out, b->d_in / b->lambda_in, b->d_out / b->lambda_out, b->n_adapters, b->rank,
        static_cast<const __nv_bfloat16*>(b->A), static_cast<const __nv_bfloat16*>(b->B), b->scaling, b->ranks};
  return true;
}

bool int_ptr_ok(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 4 == 0; }

bool rows_ok(const void* data, int64_t stride, int width, int dtype, RowsView* v) {
  if (!data || (dtype != QBLORA_F32 && dtype != QBLORA_BF16) || stride < width) return false;
  if (reinterpret_cast<uintptr_t>(data) % (dtype == QBLORA_F32 ? 4 : 2)) return false;
  *v = {const_cast<void*>(data), stride, dtype};
  return true;
}

// Calls of no more rows go to adapters_rows.cu, by the type of Y; larger ones, whose adapters have many rows then, or are many, to
// tc_adapters.cu.  An item of eight rows brings its adapter's weights for itself, from L2 where other items have them too, and yet few adapters
// are not the other path's earlier than many.  (Both in us, graph replays, one adapter / 16 / 64 of as many rows in all.  bf16, 512 rows:
// 4096 -> 11008, lambda 4, rank 256 28.8 and 27.8 / 29.6 and 32.1 / 37.2 and 53.9; 4096 -> 4096, rank 64 13.0 and 21.7 / 13.1 and 22.4 / 13.1
// and 29.0; 11008 -> 11008, lambda 1, rank 256 80 and 87 / 82 and 108 / 125 and 182.  16 adapters of 64 rows: 43 and 35, rank 64 20 and 25.
// fp32, 256 rows: 28.8 and 29.3 / 30.8 and 34.0 / 40.9 and 58.9; 12.5 and 23.4 / 13.1 and 23.9 / 13.3 and 31.0; 77 and 94 / 79 and 112 / 143
// and 194.  512 rows: 48 and 34 / 49 and 36 / 55 and 60; 18 and 24 / 20 and 24 / 21 and 31; 141 and 105 / 142 and 115 / 165 and 195.)
int few_rows(int y_dtype) { return y_dtype == QBLORA_F32 ? 256 : 512; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

int call_ok(const qblora_adapter_bank* bank, const int32_t* rows, const int32_t* start, int64_t tokens, AdaptersCall* c) {
  if (!bank_ok(bank, true, &c->k) || !int_ptr_ok(rows) || !int_ptr_ok(start) || tokens < 1) return QBLORA_ERR_INVALID_ARG;
  if (tokens >= (int64_t)1 << 31 || bank->n_adapters > kMaxAdapters) return QBLORA_ERR_UNSUPPORTED;
  c->rows = rows; c->start = start; c->T = (int)tokens;
  return QBLORA_OK;
}

}  // namespace
}  // namespace qb

using namespace qb;

extern "C" {

int qblora_adapter_plan(const int32_t* cu, const int32_t* ids, int32_t n_requests, int32_t n_adapters, int64_t tokens,
                        int32_t* rows, int32_t* start, void* stream) {
  if (!int_ptr_ok(cu) || !int_ptr_ok(ids) || !int_ptr_ok(rows) || !int_ptr_ok(start)) return QBLORA_ERR_INVALID_ARG;
  if (n_requests < 1 || n_adapters < 1 || tokens < 1) return QBLORA_ERR_INVALID_ARG;
  if (n_requests > kPlanMaxAdapterRequests || n_adapters > kMaxAdapters || tokens >= (int64_t)1 << 31) return QBLORA_ERR_UNSUPPORTED;
  // every CTA reads the requests for itself, whenever it runs
  const struct { const void* p; size_t n; } a[4] = {{rows, (size_t)tokens * 4}, {start, ((size_t)n_adapters + 1) * 4},
                                                    {cu, ((size_t)n_requests + 1) * 4}, {ids, (size_t)n_requests * 4}};
  for (int i = 0; i < 2; ++i)
    for (int j = i + 1; j < 4; ++j)
      if (overlap(a[i].p, a[i].n, a[j].p, a[j].n)) return QBLORA_ERR_INVALID_ARG;
  return launch_adapter_plan(AdapterPlanCall{cu, ids, n_requests, n_adapters, (int)tokens, rows, start}, static_cast<cudaStream_t>(stream));
}

size_t qblora_adapters_workspace_bytes(const qblora_adapter_bank* bank, int64_t tokens, int backward) {
  BankView k;
  if (!bank_ok(bank, false, &k) || tokens < 1 || tokens >= (int64_t)1 << 31) return 0;
  // alignment, which the sizes do not tell, may send a call to the general path
  const size_t general = simt_adapters_ws_bytes(k, tokens, backward != 0);
  return tc_adapters_sizes_ok(k, tokens) ? std::max(general, tc_adapters_ws_bytes(k, tokens, backward != 0)) : general;
}

int qblora_adapters_fwd(const qblora_adapter_bank* bank, const int32_t* rows, const int32_t* start, const void* X,
                        int64_t x_stride, int64_t tokens, void* Y, int64_t y_stride, int y_dtype, void* ws, size_t ws_bytes,
                        void* stream) {
  AdaptersCall c{};
  const int rc = call_ok(bank, rows, start, tokens, &c);
  if (rc) return rc;
  if (!rows_ok(X, x_stride, bank->d_in, QBLORA_BF16, &c.X) || !rows_ok(Y, y_stride, bank->d_out, y_dtype, &c.Y) || X == Y) return QBLORA_ERR_INVALID_ARG;
  if (!ws || !aligned16(ws) || ws_bytes < qblora_adapters_workspace_bytes(bank, tokens, 0)) return QBLORA_ERR_WORKSPACE;
  if (!force_general() && tc_adapters_supported(c)) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens <= few_rows(y_dtype) && rows_adapters_supported(c)) return rows_adapters_fwd(c, static_cast<int*>(ws), st);
    return tc_adapters_fwd(c, static_cast<char*>(ws), st);
  }
  return simt_adapters_fwd(c, static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
}

int qblora_adapters_bwd(const qblora_adapter_bank* bank, const int32_t* rows, const int32_t* start, const void* X,
                        int64_t x_stride, const void* dY, int64_t dy_stride, int64_t tokens, void* dX, int64_t dx_stride,
                        int dx_dtype, float* dA, float* dB, void* ws, size_t ws_bytes, void* stream) {
  AdaptersCall c{};
  const int rc = call_ok(bank, rows, start, tokens, &c);
  if (rc) return rc;
  if (!rows_ok(dY, dy_stride, bank->d_out, QBLORA_BF16, &c.Y)) return QBLORA_ERR_INVALID_ARG;
  if ((dA || dB) && !rows_ok(X, x_stride, bank->d_in, QBLORA_BF16, &c.X)) return QBLORA_ERR_INVALID_ARG;
  if (dX && (!rows_ok(dX, dx_stride, bank->d_in, dx_dtype, &c.dX) || dX == X || dX == dY)) return QBLORA_ERR_INVALID_ARG;
  if ((dA && !int_ptr_ok(dA)) || (dB && !int_ptr_ok(dB)) || (dA && dA == dB)) return QBLORA_ERR_INVALID_ARG;
  if (!ws || !aligned16(ws) || ws_bytes < qblora_adapters_workspace_bytes(bank, tokens, 1)) return QBLORA_ERR_WORKSPACE;
  const size_t slots = (size_t)c.k.n * c.k.r * 4;
  if (dA && dB && overlap(dA, slots * c.k.P, dB, slots * c.k.Q)) return QBLORA_ERR_INVALID_ARG;
  if (!dX && !dA && !dB) return QBLORA_OK;
  c.dA = dA; c.dB = dB;
  if (!force_general() && tc_adapters_supported(c)) return tc_adapters_bwd(c, static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
  return simt_adapters_bwd(c, static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
}

}  // extern "C"
