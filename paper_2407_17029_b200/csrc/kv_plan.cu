// Block tables and slot maps of one serving step, built on the GPU from the requests' lengths (qblora_kv_plan).
//
// Three running sums over the requests decide everything: pages given back, pages needed, rows asked for.  Admission is
// first come, first served, so it is one cut: with S_N, S_T the inclusive sums of pages needed and rows asked over the
// valid requests, request b is admitted iff S_N[b] <= pages there are and S_T[b] <= rows there are -- both sums only
// grow, so the first request that fails is followed by none that is admitted.  After the cut every output is a function
// of its own index and the sums: page a of the step belongs to the request with S_N[b-1] <= a < S_N[b] (a search), and is
// stack entry (free + given back - 1 - a); row t likewise in S_T.
//
// What bounds it: latency.  The data are a few hundred KB at most, so the kernel is one launch in which every CTA
// forms all sums for itself in shared memory (no CTA waits for another, and no second launch follows a scan); the
// outputs are then spread over the grid.  A page given back in this very call is read from the releasing request's
// table row, not from the stack, so no write of the call is read in it.
// Measured: 8 decoding requests 3.4 us in a graph, 512 requests with prompt chunks of 1777 tokens 6.4 us; called from the host
// one after the other 10.5 us each, which is what a launch and its arguments cost there.
#include <atomic>

#include "serving.cuh"

namespace qb {
namespace {

constexpr int KP_THREADS = 256;
constexpr uint32_t KP_MAX = 0x7fffffffu;

// Sum of two values in 0 .. 2^31 - 1, stopped at 2^31 - 1: associative, so a scan of absurd lengths cannot wrap.
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, KP_MAX); }

struct Kp3 { uint32_t back, need, rows; };
__device__ __forceinline__ Kp3 operator+(const Kp3& a, const Kp3& b) {
  return {sat_add(a.back, b.back), sat_add(a.need, b.need), sat_add(a.rows, b.rows)};
}
__device__ __forceinline__ Kp3 shfl_up(const Kp3& a, int d) {
  return {__shfl_up_sync(0xffffffffu, a.back, d), __shfl_up_sync(0xffffffffu, a.need, d), __shfl_up_sync(0xffffffffu, a.rows, d)};
}

struct KpReq { int ctx, held, add; uint32_t back, need; bool gone, valid; };
__device__ __forceinline__ KpReq kp_request(const PlanCall& c, int b) {
  KpReq r;
  const long long most = (long long)c.width * c.page;
  const int ctx = __ldg(c.ctx + b), add = __ldg(c.add + b);
  r.gone = c.release && __ldg(c.release + b) != 0;
  r.valid = !r.gone && ctx >= 0 && add >= 0 && (long long)ctx + add <= most;
  r.ctx = (int)min((long long)max(ctx, 0), most);
  r.held = (int)(((long long)r.ctx + c.page - 1) / c.page);
  r.back = r.gone ? (uint32_t)r.held : 0u;
  r.add = r.valid ? add : 0;
  r.need = r.valid ? (uint32_t)(((long long)ctx + add + c.page - 1) / c.page - r.held) : 0u;
  return r;
}

// first b in [0, n) with sums[b] > x (n if none)
__device__ __forceinline__ int kp_find(const uint32_t* sums, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(KP_THREADS) kv_plan_kernel(const __grid_constant__ PlanCall c) {
  extern __shared__ uint32_t kp_smem[];
  uint32_t* s_back = kp_smem;            // inclusive sums [B]
  uint32_t* s_need = s_back + c.B;
  uint32_t* s_rows = s_need + c.B;
  __shared__ Kp3 s_warp[KP_THREADS / 32];
  __shared__ int s_cut;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) s_cut = c.B;
  const int n_free = min(max(__ldg(c.count), 0), c.capacity);

  Kp3 carry{0, 0, 0};
  for (int b0 = 0; b0 < c.B; b0 += KP_THREADS) {
    const int b = b0 + tid;
    Kp3 x{0, 0, 0};
    if (b < c.B) {
      const KpReq r = kp_request(c, b);
      x = {r.back, r.need, (uint32_t)r.add};
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const Kp3 y = shfl_up(x, d);
      if (lane >= d) x = x + y;
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    Kp3 before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < KP_THREADS / 32; ++w) {
      const Kp3 y = s_warp[w];
      if (w < warp) before = before + y;
      all = all + y;
    }
    x = before + x;
    if (b < c.B) { s_back[b] = x.back; s_need[b] = x.need; s_rows[b] = x.rows; }
    carry = all;
    __syncthreads();
  }
  const uint32_t back = carry.back;
  const uint32_t avail = min(sat_add((uint32_t)n_free, back), (uint32_t)c.capacity);
  // the cut; a request that needs nothing and asks for nothing passes no limit by itself, so sums alone decide
  for (int b = tid; b < c.B; b += KP_THREADS)
    if (s_need[b] > avail || s_rows[b] > (uint32_t)c.T) { atomicMin(&s_cut, b); break; }
  __syncthreads();
  const int cut = s_cut;
  const uint32_t taken = cut > 0 ? s_need[cut - 1] : 0u, rows = cut > 0 ? s_rows[cut - 1] : 0u;

  const int gid = blockIdx.x * KP_THREADS + tid, gn = gridDim.x * KP_THREADS;
  // entry idx of the stack after the pages given back have been put on it
  auto stack_at = [&](uint32_t idx) -> int {
    if (idx < (uint32_t)n_free) return __ldcg(c.stack + idx);
    const uint32_t i = idx - (uint32_t)n_free;
    const int b = kp_find(s_back, c.B, i);
    const uint32_t first = b > 0 ? s_back[b - 1] : 0u;
    return __ldcg(c.table + (int64_t)b * c.width + (i - first));
  };
  for (int b = gid; b < c.B; b += gn) {
    const KpReq r = kp_request(c, b);
    const bool ok = r.valid && b < cut;
    if (b == 0) { c.cu[0] = 0; c.count_out[0] = (int)(avail - taken); }
    c.cu[b + 1] = (int)min(s_rows[b], rows);
    c.kv[b] = r.gone ? 0 : r.ctx + (ok ? r.add : 0);
    c.admitted[b] = ok ? 1 : 0;
  }
  for (int64_t i = gid; i < (int64_t)back; i += gn) {
    const int b = kp_find(s_back, c.B, (uint32_t)i);
    const uint32_t first = b > 0 ? s_back[b - 1] : 0u;
    if (n_free + i < c.capacity) c.stack[n_free + i] = __ldcg(c.table + (int64_t)b * c.width + (i - first));
  }
  for (int64_t a = gid; a < (int64_t)taken; a += gn) {
    const int b = kp_find(s_need, cut, (uint32_t)a);
    const uint32_t first = b > 0 ? s_need[b - 1] : 0u;
    const KpReq r = kp_request(c, b);
    c.table[(int64_t)b * c.width + r.held + (a - first)] = stack_at(avail - 1u - (uint32_t)a);
  }
  for (int64_t t = gid; t < (int64_t)c.T; t += gn) {
    int pos = 0, slot = -1;
    if (t < (int64_t)rows) {
      const int b = kp_find(s_rows, cut, (uint32_t)t);
      const uint32_t first = b > 0 ? s_rows[b - 1] : 0u;
      const KpReq r = kp_request(c, b);
      pos = r.ctx + (int)(t - first);
      const int j = pos / c.page;
      const int page = j < r.held ? __ldcg(c.table + (int64_t)b * c.width + j)
                                  : stack_at(avail - 1u - ((b > 0 ? s_need[b - 1] : 0u) + (uint32_t)(j - r.held)));
      slot = page * c.page + (pos - j * c.page);
    }
    c.pos[t] = pos;
    c.slots[t] = slot;
  }
}

}  // namespace

int launch_kv_plan(const PlanCall& c, cudaStream_t st) {
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  QB_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return QBLORA_ERR_UNSUPPORTED;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA(cudaFuncSetAttribute(kv_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPlanMaxRequests * 12));
    attr_set[dev].store(true, std::memory_order_release);
  }
  // one row of the step per thread, up to one CTA per SM
  const int64_t work = c.T > c.B ? c.T : c.B;
  int64_t grid = (work + KP_THREADS - 1) / KP_THREADS;
  if (grid > 148) grid = 148;
  kv_plan_kernel<<<(unsigned)grid, KP_THREADS, (size_t)c.B * 12, st>>>(c);
  count_launch();
  QB_CUDA(cudaGetLastError());
  return QBLORA_OK;
}

}  // namespace qb
