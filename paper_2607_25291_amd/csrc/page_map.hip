// Block tables and slot maps from request lengths for gfx950.
//
// Every workgroup scans the requests' lengths for itself (at most 8192 of them: the lengths and two prefix
// arrays in LDS) and then writes its share of the new table entries and of the token rows' slots,
// finding the request of an entry or a row by binary search. So one launch does it, with no pass between
// the scan and its use.
//
// Bound: latency. 64 requests of one token 4.3 us, 256 prompts with 90K rows 6.5 to 7.3, 4096 / 8192 requests 14 / 22 (18 / 40
// with the lengths read from memory in every pass).
#include <mutex>

#include "cosa_device.h"
#include "decode_internal.h"
#include "select_wave.h"

namespace cosa {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kSat = 0x7fffffffu;

// Sums of non-negative 31-bit values, held at 2^31 - 1: associative, so a scan may group them freely.
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) {
  const uint32_t s = a + b;
  return s < kSat ? s : kSat;
}

// Exclusive saturating scan of one value per thread over the workgroup, and the total.
__device__ uint32_t block_scan(uint32_t x, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)incl, d, 64);
    if (lane >= d) incl = sat_add(incl, y);
  }
  if (lane == 63) waves[w] = incl;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < w) before = sat_add(before, waves[i]);
    total = sat_add(total, waves[i]);
  }
  __syncthreads();
  uint32_t excl = (uint32_t)__shfl_up((int)incl, 1, 64);
  if (lane == 0) excl = 0;
  return sat_add(before, excl);
}

// Largest r in [0, n) with start[r] <= x (start[0] = 0, non-decreasing).
__device__ __forceinline__ int find(const uint32_t* start, int n, uint32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kThreads) void page_map_kernel(PageMapArgs A) {
  extern __shared__ uint32_t lds[];
  uint32_t* cached = lds;                  // tokens that request r holds
  uint32_t* add = lds + A.batch;           // and adds
  uint32_t* row0 = lds + 2 * A.batch;      // its first packed row
  uint32_t* page0 = lds + 3 * A.batch;     // free pages needed before it
  __shared__ uint32_t waves[kThreads / 64];
  const uint32_t cap = (uint32_t)A.max_pages << A.log2_page;
  const uint32_t last = (1u << A.log2_page) - 1u;
  const int n_free = A.batch ? min(max(*A.n_free, 0), A.free_capacity) : 0;  // an empty batch may come without it
  for (int r = threadIdx.x; r < A.batch; r += kThreads) {
    cached[r] = min((uint32_t)max(A.cached[r], 0), cap);
    add[r] = (uint32_t)max(A.add[r], 0);
  }
  __syncthreads();
  // Pages request r takes when its rows start at packed row `first`; fits: row width and slot range.
  const auto need = [&](int r, uint32_t first, bool& fits) -> uint32_t {
    const uint32_t c = cached[r], n = add[r];
    fits = n <= cap - c && first + n <= (uint32_t)A.max_new;  // below 2^32; a sum held at 2^31 - 1 leaves no row
    return fits ? ((c + n + last) >> A.log2_page) - ((c + last) >> A.log2_page) : 0u;
  };

  const int per = ((A.batch + kThreads - 1) / kThreads) | 1;  // odd: the threads' requests lie in different banks
  const int r0 = min((int)threadIdx.x * per, A.batch), r1 = min(r0 + per, A.batch);
  uint32_t sum = 0, rows = 0, pages = 0;
  for (int r = r0; r < r1; ++r) sum = sat_add(sum, add[r]);
  uint32_t at = block_scan(sum, waves, rows);
  sum = 0;
  for (int r = r0; r < r1; ++r) {
    bool fits;
    row0[r] = at;
    sum = sat_add(sum, need(r, at, fits));
    at = sat_add(at, add[r]);
  }
  at = block_scan(sum, waves, pages);
  uint32_t taken = 0;  // of this thread's last request that gets its pages
  for (int r = r0; r < r1; ++r) {
    bool fits;
    const uint32_t n = need(r, row0[r], fits);
    page0[r] = at;
    at = sat_add(at, n);
    const bool in = fits && (n == 0 || at <= (uint32_t)n_free);
    if (in && n != 0) taken = at;
    if (blockIdx.x == 0) {
      A.seq_lens[r] = (int)(cached[r] + (in ? add[r] : 0u));
      A.cu_new[r] = (int)row0[r];
    }
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0 && A.cu_new) A.cu_new[A.batch] = (int)rows;
    // pages taken: the largest need that was met (needs grow along the requests)
#pragma unroll
    for (int d = 32; d; d >>= 1) taken = max(taken, (uint32_t)__shfl_xor((int)taken, d, 64));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = taken;
    __syncthreads();
    if (threadIdx.x == 0 && A.n_taken) *A.n_taken = (int)max(max(waves[0], waves[1]), max(waves[2], waves[3]));
  }

  const uint32_t step = gridDim.x * kThreads, self = blockIdx.x * kThreads + threadIdx.x;
  // New table entries. A request's pages lie below n_free as a whole or it takes none.
  const uint32_t n_entries = min(pages, (uint32_t)n_free);
  for (uint32_t p = self; p < n_entries; p += step) {
    const int r = find(page0, A.batch, p);
    bool fits;
    const uint32_t n = need(r, row0[r], fits);
    if (page0[r] + n <= (uint32_t)n_free)
      A.table[(size_t)r * A.max_pages + ((cached[r] + last) >> A.log2_page) + (p - page0[r])] = A.free_pages[p];
  }
  for (uint32_t t = self; t < (uint32_t)A.max_new; t += step) {
    int64_t slot = -1;
    if (t < rows) {
      const int r = find(row0, A.batch, t);
      const uint32_t c = cached[r];
      bool fits;
      const uint32_t n = need(r, row0[r], fits);
      if (fits && (n == 0 || sat_add(page0[r], n) <= (uint32_t)n_free)) {
        const uint32_t pos = c + (t - row0[r]), j = pos >> A.log2_page;
        const uint32_t first = (c + last) >> A.log2_page;  // the request's first new page
        const int32_t page = j < first ? A.table[(size_t)r * A.max_pages + j] : A.free_pages[page0[r] + j - first];
        if (page >= 0) slot = ((int64_t)page << A.log2_page) + (pos & last);
      }
    }
    A.slots[t] = slot;
  }
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream) {
  static std::mutex mu;
  static bool granted[64] = {};
  const size_t lds = (size_t)a.batch * 16;
  if (lds > 48 * 1024) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    if (dev < 0 || dev >= 64 || !granted[dev]) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(&page_map_kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, kMaxRequests * 16);
      if (e != hipSuccess) return e;
      if (dev >= 0 && dev < 64) granted[dev] = true;
    }
  }
  // A workgroup for every 512 rows, so that the scan it starts with is a small part of a large map.
  const int grid = std::min(std::max(a.max_new / 512 + (a.max_new % 512 != 0), 1), 512);
  hipLaunchKernelGGL(page_map_kernel, dim3(grid), dim3(kThreads), lds, stream, a);
  return hipGetLastError();
}

}  // namespace cosa
