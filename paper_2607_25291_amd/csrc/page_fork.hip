// Block tables of rows that continue other rows, for gfx950.
//
// Every workgroup finds for itself which children take a page (the first child of each row by a minimum in LDS, their
// ranks by a scan) and then writes its share of the new table, so that one launch does it.
//
// Bound: latency. 8 samples of one row 3.4 us; 512 children of 512 rows, 3.5 MB of tables, 7.2 us (0.7 at the rate of a copy): four
// dependent loads and the scan in front of the first entry, the same in each of the 1024 workgroups. That scan is 32 children a
// thread at 8192 of them: calls of 2048 / 8192 children of as many rows 13 / 75 us.
#include "cosa_device.h"
#include "select_wave.h"
#include "serving_internal.h"

namespace cosa {
namespace {

constexpr int kThreads = 256;
constexpr int kEntries = 1024;  // table entries of a workgroup's turn
constexpr uint16_t kKeeps = 0xffff;

__global__ __launch_bounds__(kThreads) void page_fork_kernel(PageForkArgs A) {
  extern __shared__ int lds[];
  int* first = lds;                                                        // the first child of every row
  uint16_t* rank = reinterpret_cast<uint16_t*>(first + A.n_parents);       // of the page that a child takes
  __shared__ uint32_t waves[kThreads / 64];
  const int cap = A.max_pages << A.log2_page, mask = (1 << A.log2_page) - 1;
  const int n_free = min(max(*A.n_free, 0), A.free_capacity);
  const auto parent_of = [&](int c) {
    const int p = A.parent[c];
    return p >= 0 && p < A.n_parents ? p : -1;
  };
  const auto length_of = [&](int p) { return p < 0 ? 0 : min(max(A.seq_lens[p], 0), cap); };
  for (int p = threadIdx.x; p < A.n_parents; p += kThreads) first[p] = A.n_children;
  __syncthreads();
  for (int c = threadIdx.x; c < A.n_children; c += kThreads) {
    const int p = parent_of(c);
    if (p >= 0) atomicMin(&first[p], c);
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int per = (A.n_children + kThreads - 1) / kThreads;
  const int c0 = min((int)threadIdx.x * per, A.n_children), c1 = min(c0 + per, A.n_children);
  uint32_t mine = 0;
  for (int c = c0; c < c1; ++c) {
    const int p = parent_of(c);
    const bool need = (length_of(p) & mask) != 0 && (A.copy_all || first[p] != c);
    rank[c] = need ? (uint16_t)mine : kKeeps;
    mine += need;
  }
  uint32_t at = wave_incl_scan(mine, lane);
  if (lane == 63) waves[w] = at;
  __syncthreads();
  at -= mine;
  uint32_t total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < w) at += waves[i];
    total += waves[i];
  }
  for (int c = c0; c < c1; ++c)
    if (rank[c] != kKeeps) rank[c] = (uint16_t)(rank[c] + at);
  __syncthreads();

  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) *A.n_taken = min((int)total, n_free);
    for (int c = threadIdx.x; c < A.n_children; c += kThreads) {
      const int p = parent_of(c), r = rank[c];
      int length = length_of(p);
      if (r != kKeeps) {
        if (r < n_free) {
          A.src[r] = A.table[(size_t)p * A.max_pages + (length >> A.log2_page)];
          A.dst[r] = A.free_pages[r];
          A.rows[r] = length & mask;
        } else {
          length = 0;
        }
      }
      A.new_lens[c] = length;
    }
  }
  const int turns = (A.max_pages + kEntries - 1) / kEntries;
  for (int x = blockIdx.x; x < A.n_children * turns; x += gridDim.x) {
    const int c = x / turns, p = parent_of(c), r = rank[c], length = length_of(p);
    if (r != kKeeps && r >= n_free) continue;
    const int pages = (int)(((uint32_t)length + (uint32_t)mask) >> A.log2_page);
    const int j1 = min((x % turns + 1) * kEntries, pages);
    const int taken = r == kKeeps ? -1 : pages - 1;  // the entry with a page of its own
    for (int j = x % turns * kEntries + threadIdx.x; j < j1; j += kThreads)
      A.new_table[(size_t)c * A.max_pages + j] = j == taken ? A.free_pages[r] : A.table[(size_t)p * A.max_pages + j];
  }
}

}  // namespace

hipError_t launch_page_fork(const PageForkArgs& a, hipStream_t stream) {
  const size_t lds = (size_t)a.n_parents * 4 + (size_t)a.n_children * 2;  // at most 48 KiB
  const long long turns = (long long)a.n_children * ((a.max_pages + kEntries - 1) / kEntries);
  const int grid = (int)(turns < 1 ? 1 : turns < 1024 ? turns : 1024);
  hipLaunchKernelGGL(page_fork_kernel, dim3(grid), dim3(kThreads), lds, stream, a);
  return hipGetLastError();
}

}  // namespace cosa
