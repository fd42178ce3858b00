// Pages of a paged cache copied to other pages, for gfx950.
//
// A page of one tensor is a stretch of n_kv_heads * page_size rows of 256 bytes (its bounds: 2 n_kv_heads rows); the pairs'
// stretches of 64 rows are dealt to a fixed grid, since only the device knows how many pairs there are. A workgroup has
// all of its 16 KiB in flight before it stores the first. Of a partly filled page only the first rows of every head are read and
// written.
//
// Bound: HBM. 2048 pages of 128 tokens and 8 heads 433 us, 5.0 TB/s read and written, as a copy of 2 GiB in one piece; the partly
// filled pages of 64 rows 5.6 us (median of 24 calls; the shortest 4.8). Loads and stores pass the caches by: nothing of a page is used twice.
#include "cosa_device.h"
#include "serving_internal.h"

namespace cosa {
namespace {

constexpr int kThreads = 256, kRows = 64;  // rows of a stretch, 16 lanes each
constexpr int kLoads = kRows * 16 / kThreads;

__global__ __launch_bounds__(kThreads) void page_copy_kernel(PageCopyArgs A, int per_tensor, int per_pair) {
  const int n_pairs = min(max(*A.n_pairs, 0), A.max_pairs);
  const unsigned items = (unsigned)n_pairs * (unsigned)per_pair;
  const int page = 1 << A.log2_page;
  for (unsigned x = blockIdx.x; x < items; x += gridDim.x) {
    const int pair = (int)(x / (unsigned)per_pair);
    int at = (int)(x - (unsigned)pair * (unsigned)per_pair);
    const int64_t src = A.src[pair], dst = A.dst[pair];
    if (src < 0 || dst < 0 || src >= A.n_pages || dst >= A.n_pages) continue;
    uint16_t* base = A.k_cache;
    int rows = A.Hkv << A.log2_page, keep = page, in_head = page - 1;
    if (at >= 2 * per_tensor) {
      at -= 2 * per_tensor;
      base = A.bounds;
      rows = 2 * A.Hkv;
      in_head = 0;
    } else {
      if (A.rows) keep = min(max(A.rows[pair], 0), page);
      if (at >= per_tensor) {
        at -= per_tensor;
        base = A.v_cache;
      }
    }
    const int row0 = at * kRows;
    if ((row0 & in_head) >= keep && (in_head >= kRows - 1)) continue;  // a stretch behind the rows of one head
    const uint16_t* from = base + (size_t)src * rows * kHeadDim;
    uint16_t* to = base + (size_t)dst * rows * kHeadDim;
    u32x4_t v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + (i * kThreads + (int)threadIdx.x) / 16;
      if (row < rows && (row & in_head) < keep)
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(from + (size_t)row * kHeadDim) + (threadIdx.x & 15));
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + (i * kThreads + (int)threadIdx.x) / 16;
      if (row < rows && (row & in_head) < keep)
        __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4_t*>(to + (size_t)row * kHeadDim) + (threadIdx.x & 15));
    }
  }
}

long long per_tensor(int Hkv, int log2_page) { return (((long long)Hkv << log2_page) + kRows - 1) / kRows; }

}  // namespace

long long page_copy_items(int Hkv, int log2_page, bool bounds) {
  return 2 * per_tensor(Hkv, log2_page) + (bounds ? (2ll * Hkv + kRows - 1) / kRows : 0);
}

hipError_t launch_page_copy(const PageCopyArgs& a, hipStream_t stream) {
  const long long per_pair = page_copy_items(a.Hkv, a.log2_page, a.bounds != nullptr), items = per_pair * a.max_pairs;
  const int grid = (int)(items < 2048 ? items : 2048);
  hipLaunchKernelGGL(page_copy_kernel, dim3(grid), dim3(kThreads), 0, stream, a, (int)per_tensor(a.Hkv, a.log2_page),
                     (int)per_pair);
  return hipGetLastError();
}

}  // namespace cosa
