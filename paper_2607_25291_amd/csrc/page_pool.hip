// Pages given back to the free list, and pages moved to the lowest numbers, for gfx950.
//
// Both mark the pages that rows hold and then number the marked or unmarked ones in ascending order by a scan over the
// cache's pages: no atomics whose order could show, and no state between calls. Few pages in few rows: one workgroup, with
// the marks as bits in LDS. Otherwise kernels one after the other, with the marks as bytes in the workspace (plain
// stores: a page marked twice gets the same byte twice): clear, mark, count by blocks, write.
//
// Bound: few entries, latency (64 rows: release 5.2 us, compaction 11.5, of which the second walk over the table and its
// dependent loads are half). Many: the marks' stores, one byte each at random places (591K entries of 512 rows: 11.3 of
// release's 19 us; 559K: 11.2 of compaction's 33), then launches that wait for each other, 2 to 4 us each, and the
// compaction's lists and tables, 8.3 and 12.1 us. Large pools: all marks are cleared and read, and every block adds up the
// counts of all (64 rows of 4096 pages in a pool of 2^24 / 2^26 / 2^28 pages: release 32 / 136 / 1274 us, compaction 53 / 234 / 2330).
#include <algorithm>

#include "cosa_device.h"
#include "select_wave.h"
#include "serving_internal.h"

namespace cosa {
namespace {

constexpr int kThreads = 256;
constexpr int kBlockPages = kThreads * 16;  // pages of a workgroup: 16 marks a thread
constexpr int kEntries = 1024;              // table entries of a workgroup's turn

struct Header {  // in the workspace, written by one kernel for the next ones
  int a, b;
};

// 32 pages: which of them are in use, and how many in front of them.
struct Word {
  uint32_t bits, start;
};

// The workspace: header, counts of the blocks, marks, and a second array of them (release) or words (compact). All end
// with a whole block.
struct Pool {
  Header* header;
  int32_t* counts;
  uint8_t *marks, *marks2;
  Word* words;
  int blocks;
  size_t bytes;
  Pool(void* ws, long long n_pages) {
    blocks = (int)((n_pages + kBlockPages - 1) / kBlockPages);
    char* p = static_cast<char*>(ws);
    const size_t all = (size_t)blocks * kBlockPages, counts_at = 256, marks_at = counts_at + ((size_t)blocks * 4 + 255) / 256 * 256;
    header = reinterpret_cast<Header*>(p);
    counts = reinterpret_cast<int32_t*>(p + counts_at);
    marks = reinterpret_cast<uint8_t*>(p + marks_at);
    marks2 = marks + all;                                   // release
    words = reinterpret_cast<Word*>(p + marks_at + all);    // compact
    bytes = marks_at + 2 * all;
  }
};

__device__ __forceinline__ int held_pages(int length, int max_pages, int log2_page) {
  const uint32_t l = (uint32_t)min(max(length, 0), max_pages << log2_page);
  return (int)((l + (1u << log2_page) - 1u) >> log2_page);
}

// Sum over the workgroup of one value per thread, and the sum of the threads in front. waves: NT / 64 words of LDS.
template <int NT>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t at = wave_incl_scan(x, lane);
  __syncthreads();  // waves may still be read from a scan before
  if (lane == 63) waves[w] = at;
  __syncthreads();
  at -= x;
  total = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i < w) at += waves[i];
    total += waves[i];
  }
  return at;
}

__global__ __launch_bounds__(kThreads) void clear_kernel(u32x4_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (size_t)gridDim.x * kThreads) p[i] = u32x4_t{0, 0, 0, 0};
}

// f(entry, page) for entries from, from + step, ... of a row below `held`, with pages outside the cache left out. Four loads
// are in flight before the first is used: a store of f might change the next one's entry, for all the compiler knows.
template <class F>
__device__ __forceinline__ void for_pages(const int32_t* row, int from, int step, int held, long long n_pages, F&& f) {
  for (int j0 = from; j0 < held; j0 += 4 * step) {
    int p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = j0 + i * step < held ? row[j0 + i * step] : -1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p[i] >= 0 && p[i] < n_pages) f(j0 + i * step, p[i]);
  }
}


// ---- release

__device__ __forceinline__ void free_list(const PageReleaseArgs& A, int& taken, int& n_free) {
  n_free = min(max(*A.n_free, 0), A.free_capacity);
  taken = A.n_taken ? min(max(*A.n_taken, 0), n_free) : 0;
}

// The rows of both tables, or of the one that both are, whose entries are then read and marked once (512 rows, of which half
// end, 19 us, as two tables 22).
struct ReleaseRow {
  const int32_t* entries;
  int was, is;  // entries held before and afterwards; 0 for a row that the other table has
};
__host__ __device__ __forceinline__ bool one_table(const PageReleaseArgs& A) {
  return A.old_table == A.new_table && A.old_batch == A.new_batch;
}
__host__ __device__ __forceinline__ int release_rows(const PageReleaseArgs& A) {
  return one_table(A) ? A.old_batch : A.old_batch + A.new_batch;
}
__device__ __forceinline__ ReleaseRow release_row(const PageReleaseArgs& A, int row) {
  const bool old = row < A.old_batch;
  const int y = old ? row : row - A.old_batch;
  return {(old ? A.old_table : A.new_table) + (size_t)y * A.max_pages,
          old ? held_pages(A.old_lens[y], A.max_pages, A.log2_page) : 0,
          !old || one_table(A) ? held_pages(A.new_lens[y], A.max_pages, A.log2_page) : 0};
}

// marks: pages that are held afterwards or listed already; marks2: pages that were held, but for those.
__global__ __launch_bounds__(kThreads) void release_mark_kernel(PageReleaseArgs A, Pool W, int turns) {
  const int per_row = (A.max_pages + kEntries - 1) / kEntries;
  for (int x = blockIdx.x; x < turns; x += gridDim.x) {
    const ReleaseRow R = release_row(A, x / per_row);
    const int j0 = x % per_row * kEntries;
    for_pages(R.entries, j0 + (int)threadIdx.x, kThreads, min(j0 + kEntries, max(R.was, R.is)), A.n_pages,
              [&](int j, int p) { (j < R.is ? W.marks : W.marks2)[p] = 1; });
  }
  int taken, n_free;
  free_list(A, taken, n_free);
  for (int i = taken + blockIdx.x * kThreads + threadIdx.x; i < n_free; i += gridDim.x * kThreads) {
    const int p = A.free_pages[i];
    if (p >= 0 && p < A.n_pages) W.marks[p] = 1;
    if (i - taken < A.out_capacity) A.free_out[i - taken] = p;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *W.header = Header{n_free - taken, 0};  // n_free_out may be n_free
}

// 16 marks of a thread as bits; release: the pages that become free.
template <bool RELEASE>
__device__ __forceinline__ uint32_t marks16(const Pool& W, int block) {
  const size_t at = (size_t)block * kThreads + threadIdx.x;
  u32x4_t m = reinterpret_cast<const u32x4_t*>(W.marks)[at];
  if (RELEASE) m = reinterpret_cast<const u32x4_t*>(W.marks2)[at] & ~m;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = m[i] & 0x01010101u;  // bytes 0 or 1 to bits 0 .. 3
    bits |= ((v | v >> 7 | v >> 14 | v >> 21) & 15u) << (4 * i);
  }
  return bits;
}

template <bool RELEASE>
__global__ __launch_bounds__(kThreads) void count_kernel(Pool W) {
  __shared__ uint32_t waves[kThreads / 64];
  uint32_t total;
  block_scan<kThreads>(__popc(marks16<RELEASE>(W, blockIdx.x)), waves, total);
  if (threadIdx.x == 0) W.counts[blockIdx.x] = (int)total;
}

// Counts of the blocks in front of `block`, and of all.
__device__ __forceinline__ void blocks_before(const Pool& W, int block, uint32_t* waves, uint32_t& before, uint32_t& all) {
  uint32_t a = 0, b = 0;
  for (int i = threadIdx.x; i < W.blocks; i += kThreads) {
    const uint32_t c = (uint32_t)W.counts[i];
    b += c;
    if (i < block) a += c;
  }
  block_scan<kThreads>(a, waves, before);
  block_scan<kThreads>(b, waves, all);
}

__global__ __launch_bounds__(kThreads) void release_write_kernel(PageReleaseArgs A, Pool W) {
  __shared__ uint32_t waves[kThreads / 64];
  uint32_t before, all, mine;
  blocks_before(W, blockIdx.x, waves, before, all);
  uint32_t bits = marks16<true>(W, blockIdx.x);
  const int first = W.header->a;
  int at = first + (int)(before + block_scan<kThreads>(__popc(bits), waves, mine));
  const int page0 = blockIdx.x * kBlockPages + threadIdx.x * 16;
  for (; bits; bits &= bits - 1, ++at)
    if (at < A.out_capacity) A.free_out[at] = page0 + __builtin_ctz(bits);
  if (blockIdx.x == 0 && threadIdx.x == 0) *A.n_free_out = min(first + (int)all, A.out_capacity);
}

// ---- compact

struct Plan {
  int used, low, moves;  // pages in use, those of them below `used`, moves
  __device__ int holes() const { return used - low; }  // unused pages below `used`, as many as used ones above
};

// What page p is for the plan, c used pages in front of it.
__device__ __forceinline__ void plan_page(const PageCompactArgs& A, const Plan& P, int p, bool used, int c) {
  const int left = P.holes() - P.moves;  // unused pages below and used pages above that stay
  if (p < P.used) {
    if (used) return;
    const int r = p - c;
    if (r < P.moves) A.dst[r] = p;
    else if (r - P.moves < A.free_capacity) A.free_pages[r - P.moves] = p;
    return;
  }
  const int r = P.used - 1 - c;  // used pages above p
  if (used && r >= P.moves) return;
  if (used) A.src[r] = p;
  const int at = left + (p - P.used) - min(c - P.low, left);
  if (at < A.free_capacity) A.free_pages[at] = p;
}

__global__ __launch_bounds__(kThreads) void compact_mark_kernel(PageCompactArgs A, Pool W, int turns) {
  const int per_row = (A.max_pages + kEntries - 1) / kEntries;
  for (int x = blockIdx.x; x < turns; x += gridDim.x) {
    const int row = x / per_row, j0 = x % per_row * kEntries;
    const int j1 = min(j0 + kEntries, held_pages(A.seq_lens[row], A.max_pages, A.log2_page));
    for_pages(A.table + (size_t)row * A.max_pages, j0 + (int)threadIdx.x, kThreads, j1, A.n_pages,
              [&](int, int p) { W.marks[p] = 1; });
  }
}

__global__ __launch_bounds__(kThreads) void compact_plan_kernel(PageCompactArgs A, Pool W) {
  __shared__ uint32_t waves[kThreads / 64];
  uint32_t before, all, low, x;
  blocks_before(W, blockIdx.x, waves, before, all);
  const int border = (int)all / kBlockPages;  // the block in which the pages below `used` end
  if (border < W.blocks) {
    blocks_before(W, border, waves, low, x);
    const int n = (int)all - border * kBlockPages - (int)threadIdx.x * 16;  // this thread's pages below it
    const uint32_t bits = marks16<false>(W, border) & (n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1u);
    block_scan<kThreads>(__popc(bits), waves, x);
    low += x;
  } else {
    low = all;
  }
  const Plan P{(int)all, (int)low, min((int)(all - low), A.max_moves)};
  // A thread's marks and the used pages in front of them; then neighbouring threads take neighbouring pages.
  __shared__ uint32_t marks[kThreads], start[kThreads];
  const uint32_t bits = marks16<false>(W, blockIdx.x);
  marks[threadIdx.x] = bits;
  const uint32_t mine = before + block_scan<kThreads>(__popc(bits), waves, x), next = (uint32_t)__shfl_xor((int)bits, 1, 64);
  start[threadIdx.x] = mine;
  if ((threadIdx.x & 1) == 0) W.words[(blockIdx.x * kThreads + threadIdx.x) / 2] = Word{bits | next << 16, mine};
  __syncthreads();
  for (int i = 0; i < 16; ++i) {
    const int at = i * kThreads + threadIdx.x, page = blockIdx.x * kBlockPages + at;
    if (page >= A.n_pages) break;
    const uint32_t m = marks[at >> 4];
    const bool used = m >> (at & 15) & 1;
    plan_page(A, P, page, used, (int)(start[at >> 4] + __popc(m & ((1u << (at & 15)) - 1u))));
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *A.n_moves = P.moves;
    *A.n_free = (int)std::min(A.n_pages - P.used, (long long)A.free_capacity);
    *W.header = Header{P.used, P.moves};
  }
}

__global__ __launch_bounds__(kThreads) void compact_table_kernel(PageCompactArgs A, Pool W, int turns) {
  const Header H = *W.header;
  const int per_row = (A.max_pages + kEntries - 1) / kEntries;
  for (int x = blockIdx.x; x < turns; x += gridDim.x) {
    const int row = x / per_row, j0 = x % per_row * kEntries, held = held_pages(A.seq_lens[row], A.max_pages, A.log2_page);
    const int32_t* from = A.table + (size_t)row * A.max_pages;
    int32_t* to = A.new_table + (size_t)row * A.max_pages;
    constexpr int kEach = kEntries / kThreads;
    int p[kEach], r[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = j0 + i * kThreads + (int)threadIdx.x;
      p[i] = j < A.max_pages ? from[j] : -1;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = j0 + i * kThreads + (int)threadIdx.x;
      r[i] = -1;
      if (j < held && p[i] >= H.a && p[i] < A.n_pages) {
        const Word x = W.words[p[i] >> 5];
        r[i] = H.a - 1 - (int)(x.start + __popc(x.bits & ((1u << (p[i] & 31)) - 1u)));
      }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if ((unsigned)r[i] < (unsigned)H.b) p[i] = A.dst[r[i]];  // every held page was ranked, if the table is still the same
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = j0 + i * kThreads + (int)threadIdx.x;
      if (j < A.max_pages) to[j] = p[i];
    }
  }
}

// ---- one workgroup

constexpr int kOneThreads = 1024;
constexpr int kOneWords = 4096;                // words of marks in LDS
constexpr long long kOnePages = kOneWords * 32;

__global__ __launch_bounds__(kOneThreads) void release_one_kernel(PageReleaseArgs A) {
  __shared__ uint32_t now[kOneWords], before[kOneWords], waves[kOneThreads / 64];
  const int words = (int)((A.n_pages + 31) / 32);
  for (int i = threadIdx.x; i < words; i += kOneThreads) now[i] = before[i] = 0u;
  int taken, n_free;
  free_list(A, taken, n_free);
  __syncthreads();
  const int rows = release_rows(A);
  for (int row = threadIdx.x >> 6; row < rows; row += kOneThreads / 64) {
    const ReleaseRow R = release_row(A, row);
    for_pages(R.entries, threadIdx.x & 63, 64, max(R.was, R.is), A.n_pages,
              [&](int j, int p) { atomicOr((j < R.is ? now : before) + (p >> 5), 1u << (p & 31)); });
  }
  for (int i = taken + (int)threadIdx.x; i < n_free; i += kOneThreads) {
    const int p = A.free_pages[i];
    if (p >= 0 && p < A.n_pages) atomicOr(&now[p >> 5], 1u << (p & 31));
    if (i - taken < A.out_capacity) A.free_out[i - taken] = p;
  }
  __syncthreads();
  const int per = (words + kOneThreads - 1) / kOneThreads, w0 = min((int)threadIdx.x * per, words), w1 = min(w0 + per, words);
  uint32_t mine = 0, total;
  for (int w = w0; w < w1; ++w) mine += __popc(before[w] & ~now[w]);
  int at = n_free - taken + (int)block_scan<kOneThreads>(mine, waves, total);
  for (int w = w0; w < w1; ++w)
    for (uint32_t bits = before[w] & ~now[w]; bits; bits &= bits - 1, ++at)
      if (at < A.out_capacity) A.free_out[at] = w * 32 + __builtin_ctz(bits);
  if (threadIdx.x == 0) *A.n_free_out = min(n_free - taken + (int)total, A.out_capacity);
}

__global__ __launch_bounds__(kOneThreads) void compact_one_kernel(PageCompactArgs A) {
  __shared__ uint32_t marks[kOneWords], start[kOneWords], waves[kOneThreads / 64];  // start: used pages in front of a word
  const int words = (int)((A.n_pages + 31) / 32);
  for (int i = threadIdx.x; i < words; i += kOneThreads) marks[i] = 0u;
  __syncthreads();
  for (int row = threadIdx.x >> 6; row < A.batch; row += kOneThreads / 64)
    for_pages(A.table + (size_t)row * A.max_pages, threadIdx.x & 63, 64,
              held_pages(A.seq_lens[row], A.max_pages, A.log2_page), A.n_pages,
              [&](int, int p) { atomicOr(&marks[p >> 5], 1u << (p & 31)); });
  __syncthreads();
  const int per = (words + kOneThreads - 1) / kOneThreads, w0 = min((int)threadIdx.x * per, words), w1 = min(w0 + per, words);
  uint32_t mine = 0, total;
  for (int w = w0; w < w1; ++w) mine += __popc(marks[w]);
  uint32_t at = block_scan<kOneThreads>(mine, waves, total);
  for (int w = w0; w < w1; ++w) {
    start[w] = at;
    at += __popc(marks[w]);
  }
  __syncthreads();
  const auto used_before = [&](int p) {
    return (int)(start[p >> 5] + __popc(marks[p >> 5] & ((1u << (p & 31)) - 1u)));
  };
  const int low = (int)total < A.n_pages ? used_before((int)total) : (int)total;
  const Plan P{(int)total, low, min((int)total - low, A.max_moves)};
  for (int p = threadIdx.x; p < A.n_pages; p += kOneThreads)
    plan_page(A, P, p, marks[p >> 5] >> (p & 31) & 1, used_before(p));
  if (threadIdx.x == 0) {
    *A.n_moves = P.moves;
    *A.n_free = (int)std::min(A.n_pages - P.used, (long long)A.free_capacity);
  }
  __syncthreads();  // the moves are written
  const int lane = threadIdx.x & 63;
  for (int row = threadIdx.x >> 6; row < A.batch; row += kOneThreads / 64) {
    const int held = held_pages(A.seq_lens[row], A.max_pages, A.log2_page);
    const int32_t* from = A.table + (size_t)row * A.max_pages;
    int32_t* to = A.new_table + (size_t)row * A.max_pages;
    for (int j0 = lane; j0 < A.max_pages; j0 += 4 * 64) {
      int p[4], r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = j0 + i * 64 < A.max_pages ? from[j0 + i * 64] : -1;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r[i] = j0 + i * 64 < held && p[i] >= P.used && p[i] < A.n_pages ? P.used - 1 - used_before(p[i]) : -1;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((unsigned)r[i] < (unsigned)P.moves) p[i] = A.dst[r[i]];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j0 + i * 64 < A.max_pages) to[j0 + i * 64] = p[i];
    }
  }
}

int turns_of(long long rows, int max_pages) { return (int)(rows * ((max_pages + kEntries - 1) / kEntries)); }
int grid_of(long long n, int most) { return (int)std::min<long long>(std::max<long long>(n, 1), most); }

void clear(void* p, size_t bytes, hipStream_t stream) {
  const size_t n = bytes / 16;
  hipLaunchKernelGGL(clear_kernel, dim3(grid_of((long long)((n + kThreads - 1) / kThreads), 1024)), dim3(kThreads), 0, stream,
                     static_cast<u32x4_t*>(p), n);
}

// One workgroup where the tables' entries are few: it is bound by its instructions, the kernels by their launches. Release of
// 40K / 80K / 120K entries 8.9 / 14.4 / 20.7 us with one workgroup, 14 to 17 with kernels (box to box); compaction of 10K / 20K /
// 40K / 80K entries 7.1 / 12.0 / 20.7 / 38 and 17 to 20.
constexpr long long kOneRelease = 3 << 15, kOneCompact = 1 << 15;

}  // namespace

size_t page_workspace_bytes(long long n_pages) { return Pool(nullptr, n_pages).bytes; }

hipError_t launch_page_release(const PageReleaseArgs& a, hipStream_t stream) {
  if (a.n_pages <= kOnePages && (long long)release_rows(a) * a.max_pages + a.free_capacity <= kOneRelease) {
    hipLaunchKernelGGL(release_one_kernel, dim3(1), dim3(kOneThreads), 0, stream, a);
    return hipGetLastError();
  }
  const Pool W(a.workspace, a.n_pages);
  clear(W.marks, 2 * (size_t)W.blocks * kBlockPages, stream);
  const int turns = turns_of(release_rows(a), a.max_pages);
  const long long lists = ((long long)a.free_capacity + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(release_mark_kernel, dim3(grid_of(std::max<long long>(turns, lists), 2048)), dim3(kThreads), 0, stream, a,
                     W, turns);
  hipLaunchKernelGGL((count_kernel<true>), dim3(W.blocks), dim3(kThreads), 0, stream, W);
  hipLaunchKernelGGL(release_write_kernel, dim3(W.blocks), dim3(kThreads), 0, stream, a, W);
  return hipGetLastError();
}

hipError_t launch_page_compact(const PageCompactArgs& a, hipStream_t stream) {
  if (a.n_pages <= kOnePages && (long long)a.batch * a.max_pages <= kOneCompact) {
    hipLaunchKernelGGL(compact_one_kernel, dim3(1), dim3(kOneThreads), 0, stream, a);
    return hipGetLastError();
  }
  const Pool W(a.workspace, a.n_pages);
  clear(W.marks, (size_t)W.blocks * kBlockPages, stream);
  const int turns = turns_of(a.batch, a.max_pages);
  hipLaunchKernelGGL(compact_mark_kernel, dim3(grid_of(turns, 2048)), dim3(kThreads), 0, stream, a, W, turns);
  hipLaunchKernelGGL((count_kernel<false>), dim3(W.blocks), dim3(kThreads), 0, stream, W);
  hipLaunchKernelGGL(compact_plan_kernel, dim3(W.blocks), dim3(kThreads), 0, stream, a, W);
  hipLaunchKernelGGL(compact_table_kernel, dim3(grid_of(turns, 2048)), dim3(kThreads), 0, stream, a, W, turns);
  return hipGetLastError();
}

}  // namespace cosa
