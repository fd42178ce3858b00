// Internal interface between the C layer of the serving operators (serving_api.hip) and their kernels. Every
// launcher enqueues on `stream` and returns the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cosa_internal.h"

namespace cosa {

// A validated chunk problem with its cache.
struct ChunkShape {
  int B, Hq, Hkv, G;
  int max_pages, log2_page, n_rows;
  long long q_stride, n_pages;
  float scale;
  int cap() const { return max_pages << log2_page; }  // tokens a sequence can hold, < 2^31
};

struct ChunkArgs {
  const uint16_t *q, *k_cache, *v_cache;
  const int32_t *table, *seq_lens, *cu_new;
  void* workspace;
  uint16_t* o;
  float* lse;  // optional
};
size_t chunk_workspace_bytes(const ChunkShape& sh);
hipError_t launch_chunk_attention(const ChunkShape& sh, const ChunkArgs& a, hipStream_t stream);

constexpr int kMaxForkRows = 8192;            // rows of either table of one cosa_page_fork (ranks in LDS)
constexpr long long kMaxPoolPages = 1 << 28;  // pages of a cache that cosa_page_release and cosa_page_compact look over

struct PageForkArgs {
  int n_parents, n_children, log2_page, max_pages, copy_all, free_capacity;
  const int32_t *parent, *table, *seq_lens, *free_pages, *n_free;
  int32_t *new_table, *new_lens, *src, *dst, *rows, *n_taken;
};
hipError_t launch_page_fork(const PageForkArgs& a, hipStream_t stream);

struct PageCopyArgs {
  int Hkv, log2_page, max_pairs;
  long long n_pages;
  uint16_t *k_cache, *v_cache, *bounds;             // bounds: optional
  const int32_t *src, *dst, *rows, *n_pairs;        // rows: optional
};
// Stretches of 64 rows that one pair's copy has.
long long page_copy_items(int Hkv, int log2_page, bool bounds);
hipError_t launch_page_copy(const PageCopyArgs& a, hipStream_t stream);

struct PageReleaseArgs {
  int log2_page, max_pages, old_batch, new_batch, free_capacity, out_capacity;
  long long n_pages;
  const int32_t *old_table, *old_lens, *new_table, *new_lens, *free_pages, *n_free, *n_taken;  // n_taken: optional
  int32_t *free_out, *n_free_out;
  void* workspace;
};
struct PageCompactArgs {
  int batch, log2_page, max_pages, max_moves, free_capacity;
  long long n_pages;
  const int32_t *table, *seq_lens;
  int32_t *new_table, *src, *dst, *n_moves, *free_pages, *n_free;
  void* workspace;
};
size_t page_workspace_bytes(long long n_pages);  // of either call
hipError_t launch_page_release(const PageReleaseArgs& a, hipStream_t stream);
hipError_t launch_page_compact(const PageCompactArgs& a, hipStream_t stream);

}  // namespace cosa
