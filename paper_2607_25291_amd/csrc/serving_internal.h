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

}  // namespace cosa
