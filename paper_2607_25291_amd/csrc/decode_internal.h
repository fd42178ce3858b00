// Internal interface between the C layer of the decode-side operators (decode_api.hip) and their
// kernels. Every launcher enqueues on `stream` and returns the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cosa_internal.h"

namespace cosa {

constexpr int kMaxRequests = 8192;      // requests of one cosa_page_map (two prefix arrays in LDS)
constexpr int kMaxSelectPages = 32768;  // pages of one row of cosa_page_select (32-bit keys in LDS)
constexpr int kMaxSelectHeads = 1024;   // query heads of one KV head there

// A validated decode problem with its cache.
struct DecodeShape {
  int B, Hq, Hkv, G;
  int max_pages, log2_page;
  long long q_stride, n_pages;
  float scale;
  int cap() const { return max_pages << log2_page; }  // tokens a sequence can hold, < 2^31
};

struct PageMapArgs {
  int batch, log2_page, max_pages, free_capacity, max_new;
  const int32_t *cached, *add, *free_pages, *n_free;
  int32_t *table, *seq_lens, *cu_new, *n_taken;
  int64_t* slots;
};
hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream);

struct AppendArgs {
  int Hkv, log2_page;
  long long n_pages, n_tokens, k_stride, v_stride;
  uint16_t *k_cache, *v_cache, *bounds;
  const uint16_t *k, *v;
  const int64_t* slots;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);

constexpr int kScorePages = 16;  // pages of a wave of cosa_page_score
hipError_t launch_page_score(const DecodeShape& sh, const uint16_t* q, const uint16_t* bounds,
                             const int32_t* table, const int32_t* seq_lens, float* score,
                             hipStream_t stream);

struct PageSelectArgs {
  int B, Hq, Hkv, G, max_pages, log2_page;
  const int32_t* seq_lens;
  const float* score;
  int64_t fraction_micro;
  int min_keep, max_keep, sink, recent;  // max_keep: width of a list
  int32_t *pages, *count;
};
hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t stream);

struct DecodeArgs {
  const uint16_t *q, *k_cache, *v_cache;
  const int32_t *table, *seq_lens;
  const int32_t *pages, *count;  // lists per KV head, or nullptr: every page
  int list_pages;
  void* workspace;
  uint16_t* o;
  float* lse;  // optional
};
// Scratch of a decode attention call that decode_fits.
size_t decode_workspace_bytes(const DecodeShape& sh);
// Whether the units and tiles of a call (capacity `tokens` per sequence and KV head) fit a grid and 31 bits.
bool decode_fits(const DecodeShape& sh, long long tokens);
hipError_t launch_decode_attention(const DecodeShape& sh, const DecodeArgs& a, hipStream_t stream);

}  // namespace cosa
