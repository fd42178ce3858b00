// C ABI of the serving operators (include/cosa_serving.h): host-side validation, workspaces and launches. Every entry
// point validates all arguments before enqueuing anything.
#include <math.h>

#include "api_checks.h"
#include "cosa_serving.h"
#include "serving_internal.h"

namespace {

using cosa::check_n_pages;
using cosa::check_page_size;
using cosa::check_workspace;
using cosa::ChunkShape;
using cosa::fail;
using cosa::launch;
using cosa::misaligned;
using cosa::ok;
using cosa::Span;
using cosa::u16;

// Validates the problem; `empty` is set where no row is asked for.
cosa_status check_chunk(const cosa_chunk_problem* p, int page_size, ChunkShape& sh, bool& empty) {
  if (!p) return fail(COSA_ERR_INVALID_ARG, "problem is NULL");
  if (p->batch < 0 || p->max_pages < 0 || p->n_rows < 0)
    return fail(COSA_ERR_INVALID_ARG, "batch (%d), max_pages (%d) and n_rows (%d) must be >= 0", p->batch, p->max_pages,
                p->n_rows);
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0)
    return fail(COSA_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", p->n_q_heads,
                p->n_kv_heads);
  if (p->head_dim < 1) return fail(COSA_ERR_INVALID_ARG, "head_dim must be >= 1");
  if (p->head_dim != cosa::kHeadDim) return fail(COSA_ERR_UNSUPPORTED, "head_dim %d (supported: 128)", p->head_dim);
  if (!(p->sm_scale >= 0.f) || !isfinite(p->sm_scale))
    return fail(COSA_ERR_INVALID_ARG, "sm_scale must be finite and >= 0 (0 = 1/sqrt(d))");
  const int64_t dense = (int64_t)p->n_q_heads * p->head_dim;
  if ((p->q_stride != 0 && p->q_stride < dense) || p->q_stride % 8 != 0)
    return fail(COSA_ERR_INVALID_ARG, "q_stride %lld: 0, or a multiple of 8 of at least n_q_heads * head_dim = %lld",
                (long long)p->q_stride, (long long)dense);
  cosa_status st = check_page_size(page_size, sh.log2_page);
  if (st != COSA_OK) return st;
  if (((int64_t)p->max_pages << sh.log2_page) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "max_pages (%d) * page_size (%d) must stay below 2^31 tokens", p->max_pages, page_size);
  if (p->batch >= (1 << 22) || p->n_rows >= (1 << 22) || (int64_t)p->n_rows * p->n_q_heads >= (1ll << 31) ||
      (double)p->q_stride * p->n_rows > 1e18)
    return fail(COSA_ERR_UNSUPPORTED, "%d sequences, %d rows of %d heads: too large for one launch", p->batch, p->n_rows,
                p->n_q_heads);
  sh.B = p->batch;
  sh.Hq = p->n_q_heads;
  sh.Hkv = p->n_kv_heads;
  sh.G = p->n_q_heads / p->n_kv_heads;
  sh.max_pages = p->max_pages;
  sh.n_rows = p->n_rows;
  sh.q_stride = p->q_stride ? p->q_stride : dense;
  sh.n_pages = 1;
  sh.scale = p->sm_scale > 0.f ? p->sm_scale : (float)(1.0 / sqrt((double)p->head_dim));
  empty = p->batch == 0 || p->n_rows == 0;
  return ok();
}

}  // namespace

extern "C" {

size_t cosa_chunk_workspace_bytes(const cosa_chunk_problem* problem) {
  ChunkShape sh{};
  bool empty = false;
  if (check_chunk(problem, 16, sh, empty) != COSA_OK) return 0;
  return cosa::chunk_workspace_bytes(sh);
}

cosa_status cosa_chunk_attention(const cosa_chunk_problem* problem, const void* q, const cosa_paged_kv* kv,
                                 const int32_t* seq_lens, const int32_t* cu_new, void* workspace,
                                 size_t workspace_bytes, void* o, float* lse, void* stream) {
  if (!kv) return fail(COSA_ERR_INVALID_ARG, "paged kv is NULL");
  ChunkShape sh{};
  bool empty = false;
  cosa_status st = check_chunk(problem, kv->page_size, sh, empty);
  if (st != COSA_OK) return st;
  if ((st = check_n_pages(kv->n_pages)) != COSA_OK) return st;
  sh.n_pages = kv->n_pages;
  if (empty) return ok();
  if (sh.max_pages > 0 && !kv->page_table) return fail(COSA_ERR_INVALID_ARG, "page_table must be non-NULL");
  if (!kv->k_cache || !kv->v_cache || !q || !seq_lens || !cu_new || !o)
    return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache, q, seq_lens, cu_new and o must be non-NULL");
  for (const void* p : {(const void*)kv->k_cache, (const void*)kv->v_cache, q, (const void*)o})
    if (misaligned(p, 16)) return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache, q and o must be 16-byte aligned");
  if ((st = check_workspace(workspace, workspace_bytes, cosa::chunk_workspace_bytes(sh))) != COSA_OK) return st;
  const int64_t row = 2ll * sh.Hq * cosa::kHeadDim;
  const Span queries{q, 2 * (sh.n_rows - 1) * sh.q_stride + row}, out{o, sh.n_rows * row},
      sums{lse, 4ll * sh.n_rows * sh.Hq}, scratch{workspace, (int64_t)cosa::chunk_workspace_bytes(sh)};
  if (out.meets(queries) || sums.meets(queries) || scratch.meets(queries))
    return fail(COSA_ERR_INVALID_ARG, "o, lse and the workspace must not overlap q");
  if (out.meets(sums) || out.meets(scratch) || sums.meets(scratch))
    return fail(COSA_ERR_INVALID_ARG, "o, lse and the workspace must not overlap each other");
  const cosa::ChunkArgs a{u16(q), u16(kv->k_cache), u16(kv->v_cache), kv->page_table, seq_lens, cu_new, workspace,
                          static_cast<uint16_t*>(o), lse};
  return launch(stream, "chunk_attention launch",
                [&](hipStream_t s) { return cosa::launch_chunk_attention(sh, a, s); });
}

}  // extern "C"
