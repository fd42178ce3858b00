// C ABI of the serving operators (include/cosa_serving.h): host-side validation, workspaces and launches. Every entry
// point validates all arguments before enqueuing anything.
#include <math.h>

#include "api_checks.h"
#include "chunk_split.h"
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
  if (!cosa::chunk_fits(sh.B, sh.n_rows, sh.cap(), (int64_t)sh.Hkv * cosa::chunk_parts(sh.G), cosa::chunk_tokens(sh.G)))
    return fail(COSA_ERR_UNSUPPORTED, "%d sequences of up to %d tokens and %d rows: too large for one launch", sh.B, sh.cap(),
                sh.n_rows);
  empty = p->batch == 0 || p->n_rows == 0;
  return ok();
}

// A table of `batch` rows: its sizes, and what a row holds in 31 bits.
cosa_status check_table(int32_t batch, int32_t max_pages, int32_t page_size, int& log2_page) {
  if (batch < 0 || max_pages < 0)
    return fail(COSA_ERR_INVALID_ARG, "rows (%d) and max_pages (%d) must be >= 0", batch, max_pages);
  const cosa_status st = check_page_size(page_size, log2_page);
  if (st != COSA_OK) return st;
  if (((int64_t)max_pages << log2_page) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "max_pages (%d) * page_size (%d) must stay below 2^31 tokens", max_pages, page_size);
  if ((int64_t)batch * max_pages >= (1ll << 31) || batch >= (1 << 24))
    return fail(COSA_ERR_UNSUPPORTED, "a table of %d rows of %d pages is too large for one launch", batch, max_pages);
  return ok();
}

cosa_status check_pool(int64_t n_pages) {
  const cosa_status st = check_n_pages(n_pages);
  if (st != COSA_OK) return st;
  if (n_pages > cosa::kMaxPoolPages)
    return fail(COSA_ERR_UNSUPPORTED, "%lld pages (supported: <= 2^28)", (long long)n_pages);
  return ok();
}

// Outputs against inputs and against each other.
template <size_t N, size_t M>
cosa_status check_apart(const Span (&out)[N], const Span (&in)[M], const char* what) {
  for (size_t i = 0; i < N; ++i) {
    for (const Span& x : in)
      if (out[i].meets(x)) return fail(COSA_ERR_INVALID_ARG, "%s must not overlap the inputs", what);
    for (size_t j = 0; j < i; ++j)
      if (out[i].meets(out[j])) return fail(COSA_ERR_INVALID_ARG, "%s must not overlap each other", what);
  }
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
  // Other workgroups read all inputs until the call's end.
  const int64_t row = 2ll * sh.Hq * cosa::kHeadDim;
  const double pages = 2.0 * cosa::kHeadDim * sh.n_pages * sh.Hkv * kv->page_size;
  const int64_t cache = pages < 1e18 ? 2ll * cosa::kHeadDim * sh.n_pages * sh.Hkv * kv->page_size : (int64_t)1e18;
  const Span in[] = {{q, 2 * (sh.n_rows - 1) * sh.q_stride + row}, {kv->k_cache, cache}, {kv->v_cache, cache},
                     {kv->page_table, 4ll * sh.B * sh.max_pages}, {seq_lens, 4ll * sh.B}, {cu_new, 4ll * (sh.B + 1)}};
  const Span out[] = {{o, sh.n_rows * row}, {lse, 4ll * sh.n_rows * sh.Hq},
                      {workspace, (int64_t)cosa::chunk_workspace_bytes(sh)}};
  if ((st = check_apart(out, in, "o, lse and the workspace")) != COSA_OK) return st;
  const cosa::ChunkArgs a{u16(q), u16(kv->k_cache), u16(kv->v_cache), kv->page_table, seq_lens, cu_new, workspace,
                          static_cast<uint16_t*>(o), lse};
  return launch(stream, "chunk_attention launch",
                [&](hipStream_t s) { return cosa::launch_chunk_attention(sh, a, s); });
}

cosa_status cosa_page_fork(int32_t n_parents, int32_t n_children, int32_t page_size, int32_t max_pages,
                           const int32_t* parent, const int32_t* page_table, const int32_t* seq_lens, int32_t copy_all,
                           const int32_t* free_pages, int32_t free_capacity, const int32_t* n_free, int32_t* new_table,
                           int32_t* new_lens, int32_t* src, int32_t* dst, int32_t* rows, int32_t* n_taken, void* stream) {
  cosa::PageForkArgs a{};
  cosa_status st = check_table(n_parents, max_pages, page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if (n_children < 0 || free_capacity < 0)
    return fail(COSA_ERR_INVALID_ARG, "n_children (%d) and free_capacity (%d) must be >= 0", n_children, free_capacity);
  if (n_parents > cosa::kMaxForkRows || n_children > cosa::kMaxForkRows)
    return fail(COSA_ERR_UNSUPPORTED, "%d rows from %d (supported: <= %d)", n_children, n_parents, cosa::kMaxForkRows);
  if (!n_free || !n_taken) return fail(COSA_ERR_INVALID_ARG, "n_free and n_taken must be non-NULL");
  const bool some = n_children > 0, from = some && n_parents > 0, entries = max_pages > 0;
  if ((some && (!parent || !new_lens || !src || !dst || !rows || (entries && !new_table))) ||
      (from && (!seq_lens || (entries && !page_table))) || (some && free_capacity > 0 && !free_pages))
    return fail(COSA_ERR_INVALID_ARG,
                "parent, page_table, seq_lens, free_pages, new_table, new_lens, src, dst and rows must be non-NULL where they hold entries");
  const int64_t b = n_parents, c = n_children, w = max_pages;
  const Span in[] = {{parent, 4 * c}, {page_table, 4 * b * w}, {seq_lens, 4 * b}, {free_pages, 4ll * free_capacity}, {n_free, 4}};
  const Span out[] = {{new_table, 4 * c * w}, {new_lens, 4 * c}, {src, 4 * c}, {dst, 4 * c}, {rows, 4 * c}, {n_taken, 4}};
  if ((st = check_apart(out, in, "new_table, new_lens, src, dst, rows and n_taken")) != COSA_OK) return st;
  a.n_parents = n_parents;
  a.n_children = n_children;
  a.max_pages = max_pages;
  a.copy_all = copy_all;
  a.free_capacity = free_capacity;
  a.parent = parent;
  a.table = page_table;
  a.seq_lens = seq_lens;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.new_table = new_table;
  a.new_lens = new_lens;
  a.src = src;
  a.dst = dst;
  a.rows = rows;
  a.n_taken = n_taken;
  return launch(stream, "page_fork launch", [&](hipStream_t s) { return cosa::launch_page_fork(a, s); });
}

cosa_status cosa_page_copy(int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int64_t n_pages, void* k_cache,
                           void* v_cache, void* bounds, const int32_t* src, const int32_t* dst, const int32_t* rows,
                           int32_t max_pairs, const int32_t* n_pairs, void* stream) {
  if (n_kv_heads < 1 || head_dim < 1 || max_pairs < 0)
    return fail(COSA_ERR_INVALID_ARG, "n_kv_heads (%d) and head_dim (%d) must be >= 1, max_pairs (%d) >= 0", n_kv_heads,
                head_dim, max_pairs);
  if (head_dim != cosa::kHeadDim) return fail(COSA_ERR_UNSUPPORTED, "head_dim %d (supported: 128)", head_dim);
  cosa::PageCopyArgs a{};
  cosa_status st = check_page_size(page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if ((st = check_n_pages(n_pages)) != COSA_OK) return st;
  const int64_t rows_of_page = (int64_t)n_kv_heads << a.log2_page;
  if (rows_of_page >= (1ll << 30) || (double)n_pages * (double)rows_of_page * head_dim > 1e18 ||
      (double)max_pairs * (double)cosa::page_copy_items(n_kv_heads, a.log2_page, true) >= 2147483648.0)
    return fail(COSA_ERR_UNSUPPORTED, "%d pairs of pages of %d heads and %d tokens: too large for one launch", max_pairs,
                n_kv_heads, page_size);
  if (max_pairs == 0) return ok();
  if (!k_cache || !v_cache || !src || !dst || !n_pairs)
    return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache, src, dst and n_pairs must be non-NULL");
  for (const void* p : {(const void*)k_cache, (const void*)v_cache, (const void*)bounds})
    if (misaligned(p, 16)) return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache and bounds must be 16-byte aligned");
  const int64_t cache = 2ll * n_pages * rows_of_page * head_dim, list = 4ll * max_pairs;
  const Span in[] = {{src, list}, {dst, list}, {rows, list}, {n_pairs, 4}};
  const Span out[] = {{k_cache, cache}, {v_cache, cache}, {bounds, 4ll * n_pages * n_kv_heads * head_dim}};
  if ((st = check_apart(out, in, "k_cache, v_cache and bounds")) != COSA_OK) return st;
  a.Hkv = n_kv_heads;
  a.n_pages = n_pages;
  a.max_pairs = max_pairs;
  a.k_cache = static_cast<uint16_t*>(k_cache);
  a.v_cache = static_cast<uint16_t*>(v_cache);
  a.bounds = static_cast<uint16_t*>(bounds);
  a.src = src;
  a.dst = dst;
  a.rows = rows;
  a.n_pairs = n_pairs;
  return launch(stream, "page_copy launch", [&](hipStream_t s) { return cosa::launch_page_copy(a, s); });
}

size_t cosa_page_workspace_bytes(int64_t n_pages) {
  return check_pool(n_pages) == COSA_OK ? cosa::page_workspace_bytes(n_pages) : 0;
}

cosa_status cosa_page_release(int32_t page_size, int32_t max_pages, int64_t n_pages, int32_t old_batch,
                              const int32_t* old_table, const int32_t* old_lens, int32_t new_batch,
                              const int32_t* new_table, const int32_t* new_lens, const int32_t* free_pages,
                              int32_t free_capacity, const int32_t* n_free, const int32_t* n_taken, int32_t* free_out,
                              int32_t out_capacity, int32_t* n_free_out, void* workspace, size_t workspace_bytes,
                              void* stream) {
  cosa::PageReleaseArgs a{};
  cosa_status st = check_table(old_batch, max_pages, page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if ((st = check_table(new_batch, max_pages, page_size, a.log2_page)) != COSA_OK) return st;
  if (((int64_t)old_batch + new_batch) * ((max_pages + 1023) / 1024) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "tables of %d and %d rows are too large for one launch", old_batch, new_batch);
  if ((st = check_pool(n_pages)) != COSA_OK) return st;
  if (free_capacity < 0 || out_capacity < 0)
    return fail(COSA_ERR_INVALID_ARG, "free_capacity (%d) and out_capacity (%d) must be >= 0", free_capacity, out_capacity);
  if (free_capacity > cosa::kMaxPoolPages)
    return fail(COSA_ERR_UNSUPPORTED, "a free list of %d pages (supported: <= 2^28)", free_capacity);
  if (!n_free || !n_free_out) return fail(COSA_ERR_INVALID_ARG, "n_free and n_free_out must be non-NULL");
  const bool entries = max_pages > 0;
  if ((old_batch > 0 && (!old_lens || (entries && !old_table))) || (new_batch > 0 && (!new_lens || (entries && !new_table))) ||
      (free_capacity > 0 && !free_pages) || (out_capacity > 0 && !free_out))
    return fail(COSA_ERR_INVALID_ARG, "tables, lengths, free_pages and free_out must be non-NULL where they hold entries");
  if ((st = check_workspace(workspace, workspace_bytes, cosa::page_workspace_bytes(n_pages))) != COSA_OK) return st;
  const int64_t w = max_pages;
  const Span in[] = {{old_table, 4 * old_batch * w}, {old_lens, 4ll * old_batch}, {new_table, 4 * new_batch * w},
                     {new_lens, 4ll * new_batch}, {free_pages, 4ll * free_capacity}, {n_taken, 4},
                     {n_free, n_free_out == n_free ? 0 : 4}};
  const Span out[] = {{free_out, 4ll * out_capacity}, {n_free_out, 4},
                      {workspace, (int64_t)cosa::page_workspace_bytes(n_pages)}};
  if ((st = check_apart(out, in, "free_out, n_free_out and the workspace")) != COSA_OK) return st;
  a.max_pages = max_pages;
  a.old_batch = old_batch;
  a.new_batch = new_batch;
  a.free_capacity = free_capacity;
  a.out_capacity = out_capacity;
  a.n_pages = n_pages;
  a.old_table = old_table;
  a.old_lens = old_lens;
  a.new_table = new_table;
  a.new_lens = new_lens;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.n_taken = n_taken;
  a.free_out = free_out;
  a.n_free_out = n_free_out;
  a.workspace = workspace;
  return launch(stream, "page_release launch", [&](hipStream_t s) { return cosa::launch_page_release(a, s); });
}

cosa_status cosa_page_compact(int32_t batch, int32_t page_size, int32_t max_pages, int64_t n_pages,
                              const int32_t* page_table, const int32_t* seq_lens, int32_t max_moves, int32_t* new_table,
                              int32_t* src, int32_t* dst, int32_t* n_moves, int32_t* free_pages, int32_t free_capacity,
                              int32_t* n_free, void* workspace, size_t workspace_bytes, void* stream) {
  cosa::PageCompactArgs a{};
  cosa_status st = check_table(batch, max_pages, page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if ((st = check_pool(n_pages)) != COSA_OK) return st;
  if (max_moves < 0 || free_capacity < 0)
    return fail(COSA_ERR_INVALID_ARG, "max_moves (%d) and free_capacity (%d) must be >= 0", max_moves, free_capacity);
  if (!n_moves || !n_free) return fail(COSA_ERR_INVALID_ARG, "n_moves and n_free must be non-NULL");
  if ((batch > 0 && (!seq_lens || (max_pages > 0 && (!page_table || !new_table)))) || (max_moves > 0 && (!src || !dst)) ||
      (free_capacity > 0 && !free_pages))
    return fail(COSA_ERR_INVALID_ARG,
                "page_table, seq_lens, new_table, src, dst and free_pages must be non-NULL where they hold entries");
  if ((st = check_workspace(workspace, workspace_bytes, cosa::page_workspace_bytes(n_pages))) != COSA_OK) return st;
  const int64_t table = 4ll * batch * max_pages;
  const Span in[] = {{page_table, new_table == page_table ? 0 : table}, {seq_lens, 4ll * batch}};
  const Span out[] = {{new_table, table}, {src, 4ll * max_moves}, {dst, 4ll * max_moves}, {n_moves, 4},
                      {free_pages, 4ll * free_capacity}, {n_free, 4},
                      {workspace, (int64_t)cosa::page_workspace_bytes(n_pages)}};
  if ((st = check_apart(out, in, "new_table, src, dst, n_moves, free_pages, n_free and the workspace")) != COSA_OK) return st;
  a.batch = batch;
  a.max_pages = max_pages;
  a.max_moves = max_moves;
  a.free_capacity = free_capacity;
  a.n_pages = n_pages;
  a.table = page_table;
  a.seq_lens = seq_lens;
  a.new_table = new_table;
  a.src = src;
  a.dst = dst;
  a.n_moves = n_moves;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.workspace = workspace;
  return launch(stream, "page_compact launch", [&](hipStream_t s) { return cosa::launch_page_compact(a, s); });
}

}  // extern "C"
