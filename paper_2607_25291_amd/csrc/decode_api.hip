// C ABI of the decode-side operators (include/cosa_decode.h): host-side validation, workspace layout and
// launches. Every entry point validates all arguments before enqueuing anything.
#include <math.h>

#include <algorithm>

#include "api_status.h"
#include "cosa_decode.h"
#include "decode_internal.h"

namespace {

using cosa::align256;
using cosa::as_stream;
using cosa::DecodeShape;
using cosa::fail;
using cosa::hip_fail;
using cosa::ok;

// Makes the device of `stream` current for the launches of one call (null, legacy and per-thread streams belong to the current device).
class OnDevice {
 public:
  explicit OnDevice(hipStream_t stream) {
    // the null stream, the legacy and the per-thread one belong to whichever device is current
    if (stream == nullptr || stream == hipStreamLegacy || stream == hipStreamPerThread) return;
    hipDevice_t dev;
    if ((err_ = hipGetDevice(&before_)) != hipSuccess) return;
    if ((err_ = hipStreamGetDevice(stream, &dev)) != hipSuccess) return;
    if ((int)dev == before_) return;
    err_ = hipSetDevice((int)dev);
    moved_ = err_ == hipSuccess;
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool moved_ = false;
  hipError_t err_ = hipSuccess;
};

template <class F>
cosa_status launch(void* stream, const char* what, F&& f) {
  const hipStream_t s = as_stream(stream);
  const OnDevice device(s);
  hipError_t e = device.error();
  if (e != hipSuccess) return hip_fail(e, "device of the stream");
  e = f(s);
  return e == hipSuccess ? ok() : hip_fail(e, what);
}

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// A range of memory that a call reads or writes.
struct Span {
  const void* p;
  int64_t bytes;
  bool meets(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && bytes > 0 && o.bytes > 0 && a < b + (uintptr_t)o.bytes && b < a + (uintptr_t)bytes;
  }
};

cosa_status check_page_size(int ps, int& log2_page) {
  if (ps < 16 || ps > (1 << 20) || (ps & (ps - 1)) != 0)
    return fail(COSA_ERR_INVALID_ARG, "page_size %d is not a power of two in [16, 2^20]", ps);
  log2_page = 0;
  while ((1 << log2_page) < ps) ++log2_page;
  return ok();
}

cosa_status check_n_pages(int64_t n) {
  if (n < 1 || n > (1ll << 31))
    return fail(COSA_ERR_INVALID_ARG, "n_pages (%lld) outside [1, 2^31]", (long long)n);
  return ok();
}

// Validates the problem; `empty` is set for batch == 0.
cosa_status check_problem(const cosa_decode_problem* p, int page_size, DecodeShape& sh, bool& empty) {
  if (!p) return fail(COSA_ERR_INVALID_ARG, "problem is NULL");
  if (p->batch < 0 || p->max_pages < 0)
    return fail(COSA_ERR_INVALID_ARG, "batch (%d) and max_pages (%d) must be >= 0", p->batch, p->max_pages);
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0)
    return fail(COSA_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", p->n_q_heads,
                p->n_kv_heads);
  if (p->head_dim < 1) return fail(COSA_ERR_INVALID_ARG, "head_dim must be >= 1");
  if (p->head_dim != cosa::kHeadDim) return fail(COSA_ERR_UNSUPPORTED, "head_dim %d (supported: 128)", p->head_dim);
  if (!(p->sm_scale >= 0.f) || !isfinite(p->sm_scale))
    return fail(COSA_ERR_INVALID_ARG, "sm_scale must be finite and >= 0 (0 = 1/sqrt(d))");
  const int64_t dense = (int64_t)p->n_q_heads * p->head_dim;
  if (p->q_stride != 0 && p->q_stride < dense)
    return fail(COSA_ERR_INVALID_ARG, "q_stride (%lld) below n_q_heads * head_dim = %lld", (long long)p->q_stride,
                (long long)dense);
  if (p->q_stride % 8 != 0) return fail(COSA_ERR_INVALID_ARG, "q_stride must be a multiple of 8 elements");
  cosa_status st = check_page_size(page_size, sh.log2_page);
  if (st != COSA_OK) return st;
  if (((int64_t)p->max_pages << sh.log2_page) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "max_pages (%d) * page_size (%d) must stay below 2^31 tokens", p->max_pages, page_size);
  sh.B = p->batch;
  sh.Hq = p->n_q_heads;
  sh.Hkv = p->n_kv_heads;
  sh.G = p->n_q_heads / p->n_kv_heads;
  sh.max_pages = p->max_pages;
  sh.q_stride = p->q_stride ? p->q_stride : dense;
  sh.n_pages = 1;
  sh.scale = p->sm_scale > 0.f ? p->sm_scale : (float)(1.0 / sqrt((double)p->head_dim));
  empty = p->batch == 0;
  if (!cosa::decode_fits(sh, 0)) return fail(COSA_ERR_UNSUPPORTED, "batch (%d) too large for one launch", p->batch);
  return ok();
}

cosa_status check_kv(const cosa_paged_kv* kv, bool caches, DecodeShape& sh) {
  cosa_status st = check_n_pages(kv->n_pages);
  if (st != COSA_OK) return st;
  sh.n_pages = kv->n_pages;
  if (sh.B > 0 && sh.max_pages > 0 && !kv->page_table) return fail(COSA_ERR_INVALID_ARG, "page_table must be non-NULL");
  if (!caches) return ok();
  if (!kv->k_cache || !kv->v_cache) return fail(COSA_ERR_INVALID_ARG, "k_cache and v_cache must be non-NULL");
  if (misaligned(kv->k_cache, 16) || misaligned(kv->v_cache, 16))
    return fail(COSA_ERR_INVALID_ARG, "k_cache and v_cache must be 16-byte aligned");
  return ok();
}

cosa_status check_budget(const cosa_page_budget* b, int64_t& micro) {
  if (!b) return fail(COSA_ERR_INVALID_ARG, "budget is NULL");
  if (!(b->fraction > 0.f && b->fraction <= 1.f))
    return fail(COSA_ERR_INVALID_ARG, "budget fraction %g outside (0, 1]", (double)b->fraction);
  if (b->min_pages < 1 || b->min_pages > b->max_pages)
    return fail(COSA_ERR_INVALID_ARG, "budget pages %d .. %d (1 <= min_pages <= max_pages)", b->min_pages, b->max_pages);
  if (b->sink_pages < 0 || b->recent_pages < 0 || (int64_t)b->sink_pages + b->recent_pages > b->max_pages)
    return fail(COSA_ERR_INVALID_ARG, "sink_pages (%d) and recent_pages (%d) must be >= 0 and together at most max_pages (%d)",
                b->sink_pages, b->recent_pages, b->max_pages);
  micro = (int64_t)floor((double)b->fraction * 1e6 + 0.5);
  return ok();
}

cosa_status check_select_space(const DecodeShape& sh) {
  if (sh.max_pages > cosa::kMaxSelectPages || sh.G > cosa::kMaxSelectHeads)
    return fail(COSA_ERR_UNSUPPORTED, "%d pages and %d query heads per KV head (supported: <= %d and %d)", sh.max_pages,
                sh.G, cosa::kMaxSelectPages, cosa::kMaxSelectHeads);
  return ok();
}

cosa_status check_tokens(const DecodeShape& sh, int64_t pages) {
  if ((pages << sh.log2_page) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "lists of %lld pages must stay below 2^31 tokens", (long long)pages);
  if (!cosa::decode_fits(sh, pages << sh.log2_page)) return fail(COSA_ERR_UNSUPPORTED, "problem too large for one launch");
  return ok();
}

cosa_status check_score_space(const DecodeShape& sh) {
  const int64_t waves = (int64_t)sh.B * sh.Hkv * ((sh.G + 15) / 16) *
                        ((sh.max_pages + cosa::kScorePages - 1) / cosa::kScorePages);
  if (waves >= (1ll << 26))  // 2^32 threads of a grid
    return fail(COSA_ERR_UNSUPPORTED, "%d sequences of %d pages: too large for one launch", sh.B, sh.max_pages);
  return ok();
}

cosa_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || bytes < need) return fail(COSA_ERR_WORKSPACE, "workspace of %zu bytes at %p, need %zu", bytes, ws, need);
  if (misaligned(ws, 16)) return fail(COSA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  return ok();
}

cosa_status check_q(const void* q) {
  if (!q || misaligned(q, 16)) return fail(COSA_ERR_INVALID_ARG, "q must be non-NULL and 16-byte aligned");
  return ok();
}

// Other workgroups may still read queries when one writes its outputs.
cosa_status check_o(const DecodeShape& sh, const void* q, const int32_t* seq_lens, const void* o) {
  if (!seq_lens || !o || misaligned(o, 16))
    return fail(COSA_ERR_INVALID_ARG, "seq_lens and o must be non-NULL, o 16-byte aligned");
  const int64_t row = 2ll * sh.Hq * cosa::kHeadDim;
  if (Span{q, 2 * (sh.B - 1) * sh.q_stride + row}.meets({o, sh.B * row}))
    return fail(COSA_ERR_INVALID_ARG, "o must not overlap q");
  return ok();
}

const uint16_t* u16(const void* p) { return static_cast<const uint16_t*>(p); }

// Problem, cache and lengths of the attention calls, up to the workspace.
cosa_status attention_shape(const cosa_decode_problem* problem, const cosa_paged_kv* kv, DecodeShape& sh, bool& empty) {
  if (!kv) return fail(COSA_ERR_INVALID_ARG, "paged kv is NULL");
  cosa_status st = check_problem(problem, kv->page_size, sh, empty);
  if (st != COSA_OK) return st;
  return check_kv(kv, true, sh);
}

cosa_status attention(const DecodeShape& sh, const cosa_paged_kv* kv, const void* q, const int32_t* seq_lens,
                      const int32_t* pages, const int32_t* count, int list_pages, void* workspace, size_t workspace_bytes,
                      void* o, float* lse, void* stream) {
  cosa_status st = check_q(q);
  if (st != COSA_OK) return st;
  if ((st = check_o(sh, q, seq_lens, o)) != COSA_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, cosa::decode_workspace_bytes(sh))) != COSA_OK) return st;
  const cosa::DecodeArgs a{u16(q), u16(kv->k_cache), u16(kv->v_cache), kv->page_table, seq_lens, pages, count,
                           list_pages, workspace, static_cast<uint16_t*>(o), lse};
  return launch(stream, "decode_attention launch",
                [&](hipStream_t s) { return cosa::launch_decode_attention(sh, a, s); });
}

cosa_status sparse_layout(const cosa_decode_problem* problem, const cosa_page_budget* budget, DecodeShape& sh,
                          int64_t& micro, bool& empty, cosa_decode_sparse_layout& l) {
  // the layout does not depend on the page size: the smallest one admits the most pages
  cosa_status st = check_problem(problem, 16, sh, empty);
  if (st != COSA_OK) return st;
  if ((st = check_budget(budget, micro)) != COSA_OK) return st;
  if ((st = check_select_space(sh)) != COSA_OK) return st;
  const size_t rows = (size_t)sh.B * sh.Hkv;
  l.score = 0;
  l.pages = align256(l.score + (size_t)sh.B * sh.Hq * sh.max_pages * sizeof(float));
  l.count = align256(l.pages + rows * budget->max_pages * sizeof(int32_t));
  l.partial = align256(l.count + rows * sizeof(int32_t));
  l.total = align256(l.partial + cosa::decode_workspace_bytes(sh));
  return ok();
}

}  // namespace

extern "C" {

cosa_status cosa_page_map(int32_t batch, int32_t page_size, int32_t max_pages, const int32_t* cached_lens,
                          const int32_t* new_lens, const int32_t* free_pages, int32_t free_capacity,
                          const int32_t* n_free, int32_t* page_table, int32_t* seq_lens, int32_t* cu_new,
                          int64_t* slots, int32_t max_new, int32_t* n_taken, void* stream) {
  if (batch < 0 || max_pages < 0 || free_capacity < 0 || max_new < 0)
    return fail(COSA_ERR_INVALID_ARG, "batch (%d), max_pages (%d), free_capacity (%d) and max_new (%d) must be >= 0", batch,
                max_pages, free_capacity, max_new);
  cosa::PageMapArgs a{};
  cosa_status st = check_page_size(page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if (((int64_t)max_pages << a.log2_page) >= (1ll << 31))
    return fail(COSA_ERR_UNSUPPORTED, "max_pages (%d) * page_size (%d) must stay below 2^31 tokens", max_pages, page_size);
  if (batch > cosa::kMaxRequests)
    return fail(COSA_ERR_UNSUPPORTED, "%d requests (supported: <= %d)", batch, cosa::kMaxRequests);
  const bool some = batch > 0;  // an empty batch still has rows without a request, and takes no page
  if (some && (!cached_lens || !new_lens || !n_free || !seq_lens || !cu_new || !n_taken))
    return fail(COSA_ERR_INVALID_ARG, "cached_lens, new_lens, n_free, seq_lens, cu_new and n_taken must be non-NULL");
  if (some && ((free_capacity > 0 && !free_pages) || (max_pages > 0 && !page_table) || (max_new > 0 && !slots)))
    return fail(COSA_ERR_INVALID_ARG, "free_pages, page_table and slots must be non-NULL where they hold entries");
  if (!some && !cu_new && !n_taken && (max_new == 0 || !slots)) return ok();
  const int64_t n = batch;
  const Span in[] = {{cached_lens, 4 * n}, {new_lens, 4 * n}, {free_pages, some ? 4ll * free_capacity : 0},
                     {n_free, some ? 4 : 0}};
  const Span out[] = {{page_table, 4 * n * max_pages}, {seq_lens, 4 * n}, {cu_new, 4 * (n + 1)}, {slots, 8ll * max_new},
                      {n_taken, 4}};
  for (const Span& o : out)
    for (const Span& i : in)
      if (o.meets(i))
        return fail(COSA_ERR_INVALID_ARG, "page_table, seq_lens, cu_new, slots and n_taken must not overlap the inputs");
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (out[i].meets(out[j])) return fail(COSA_ERR_INVALID_ARG, "the outputs must not overlap each other");
  a.batch = batch;
  a.max_pages = max_pages;
  a.free_capacity = free_capacity;
  a.max_new = slots ? max_new : 0;
  a.cached = cached_lens;
  a.add = new_lens;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.table = page_table;
  a.seq_lens = seq_lens;
  a.cu_new = cu_new;
  a.n_taken = n_taken;
  a.slots = slots;
  return launch(stream, "page_map launch", [&](hipStream_t s) { return cosa::launch_page_map(a, s); });
}

cosa_status cosa_kv_append(int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int64_t n_pages, void* k_cache,
                           void* v_cache, void* bounds, int64_t n_tokens, const void* k, int64_t k_stride,
                           const void* v, int64_t v_stride, const int64_t* slots, void* stream) {
  if (n_kv_heads < 1 || head_dim < 1 || n_tokens < 0)
    return fail(COSA_ERR_INVALID_ARG, "n_kv_heads (%d) and head_dim (%d) must be >= 1, n_tokens (%lld) >= 0", n_kv_heads,
                head_dim, (long long)n_tokens);
  if (head_dim != cosa::kHeadDim) return fail(COSA_ERR_UNSUPPORTED, "head_dim %d (supported: 128)", head_dim);
  cosa::AppendArgs a{};
  cosa_status st = check_page_size(page_size, a.log2_page);
  if (st != COSA_OK) return st;
  if ((st = check_n_pages(n_pages)) != COSA_OK) return st;
  const int64_t dense = (int64_t)n_kv_heads * head_dim;
  for (const int64_t s : {k_stride, v_stride})
    if ((s != 0 && s < dense) || s % 8 != 0)
      return fail(COSA_ERR_INVALID_ARG, "row stride %lld: 0, or a multiple of 8 of at least n_kv_heads * head_dim = %lld",
                  (long long)s, (long long)dense);
  if (n_tokens > (1ll << 29) / n_kv_heads)  // 2^32 threads of a grid, 64 for 16 rows of a head
    return fail(COSA_ERR_UNSUPPORTED, "%lld tokens of %d heads: too large for one launch", (long long)n_tokens, n_kv_heads);
  if (n_tokens == 0) return ok();
  if (!k_cache || !v_cache || !k || !v || !slots)
    return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache, k, v and slots must be non-NULL");
  for (const void* p : {(const void*)k_cache, (const void*)v_cache, (const void*)bounds, k, v})
    if (misaligned(p, 16)) return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache, bounds, k and v must be 16-byte aligned");
  if ((double)n_pages * (double)dense * page_size > 1e18)
    return fail(COSA_ERR_UNSUPPORTED, "caches of %lld pages are too large", (long long)n_pages);
  const int64_t cache = 2ll * n_pages * dense << a.log2_page, rows = n_tokens - 1;
  const Span in[] = {{k, 2 * (rows * (k_stride ? k_stride : dense) + dense)},
                     {v, 2 * (rows * (v_stride ? v_stride : dense) + dense)}, {slots, 8 * n_tokens}};
  const Span out[] = {{k_cache, cache}, {v_cache, cache}, {bounds, 4 * n_pages * dense}};
  for (const Span& o : out)
    for (const Span& i : in)
      if (o.meets(i)) return fail(COSA_ERR_INVALID_ARG, "k, v and slots must not overlap the caches and bounds");
  if (out[0].meets(out[1]) || out[0].meets(out[2]) || out[1].meets(out[2]))
    return fail(COSA_ERR_INVALID_ARG, "k_cache, v_cache and bounds must not overlap each other");
  a.Hkv = n_kv_heads;
  a.n_pages = n_pages;
  a.n_tokens = n_tokens;
  a.k_stride = k_stride ? k_stride : dense;
  a.v_stride = v_stride ? v_stride : dense;
  a.k_cache = static_cast<uint16_t*>(k_cache);
  a.v_cache = static_cast<uint16_t*>(v_cache);
  a.bounds = static_cast<uint16_t*>(bounds);
  a.k = u16(k);
  a.v = u16(v);
  a.slots = slots;
  return launch(stream, "kv_append launch", [&](hipStream_t s) { return cosa::launch_kv_append(a, s); });
}

cosa_status cosa_page_score(const cosa_decode_problem* problem, const void* q, const cosa_paged_kv* kv,
                            const void* bounds, const int32_t* seq_lens, float* score, void* stream) {
  if (!kv) return fail(COSA_ERR_INVALID_ARG, "paged kv is NULL");
  DecodeShape sh{};
  bool empty = false;
  cosa_status st = check_problem(problem, kv->page_size, sh, empty);
  if (st != COSA_OK) return st;
  if ((st = check_kv(kv, false, sh)) != COSA_OK) return st;
  if ((st = check_score_space(sh)) != COSA_OK) return st;
  if (empty || sh.max_pages == 0) return ok();
  if ((st = check_q(q)) != COSA_OK) return st;
  if (!bounds || !seq_lens || !score) return fail(COSA_ERR_INVALID_ARG, "bounds, seq_lens and score must be non-NULL");
  if (misaligned(bounds, 16)) return fail(COSA_ERR_INVALID_ARG, "bounds must be 16-byte aligned");
  return launch(stream, "page_score launch", [&](hipStream_t s) {
    return cosa::launch_page_score(sh, u16(q), u16(bounds), kv->page_table, seq_lens, score, s);
  });
}

cosa_status cosa_page_select(const cosa_decode_problem* problem, int32_t page_size, const int32_t* seq_lens,
                             const float* score, const cosa_page_budget* budget, int32_t* pages, int32_t* count,
                             void* stream) {
  DecodeShape sh{};
  bool empty = false;
  cosa_status st = check_problem(problem, page_size, sh, empty);
  if (st != COSA_OK) return st;
  int64_t micro = 0;
  if ((st = check_budget(budget, micro)) != COSA_OK) return st;
  if ((st = check_select_space(sh)) != COSA_OK) return st;
  if (empty) return ok();
  if (!seq_lens || (sh.max_pages > 0 && !score) || !pages || !count)
    return fail(COSA_ERR_INVALID_ARG, "seq_lens, score, pages and count must be non-NULL");
  const cosa::PageSelectArgs a{sh.B, sh.Hq, sh.Hkv, sh.G, sh.max_pages, sh.log2_page, seq_lens, score, micro,
                               budget->min_pages, budget->max_pages, budget->sink_pages, budget->recent_pages, pages, count};
  return launch(stream, "page_select launch", [&](hipStream_t s) { return cosa::launch_page_select(a, s); });
}

size_t cosa_decode_workspace_bytes(const cosa_decode_problem* problem) {
  DecodeShape sh{};
  bool empty = false;
  if (check_problem(problem, 16, sh, empty) != COSA_OK) return 0;
  return cosa::decode_workspace_bytes(sh);
}

cosa_status cosa_decode_attention(const cosa_decode_problem* problem, const void* q, const cosa_paged_kv* kv,
                                  const int32_t* seq_lens, void* workspace, size_t workspace_bytes, void* o, float* lse,
                                  void* stream) {
  DecodeShape sh{};
  bool empty = false;
  cosa_status st = attention_shape(problem, kv, sh, empty);
  if (st != COSA_OK) return st;
  if ((st = check_tokens(sh, sh.max_pages)) != COSA_OK) return st;
  if (empty) return ok();
  return attention(sh, kv, q, seq_lens, nullptr, nullptr, 0, workspace, workspace_bytes, o, lse, stream);
}

cosa_status cosa_decode_attention_listed(const cosa_decode_problem* problem, const void* q, const cosa_paged_kv* kv,
                                         const int32_t* seq_lens, const int32_t* pages, const int32_t* count,
                                         int32_t list_pages, void* workspace, size_t workspace_bytes, void* o,
                                         float* lse, void* stream) {
  DecodeShape sh{};
  bool empty = false;
  cosa_status st = attention_shape(problem, kv, sh, empty);
  if (st != COSA_OK) return st;
  if (list_pages < 1) return fail(COSA_ERR_INVALID_ARG, "list_pages (%d) must be >= 1", list_pages);
  if ((st = check_tokens(sh, list_pages)) != COSA_OK) return st;
  if (empty) return ok();
  if (!pages || !count) return fail(COSA_ERR_INVALID_ARG, "pages and count must be non-NULL");
  return attention(sh, kv, q, seq_lens, pages, count, list_pages, workspace, workspace_bytes, o, lse, stream);
}

cosa_status cosa_decode_sparse_workspace_layout(const cosa_decode_problem* problem, const cosa_page_budget* budget,
                                                cosa_decode_sparse_layout* layout) {
  DecodeShape sh{};
  bool empty = false;
  int64_t micro = 0;
  cosa_decode_sparse_layout l;
  const cosa_status st = sparse_layout(problem, budget, sh, micro, empty, l);
  if (st != COSA_OK) return st;
  if (!layout) return fail(COSA_ERR_INVALID_ARG, "layout is NULL");
  *layout = l;
  return ok();
}

size_t cosa_decode_sparse_workspace_bytes(const cosa_decode_problem* problem, const cosa_page_budget* budget) {
  cosa_decode_sparse_layout l;
  return cosa_decode_sparse_workspace_layout(problem, budget, &l) == COSA_OK ? l.total : 0;
}

cosa_status cosa_decode_sparse(const cosa_decode_problem* problem, const void* q, const cosa_paged_kv* kv,
                               const void* bounds, const int32_t* seq_lens, const cosa_page_budget* budget,
                               void* workspace, size_t workspace_bytes, void* o, float* lse, void* stream) {
  DecodeShape sh{};
  bool empty = false;
  cosa_status st = attention_shape(problem, kv, sh, empty);
  if (st != COSA_OK) return st;
  DecodeShape any{};
  int64_t micro = 0;
  cosa_decode_sparse_layout l;
  if ((st = sparse_layout(problem, budget, any, micro, empty, l)) != COSA_OK) return st;
  // a list holds no more pages than the table
  if ((st = check_tokens(sh, std::min(budget->max_pages, sh.max_pages))) != COSA_OK) return st;
  if ((st = check_score_space(sh)) != COSA_OK) return st;
  if (empty) return ok();
  if ((st = check_q(q)) != COSA_OK) return st;
  if (!bounds || misaligned(bounds, 16)) return fail(COSA_ERR_INVALID_ARG, "bounds must be non-NULL and 16-byte aligned");
  if ((st = check_o(sh, q, seq_lens, o)) != COSA_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, l.total)) != COSA_OK) return st;
  char* ws = static_cast<char*>(workspace);
  float* score = reinterpret_cast<float*>(ws + l.score);
  int32_t* pages = reinterpret_cast<int32_t*>(ws + l.pages);
  int32_t* count = reinterpret_cast<int32_t*>(ws + l.count);
  const cosa::PageSelectArgs sa{sh.B, sh.Hq, sh.Hkv, sh.G, sh.max_pages, sh.log2_page, seq_lens, score, micro,
                                budget->min_pages, budget->max_pages, budget->sink_pages, budget->recent_pages, pages, count};
  const cosa::DecodeArgs a{u16(q), u16(kv->k_cache), u16(kv->v_cache), kv->page_table, seq_lens, pages, count,
                           budget->max_pages, ws + l.partial, static_cast<uint16_t*>(o), lse};
  return launch(stream, "decode_sparse launch", [&](hipStream_t s) {
    hipError_t e = sh.max_pages > 0 ? cosa::launch_page_score(sh, u16(q), u16(bounds), kv->page_table, seq_lens, score, s)
                                    : hipSuccess;
    if (e == hipSuccess) e = cosa::launch_page_select(sa, s);
    if (e == hipSuccess) e = cosa::launch_decode_attention(sh, a, s);
    return e;
  });
}

}  // extern "C"
