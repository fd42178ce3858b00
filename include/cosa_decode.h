/*
 * cosa_decode.h — C ABI of the decode-side operators of the CoSA library for AMD Instinct MI355X
 * (gfx950): filling a paged KV cache and attending to it with one new token per sequence.
 *
 * After a prompt's prefill (cosa_prefill_paged reads the same cache), one decode step is
 *   1. cosa_page_map          once per step: pages for the new tokens, block table, slot map;
 *   2. cosa_kv_append         per layer: the step's K and V rows into their slots, and the bounds of
 *                             the keys of the pages they touch;
 *   3. cosa_decode_attention  per layer: the new token of every sequence over its whole context, or
 *      cosa_decode_sparse     the same over the pages that a cheap score selects (cosa_page_score,
 *                             cosa_page_select and cosa_decode_attention_listed in one call).
 * Prompts enter the cache the same way: steps 1 and 2 with as many new tokens as a request has.
 *
 * The conventions of cosa.h hold: device pointers owned by the caller, bf16 as raw 16-bit storage,
 * work enqueued on `stream` without synchronising or allocating, host validation before anything is
 * enqueued, no state kept between calls. In addition:
 *   - Kernels run on the device of `stream` (the current device for the null stream), whichever
 *     device is current.
 *   - Lengths, tables, lists and slots are device data that the host does not see, so that a step
 *     can be captured into a graph and replayed with others. What they may hold is bounded on the
 *     device as each entry point says; nothing outside the given buffers is read or written.
 *   - Calls that may run at the same time need distinct workspaces and outputs. Outputs must not overlap
 *     inputs (o and q, and the arrays of cosa_page_map and cosa_kv_append, are checked).
 *   - bf16 pointers (q, k, v, caches, bounds, o) and workspaces are 16-byte aligned; row strides are
 *     multiples of 8 elements.
 *
 * Supported problem space (COSA_ERR_UNSUPPORTED otherwise): head_dim == 128, page_size a power of two
 * in [16, 2^20], max_pages * page_size < 2^31, and what one launch holds. With U = batch * n_kv_heads * ceil(G / 16)
 * for G query heads per KV head: U < 2^22 in every call with a problem, U * (tiles of 128 tokens in a table row or list + 1) < 2^31
 * in attention, U * ceil(max_pages / 16) < 2^26 in page scores, n_tokens * n_kv_heads <= 2^29 in an append.
 */
#ifndef COSA_DECODE_H_
#define COSA_DECODE_H_

#include "cosa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One new token for each sequence of a batch. The paged cache is a cosa_paged_kv, with page_table
 * [batch, max_pages]: entry [n, j] is the physical page of tokens j * page_size .. of sequence n. Entries
 * behind a sequence's last page are not used; an entry outside [0, n_pages) is read as page 0. */
typedef struct {
  int32_t batch;      /* B >= 0                                                                   */
  int32_t n_q_heads;  /* Hq, a multiple of n_kv_heads; query head h reads KV head h / (Hq / Hkv)   */
  int32_t n_kv_heads; /* Hkv >= 1                                                                 */
  int32_t head_dim;   /* d                                                                        */
  int32_t max_pages;  /* width of the page table >= 0: pages a sequence can hold                   */
  int64_t q_stride;   /* elements between the queries of consecutive sequences, 0: Hq * d (dense)  */
  float sm_scale;     /* logit scale; 0 selects 1/sqrt(head_dim)                                  */
} cosa_decode_problem;

/* Pages that cosa_page_select keeps of a sequence that holds p of them:
 *   K = min(p, max(sink_pages + recent_pages, min(max_pages, max(min_pages, ceil(fraction * p))))). */
typedef struct {
  float fraction;       /* share of the sequence's pages, in (0, 1], taken at 1e-6 resolution       */
  int32_t min_pages;    /* 1 <= min_pages <= max_pages                                            */
  int32_t max_pages;    /* width of a list; sink_pages + recent_pages <= max_pages                 */
  int32_t sink_pages;   /* leading pages that are always kept, >= 0                               */
  int32_t recent_pages; /* trailing pages that are always kept, >= 0                              */
} cosa_page_budget;

/*
 * Block tables and slot maps from request lengths. Request r holds cached_lens[r] tokens in the pages
 * of its table row and adds new_lens[r]; pages it lacks are taken from the front of the free list, in
 * request order and, within a request, in token order. Written:
 *   page_table [batch, max_pages]: the entries of the pages taken; all others stay as they are
 *   seq_lens [batch]     cached + new tokens
 *   cu_new [batch + 1]   prefix sums of new_lens: request r's new tokens are rows cu_new[r] ..
 *                        cu_new[r + 1] - 1 of the step's packed token rows (saturating at 2^31 - 1)
 *   slots int64 [max_new] slot (page * page_size + token within the page) of every packed row; -1 for
 *                        rows behind the last request's
 *   n_taken [1]          free pages taken (the caller's free list starts there next time)
 * free_pages int32 [free_capacity]; n_free: how many of them are there, device int32 [1], read as clamped
 * to [0, free_capacity]. A request does not fit when cached + new exceeds max_pages * page_size, when its rows
 * end behind max_new, or when the pages needed by it and by the requests before it (of those that fit
 * the first two) exceed n_free and it needs one. Such a request adds nothing: its seq_lens is cached_lens, its
 * slots are -1, it takes no page. Negative lengths are read as 0, cached lengths above the row's capacity as that
 * capacity. The old part of a row is read only for the page that is partly filled; a negative entry
 * there gives slots of -1. batch <= 8192. An empty batch writes cu_new[0] = 0, n_taken = 0 and slots of -1, each
 * of them unless it is NULL; its other arrays are not used.
 */
cosa_status cosa_page_map(int32_t batch, int32_t page_size, int32_t max_pages,
                          const int32_t* cached_lens, const int32_t* new_lens,
                          const int32_t* free_pages, int32_t free_capacity, const int32_t* n_free,
                          int32_t* page_table, int32_t* seq_lens, int32_t* cu_new, int64_t* slots,
                          int32_t max_new, int32_t* n_taken, void* stream);

/*
 * K and V rows of n_tokens new tokens into the caches [n_pages, n_kv_heads, page_size, head_dim]: row t of
 * k and v ([n_tokens, n_kv_heads, head_dim], k_stride and v_stride elements between tokens, 0: dense) goes
 * to slot slots[t] (page slots[t] / page_size). Slots outside [0, n_pages * page_size) are skipped.
 * Every slot may occur once in a call.
 * bounds (NULL: not kept): bf16 [n_pages, n_kv_heads, 2, head_dim], the elementwise minimum [0] and maximum [1] of the
 * keys in a page. A page that receives its token 0 starts anew; a page that receives later tokens keeps
 * the smaller minimum and larger maximum of what its bounds hold and the new keys. With bounds the new
 * tokens of one page must be consecutive in slots, in ascending order, as cosa_page_map lays them out
 * (the cache rows are right in any order; the page's bounds then are those of some of its runs).
 * A NaN key makes one of the two bounds NaN in that element, the maximum for a positive sign bit.
 */
cosa_status cosa_kv_append(int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int64_t n_pages,
                           void* k_cache, void* v_cache, void* bounds, int64_t n_tokens,
                           const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                           const int64_t* slots, void* stream);

/*
 * Upper bound on the logits of every page (the cheap score of cosa_page_select):
 *   score[n, h, j] = sm_scale * sum_d max(q[n, h, d] * min[d], q[n, h, d] * max[d])
 * with min, max the bounds of page page_table[n, j] and KV head h / (Hq / Hkv): but for rounding, no key of
 * the page has a larger logit. score is fp32 [batch, n_q_heads, max_pages]; entries of pages that sequence n does not hold
 * (j >= ceil(seq_lens[n] / page_size)) are not written. seq_lens is read as clamped to [0, max_pages * page_size]
 * (here and below). Only page_table, page_size and n_pages of kv are used. A page with an infinite or NaN
 * bound scores NaN or infinity. fp32 sums in a fixed order.
 */
cosa_status cosa_page_score(const cosa_decode_problem* problem, const void* q,
                            const cosa_paged_kv* kv, const void* bounds, const int32_t* seq_lens,
                            float* score, void* stream);

/*
 * The pages that every KV head keeps. With g the query heads of KV head h and p the sequence's pages,
 *   s[j] = max over g of (score[n, g, j] - max over j' < p of score[n, g, j']),
 * so that a page holding some head's row maximum has s = 0 and comes before all others. The sink and
 * recent pages are kept, then the pages of largest s, ties by ascending j, up to K (cosa_page_budget).
 * pages int32 [batch, n_kv_heads, budget->max_pages]: the kept pages in ascending order, then -1;
 * count int32 [batch, n_kv_heads] = K (0 for an empty sequence). A NaN difference counts as the largest; the
 * row maximum passes over NaN scores. max_pages <= 32768, at most 1024 query heads per KV head.
 */
cosa_status cosa_page_select(const cosa_decode_problem* problem, int32_t page_size,
                             const int32_t* seq_lens, const float* score,
                             const cosa_page_budget* budget, int32_t* pages, int32_t* count,
                             void* stream);

/*
 * Attention of one token per sequence: o[n, h] = softmax over the tokens t < seq_lens[n] of
 * (sm_scale * <q[n, h], k[t]>) applied to v[t]. q [batch, Hq, d] (q_stride between sequences), o
 * [batch, Hq, d] dense, bf16; lse (NULL to omit) fp32 [batch, Hq]: the natural logarithm of the softmax's sum of
 * exponentials. fp32 arithmetic; probabilities enter the product with V as three bf16 terms (all 24 bits). An
 * empty sequence, or one whose logits are all -inf, gives o = 0 and lse = -inf. An infinite v[t] gives that infinity in its
 * element (NaN beside one of the other sign, or where its weight is 0 or below 2^-100 of the largest); NaN values and
 * logits give NaN. What the cache holds behind seq_lens does not matter (NaN included). The tokens are split over a
 * fixed grid and joined in a fixed order: results are deterministic. The workspace is scratch of at least
 * cosa_decode_workspace_bytes() bytes.
 */
size_t cosa_decode_workspace_bytes(const cosa_decode_problem* problem);
cosa_status cosa_decode_attention(const cosa_decode_problem* problem, const void* q,
                                  const cosa_paged_kv* kv, const int32_t* seq_lens, void* workspace,
                                  size_t workspace_bytes, void* o, float* lse, void* stream);

/*
 * cosa_decode_attention over listed pages: KV head g of sequence n attends to the tokens t < seq_lens[n] of
 * the logical pages pages[n, g, 0 .. count[n, g] - 1], in any order (int32 [batch, Hkv, list_pages]; count
 * is read as clamped to [0, list_pages]). Entries outside [0, max_pages) or behind the sequence's end
 * add nothing; a page listed twice counts twice. On the list of all pages the result equals
 * cosa_decode_attention up to the order of its sums. list_pages * page_size < 2^31.
 */
cosa_status cosa_decode_attention_listed(const cosa_decode_problem* problem, const void* q,
                                         const cosa_paged_kv* kv, const int32_t* seq_lens,
                                         const int32_t* pages, const int32_t* count,
                                         int32_t list_pages, void* workspace,
                                         size_t workspace_bytes, void* o, float* lse, void* stream);

/* Byte offsets inside a cosa_decode_sparse workspace (each 256-byte aligned). */
typedef struct {
  size_t score;   /* float   [B, Hq, max_pages]                        */
  size_t pages;   /* int32_t [B, Hkv, budget.max_pages]                */
  size_t count;   /* int32_t [B, Hkv]                                  */
  size_t partial; /* cosa_decode_workspace_bytes() of scratch          */
  size_t total;   /* bytes required                                    */
} cosa_decode_sparse_layout;

cosa_status cosa_decode_sparse_workspace_layout(const cosa_decode_problem* problem,
                                                const cosa_page_budget* budget,
                                                cosa_decode_sparse_layout* layout);
/* layout.total (0 if the arguments are invalid; see cosa_last_error()). */
size_t cosa_decode_sparse_workspace_bytes(const cosa_decode_problem* problem,
                                          const cosa_page_budget* budget);

/*
 * cosa_page_score, cosa_page_select and cosa_decode_attention_listed back to back on one stream,
 * bit-identical to those calls; their results stay in the workspace at the layout's offsets. A budget above the
 * table's max_pages keeps at most those, so min(budget->max_pages, max_pages) * page_size < 2^31 is enough.
 */
cosa_status cosa_decode_sparse(const cosa_decode_problem* problem, const void* q,
                               const cosa_paged_kv* kv, const void* bounds,
                               const int32_t* seq_lens, const cosa_page_budget* budget,
                               void* workspace, size_t workspace_bytes, void* o, float* lse,
                               void* stream);

#ifdef __cplusplus
}
#endif

#endif /* COSA_DECODE_H_ */
