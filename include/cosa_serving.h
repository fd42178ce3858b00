/*
 * cosa_serving.h — C ABI of the operators that a serving loop needs beside a decode step, on AMD Instinct
 * MI355X (gfx950): attention of chunks of new tokens over a paged KV cache, and the cache's pages (forked,
 * copied, given back, compacted).
 *
 * cosa_page_map and cosa_kv_append (cosa_decode.h) put any number of new tokens of every request into the cache;
 * cosa_chunk_attention then attends to them and to everything in front of them: a prompt in chunks, a prompt
 * behind a prefix that is cached already, drafted tokens to be verified, or a step that mixes these with
 * sequences that add one token. Its problem, table and lengths are those of a decode step, its cu_new is
 * cosa_page_map's.
 *
 * A page is in use while a row of a block table holds it below the row's length. There are no reference counts: the
 * tables say who holds a page, so rows may share pages in any way, and
 *   cosa_page_fork     makes the rows of a new table from rows of an old one (samples of one prompt, beams);
 *   cosa_page_copy     then copies, per layer, the partly filled pages that several of them would write to;
 *   cosa_page_release  gives the pages back that the old table held and the new one does not;
 *   cosa_page_compact  moves pages to the lowest numbers, so that the end of the cache becomes free.
 *
 * The conventions of cosa.h and cosa_decode.h hold: device pointers owned by the caller, bf16 as raw 16-bit
 * storage, work enqueued on `stream` (and on its device) without synchronising or allocating, host validation before
 * anything is enqueued, no state kept between calls; lengths, tables and lists are device data that are bounded on the device;
 * calls that may run at the same time need distinct workspaces and outputs.
 */
#ifndef COSA_SERVING_H_
#define COSA_SERVING_H_

#include "cosa_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* New tokens of a batch of sequences, packed one sequence behind the other. Limits as in cosa_decode.h: head_dim == 128,
 * page_size a power of two in [16, 2^20], max_pages * page_size < 2^31; batch and n_rows below 2^22,
 * n_rows * n_q_heads below 2^31 (COSA_ERR_UNSUPPORTED otherwise). */
typedef struct {
  int32_t batch;      /* B >= 0                                                                   */
  int32_t n_q_heads;  /* Hq, a multiple of n_kv_heads; query head h reads KV head h / (Hq / Hkv)   */
  int32_t n_kv_heads; /* Hkv >= 1                                                                 */
  int32_t head_dim;   /* d                                                                        */
  int32_t max_pages;  /* width of the page table >= 0: pages a sequence can hold                   */
  int32_t n_rows;     /* rows of q and o >= 0                                                     */
  int64_t q_stride;   /* elements between the queries of consecutive rows, 0: Hq * d (dense)       */
  float sm_scale;     /* logit scale; 0 selects 1/sqrt(head_dim)                                  */
} cosa_chunk_problem;

/*
 * Attention of new tokens: sequence n has seq_lens[n] tokens in its pages (the new ones among them), and the rows
 * cu_new[n] .. cu_new[n + 1] - 1 of q are its last w = cu_new[n + 1] - cu_new[n] tokens, in order. Row i of them
 * stands at token p = seq_lens[n] - w + i and attends to the tokens t <= p:
 *   o[row, h] = softmax over t <= p of (sm_scale * <q[row, h], k[t]>) applied to v[t].
 * q [n_rows, Hq, d] (q_stride between rows), o [n_rows, Hq, d] dense, bf16; lse (NULL to omit) fp32 [n_rows, Hq]: the
 * natural logarithm of the softmax's sum of exponentials. A row with p < 0 sees nothing: o = 0 and lse = -inf, as
 * where all its logits are -inf. Rows of no sequence are not written.
 * fp32 logits, softmax and sums; probabilities are rounded to bf16 for the product with V, as in the prefill. What
 * the cache holds behind seq_lens, and behind p for one row, does not matter, NaN and infinities included. An
 * infinite v[t] that is seen gives that infinity in its element (NaN beside one of the other sign, or where its
 * weight is 0 or below 2^-100 of the largest); NaN values and logits that are seen give NaN.
 * The keys are split over a fixed grid and joined in a fixed order: results are deterministic.
 * seq_lens is read as clamped to [0, max_pages * page_size], cu_new to [0, n_rows], a sequence that ends in front of
 * its start as empty; sequences whose rows overlap leave one of their results in them. A request that cosa_page_map left
 * out has rows in cu_new but no new tokens: they count as its last cached ones. Table entries outside [0, n_pages) are
 * read as page 0. The workspace is scratch of at least cosa_chunk_workspace_bytes() bytes, 16-byte aligned.
 */
size_t cosa_chunk_workspace_bytes(const cosa_chunk_problem* problem);
cosa_status cosa_chunk_attention(const cosa_chunk_problem* problem, const void* q,
                                 const cosa_paged_kv* kv, const int32_t* seq_lens,
                                 const int32_t* cu_new, void* workspace, size_t workspace_bytes,
                                 void* o, float* lse, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* COSA_SERVING_H_ */
