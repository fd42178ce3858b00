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
 * n_rows * n_q_heads below 2^31, and, roughly, 3 * batch * n_rows * n_q_heads * max_pages * page_size below 2^70
 * (COSA_ERR_UNSUPPORTED otherwise). */
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
 * fp32 logits, softmax and sums; probabilities are rounded to bf16 for the product with V, as in the prefill (those of
 * cosa_decode_attention keep 32 bits). What
 * the cache holds behind seq_lens, and behind p for one row, does not matter, NaN and infinities included. An
 * infinite v[t] that is seen gives that infinity in its element: NaN beside one of the other sign or where its logit
 * is -inf (a weight of 0), either of the two where its weight is below 2^-100 of the largest. NaN values and logits that
 * are seen give NaN.
 * The keys are split over a fixed grid and joined in a fixed order: results are deterministic where no row belongs to
 * several sequences.
 * seq_lens is read as clamped to [0, max_pages * page_size], cu_new to [0, n_rows], a sequence that ends in front of
 * its start as empty; rows of several sequences (offsets that fall) hold parts of any of their results, and not the same
 * ones every time. A request that cosa_page_map left
 * out has rows in cu_new but no new tokens: they count as its last cached ones. Table entries outside [0, n_pages) are
 * read as page 0. The workspace is scratch of at least cosa_chunk_workspace_bytes() bytes, 16-byte aligned. o, lse and the
 * workspace overlap neither the inputs, the caches' n_pages pages among them, nor each other.
 */
size_t cosa_chunk_workspace_bytes(const cosa_chunk_problem* problem);
cosa_status cosa_chunk_attention(const cosa_chunk_problem* problem, const void* q,
                                 const cosa_paged_kv* kv, const int32_t* seq_lens,
                                 const int32_t* cu_new, void* workspace, size_t workspace_bytes,
                                 void* o, float* lse, void* stream);

/*
 * Rows of a new table that continue rows of an old one: samples of one prompt, the beams that a search keeps. Row c of
 * n_children continues row parent[c] of page_table [n_parents, max_pages] (a parent outside [0, n_parents): it starts
 * empty) and holds the same pages, but for a last page that is partly filled, which both would write to: the first
 * child of a row goes on with that page itself, every further one takes a page from the front of the free list, in
 * order of c. copy_all != 0: the first child takes one as well (where a row that lives on, here or in another table,
 * holds the parent's last page too). Written:
 *   new_table [n_children, max_pages]: the entries of the pages held; all others stay as they are
 *   new_lens [n_children]   the parent's length, or 0 where the free list has no page left for the child (its entries and
 *                           those behind it in the lists below are not written)
 *   src, dst, rows int32 [n_children]: of the i-th page taken the page whose rows it needs, itself and how many rows
 *                           they are: the lists of cosa_page_copy, once per layer
 *   n_taken [1]             pages taken, the length of these lists (the caller's free list starts there next time)
 * free_pages int32 [free_capacity]; n_free device int32 [1], read as clamped to [0, free_capacity]; lengths as clamped to
 * what a row holds. n_parents and n_children <= 8192. The outputs overlap neither the inputs nor each other.
 */
cosa_status cosa_page_fork(int32_t n_parents, int32_t n_children, int32_t page_size, int32_t max_pages,
                           const int32_t* parent, const int32_t* page_table, const int32_t* seq_lens,
                           int32_t copy_all, const int32_t* free_pages, int32_t free_capacity,
                           const int32_t* n_free, int32_t* new_table, int32_t* new_lens, int32_t* src,
                           int32_t* dst, int32_t* rows, int32_t* n_taken, void* stream);

/*
 * Pages copied within the caches [n_pages, n_kv_heads, page_size, head_dim] and bounds (NULL: not kept; layouts of
 * cosa_kv_append): page src[i] to page dst[i] for i < n_pairs (device int32 [1], read as clamped to [0, max_pairs]). rows (NULL:
 * whole pages): only the first rows[i] tokens of every head (as clamped to [0, page_size]); the bounds as a whole.
 * Pairs with a page outside [0, n_pages) are skipped. All pairs run side by side: no page may be dst twice, or dst of one
 * pair and src of another.
 */
cosa_status cosa_page_copy(int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int64_t n_pages,
                           void* k_cache, void* v_cache, void* bounds, const int32_t* src,
                           const int32_t* dst, const int32_t* rows, int32_t max_pairs,
                           const int32_t* n_pairs, void* stream);

/* Scratch of cosa_page_release and cosa_page_compact over a cache of n_pages pages (0 if that is outside [1, 2^28]). */
size_t cosa_page_workspace_bytes(int64_t n_pages);

/*
 * The free list after a step: pages that some row of old_table [old_batch, max_pages] holds with old_lens and no row
 * of new_table [new_batch, max_pages] with new_lens become free. The tables may be the same one: requests that
 * end have new length 0, drafted tokens that are turned down a smaller one; after a fork they are the two
 * tables. old_lens count the new tokens (cosa_page_map's seq_lens): a page that was taken for tokens which neither
 * length counts would be lost. free_out int32 [out_capacity] gets
 *   the entries n_taken .. n_free - 1 of free_pages [free_capacity] (n_taken: what cosa_page_map or cosa_page_fork took
 *   from its front, device int32 [1], NULL for 0, read as clamped to [0, n_free]), then
 *   the pages that become free, in ascending order, but for those that are among these entries already;
 * n_free_out [1] their number. What does not fit out_capacity is left out; entries behind stay as they are. Lengths and
 * table entries are read as in cosa_page_fork, entries outside [0, n_pages) are no pages. n_free_out may be n_free;
 * otherwise the outputs and the workspace overlap neither the inputs nor each other. n_pages and free_capacity <= 2^28,
 * rows below 2^24, rows * max_pages below 2^31.
 */
cosa_status cosa_page_release(int32_t page_size, int32_t max_pages, int64_t n_pages, int32_t old_batch,
                              const int32_t* old_table, const int32_t* old_lens, int32_t new_batch,
                              const int32_t* new_table, const int32_t* new_lens,
                              const int32_t* free_pages, int32_t free_capacity, const int32_t* n_free,
                              const int32_t* n_taken, int32_t* free_out, int32_t out_capacity,
                              int32_t* n_free_out, void* workspace, size_t workspace_bytes,
                              void* stream);

/*
 * Pages to the lowest numbers: the highest page in use (held by some row of page_table [batch, max_pages] with
 * seq_lens) moves to the lowest unused one, the next highest to the next lowest, and so on while the page moved to is
 * the lower one, at most max_moves times (more calls go on with it). Written:
 *   new_table [batch, max_pages] (may be page_table itself): the table with the pages' new numbers, entries behind a
 *                       row's last page and outside [0, n_pages) as they are
 *   src, dst int32 [max_moves], n_moves [1]: the moves, for cosa_page_copy once per layer before the pages are used again
 *   free_pages int32 [free_capacity], n_free [1]: all pages that are unused then, in ascending order (what does not fit
 *                       is left out)
 * Every row that holds pages of the cache has to be in the table. The outputs and the workspace overlap neither the
 * inputs, but for new_table, nor each other. Limits as in cosa_page_release.
 */
cosa_status cosa_page_compact(int32_t batch, int32_t page_size, int32_t max_pages, int64_t n_pages,
                              const int32_t* page_table, const int32_t* seq_lens, int32_t max_moves,
                              int32_t* new_table, int32_t* src, int32_t* dst, int32_t* n_moves,
                              int32_t* free_pages, int32_t free_capacity, int32_t* n_free,
                              void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* COSA_SERVING_H_ */
