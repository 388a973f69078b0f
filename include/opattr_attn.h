/*
 * opattr_attn.h -- attention operators of the profiled workload, and the paged
 * key-value cache that serves them.
 *
 *   opattr_attn_prompt       attention over whole prompts: packed sequences,
 *                            causal or not, grouped heads
 *   opattr_attn_prompt_grad  its gradient
 *   opattr_attn_paged        attention of one new token a sequence over a paged
 *                            cache, split over the cache's length and joined
 *   opattr_kv_append         new tokens' keys and values into their pages
 *   opattr_pages_fork        the next page table from the present one: sequences
 *                            dropped, continued, forked, and given room
 *   opattr_pages_compact     the pages in use moved to the front of the pool
 *
 * The conventions of opattr.h hold: device pointers unless marked (host); work
 * enqueued on `stream` without synchronising; the caller owns every buffer and
 * the library allocates none; 0 or a negative OPATTR_ERR_* for argument errors,
 * found before anything is enqueued; errors that depend on the data go to the
 * opattr_diag record. Here diag may be NULL (they are then not reported); it is
 * cleared by opattr_diag_clear and read by opattr_read_diag, and a call adds to
 * bad_records and sets flags and status.
 *
 * Element types: OPATTR_BF16 and OPATTR_F16 for queries, keys, values, outputs
 * and gradients; sums, the softmax statistics and the gradients' accumulators
 * are float32. head_dim is a multiple of 8, at most 128.
 *
 * Rows: an opattr_rows names a [tokens, heads, head_dim] tensor by its first
 * element and its strides in ELEMENTS; a head's head_dim values lie side by
 * side. Pointers are 16-byte aligned, strides multiples of 8, the token stride
 * in [head_dim, 2^22], the head stride in [0, 2^40]: a slice of a packed
 * projection, or [heads, tokens, head_dim], is passed as it is. Outputs must
 * not overlap inputs or each other; outputs, caches that are appended to, and pools of
 * pages that have one place for two of their own rows or pages are refused.
 *
 * A query that sees no key (an empty sequence, or a causal mask that hides all
 * of them) has output 0, row statistic -inf, and gives and takes no gradient.
 * What a query does not see takes no part in its output, whatever its bits: rows
 * beside a sequence, tokens past a length, keys and values that the causal mask
 * hides, NaN and infinities among them. The gradient is defined for finite
 * inputs: in a sequence that holds others, also rows that do not see them may
 * become NaN. bfloat16 values of up to 2^136 over the number of keys keep the sum
 * before its division by the weights' in float32's range.
 *
 * float16 gradients: ds is rounded after a power of two by the largest |dout| and |v|
 * of its sequence and head, so neither another sequence nor, for dq, another query
 * head costs it bits.
 */
#ifndef OPATTR_ATTN_H
#define OPATTR_ATTN_H

#include "opattr.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { OPATTR_BF16 = 0, OPATTR_F16 = 1 };

typedef struct {
  void *p;
  int64_t token_stride, head_stride; /* elements */
} opattr_rows;

/* Packed sequences: sequence b has queries cu_q[b] .. cu_q[b+1]) of the n_q
   query rows and keys cu_k[b] .. cu_k[b+1]) of the n_k key rows (n_seqs + 1
   non-decreasing offsets each). Values outside [0, n], and decreasing ones, are
   clamped and flagged DATA. Rows outside every sequence are not written.
   Query head h reads key head h / (n_heads / n_kv_heads). With causal, query i
   of a sequence sees key j when j <= i + (keys - queries): the last query sees
   every key. scale multiplies q.k. (max(n_q, n_k) / 128 + n_seqs) n_heads is
   below 2^24. */
typedef struct {
  int64_t n_q, n_k;
  const int32_t *cu_q, *cu_k;
  int32_t n_seqs;
  int32_t n_heads, n_kv_heads, head_dim;
  int32_t dtype;  /* OPATTR_BF16 | OPATTR_F16 */
  int32_t causal; /* 0 | 1 */
  float scale;
} opattr_attn_shape;

/* out[i] = sum_j softmax_j(scale q_i.k_j) v_j over the keys that query i sees.
   lse (or NULL) receives [n_heads][n_q] float32, the natural logarithm of
   sum_j exp(scale q_i.k_j), which the gradient reads. */
int opattr_attn_prompt(const opattr_attn_shape *a, const opattr_rows *q, const opattr_rows *k,
                       const opattr_rows *v, const opattr_rows *out, float *lse,
                       opattr_diag *diag, void *stream);

/* Gradients of sum(out * dout): with p_ij = exp(scale q_i.k_j - lse_i) and
   D_i = dout_i.out_i,
     dv_j = sum_i p_ij dout_i,   ds_ij = scale p_ij (dout_i.v_j - D_i),
     dq_i = sum_j ds_ij k_j,     dk_j = sum_i ds_ij q_i,
   key heads summing over the query heads that read them. The same bits on
   every run. out and lse are opattr_attn_prompt's for the same inputs. */
size_t opattr_attn_prompt_grad_workspace_bytes(const opattr_attn_shape *a);
int opattr_attn_prompt_grad(const opattr_attn_shape *a, const opattr_rows *dout,
                            const opattr_rows *q, const opattr_rows *k, const opattr_rows *v,
                            const opattr_rows *out, const float *lse, const opattr_rows *dq,
                            const opattr_rows *dk, const opattr_rows *dv, opattr_diag *diag,
                            void *ws, size_t ws_bytes, void *stream);

/* One layer's paged cache: key (value) head g of token t of page x is at
   k (v) + x page_stride + t token_stride + g head_stride (elements, the same
   for both; 16-byte aligned, multiples of 8). page_size is a power of two
   in [1, 1024], a table names fewer than 2^30 tokens; token n of sequence b is on
   page table[b * table_stride + n / page_size], slot n % page_size. */
typedef struct {
  void *k, *v;
  int64_t page_stride, token_stride, head_stride;
  int32_t n_pages, page_size;
  const int32_t *table; /* [n_seqs][table_stride] */
  int32_t n_seqs, table_stride;
  int32_t n_kv_heads, head_dim;
  int32_t dtype;
} opattr_kv_pages;

/* One query token a sequence: out[b] over the first lens[b] tokens of sequence
   b. q and out have n_seqs rows of n_heads heads (n_heads / n_kv_heads at most
   16, n_seqs n_heads below 2^23); lse (or NULL) receives [n_heads][n_seqs]. lens[b] is clamped to what the
   table can name; tokens on a page outside [0, n_pages) are masked; both are
   flagged DATA. Partial results of a sequence's shares are joined in their
   order: the same bits on every run. */
size_t opattr_attn_paged_workspace_bytes(const opattr_kv_pages *c, int32_t n_heads);
int opattr_attn_paged(const opattr_kv_pages *c, int32_t n_heads, const opattr_rows *q,
                      const int32_t *lens, float scale, const opattr_rows *out, float *lse,
                      opattr_diag *diag, void *ws, size_t ws_bytes, void *stream);

/* Rows cu[b] .. cu[b+1]) of k_new and v_new (n_new rows, fewer than 2^26 - 4) become tokens lens[b],
   lens[b] + 1, ... of sequence b. lens_out (or NULL; not lens itself) receives
   lens[b] + (cu[b+1] - cu[b]). Tokens past the table's width or on a page
   outside [0, n_pages) are not written and flagged DATA; no two tokens may
   have the same place. */
int opattr_kv_append(const opattr_kv_pages *c, int64_t n_new, const int32_t *cu,
                     const opattr_rows *k_new, const opattr_rows *v_new, const int32_t *lens,
                     int32_t *lens_out, opattr_diag *diag, void *stream);

/* A pool of pages: n_planes arrays (keys and values of each layer) of n_pages
   pages that share one page table. Page x of plane l is the page_bytes bytes
   (a multiple of 16) at data + l plane_stride + x page_stride (BYTES, multiples
   of 16); page_size tokens lie on a page. held (or NULL) [n_pages] counts the
   references to each page from outside the table. */
typedef struct {
  void *data;
  int64_t plane_stride, page_stride;
  int32_t n_planes, n_pages;
  int32_t page_bytes, page_size;
  const int32_t *held;
} opattr_page_pool;

/* The next page table. Row i of table_out continues row parent[i] of table
   (-1: a new, empty row), with n = lens[parent[i]] tokens (lens_out[i]):
     - its full pages are the parent's, shared;
     - a last page filled in part stays with the lowest row of that parent and
       is copied, in every plane, to a new page for each other one;
     - it gets new pages up to ceil(max(room[i], n) / page_size) (room NULL: n);
     - the remaining entries are -1.
   Rows that no row continues are dropped. New pages are those that no kept
   entry and no held count refers to, lowest first, given to the rows in order.
   refs (or NULL) [n_pages] receives the references from table_out and held.
   When the free pages run out the remaining entries are -1, LIMIT is flagged,
   and a row whose copy got no page ends at its full pages. A parent out of
   range reads as -1, a kept entry out of range becomes -1, a length or room
   past what the table can name is cut; all flagged DATA. table and table_out are
   [rows][width]; they, lens, lens_out, refs and held do not overlap. */
size_t opattr_pages_fork_workspace_bytes(int32_t n_rows, int32_t n_out, int32_t width,
                                         int32_t n_pages);
int opattr_pages_fork(const opattr_page_pool *p, const int32_t *table, const int32_t *lens,
                      int32_t n_rows, int32_t width, const int32_t *parent, const int32_t *room,
                      int32_t n_out, int32_t *table_out, int32_t *lens_out, int32_t *refs,
                      opattr_diag *diag, void *ws, size_t ws_bytes, void *stream);

/* Moves the pages in use (those that an entry of table or a held count refers
   to; m of them) to places 0 .. m-1: pages already below m stay, and the others,
   in order, take the free places below m in order. table_out[i] = the new place
   of table[i]'s page (-1 stays; an entry out of range becomes -1, flagged DATA);
   moved[n_pages] the new place of each page, -1 for free ones; live (or NULL)
   receives m. table_out may be table itself; moved does not overlap held. */
size_t opattr_pages_compact_workspace_bytes(int32_t n_pages);
int opattr_pages_compact(const opattr_page_pool *p, const int32_t *table, int32_t n_rows,
                         int32_t width, int32_t *table_out, int32_t *moved, int32_t *live,
                         opattr_diag *diag, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
