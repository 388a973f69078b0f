// Arguments and launchers of the attention kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/opattr_attn.h"

namespace opa {

// A [tokens, heads, head_dim] tensor of 16-bit values; strides in elements.
struct Rows {
  uint16_t *p;
  int64_t ts, hs;
};

struct PromptArgs {
  Rows q, k, v, out;
  float *lse;  // [heads][n_q]
  const int32_t *cu_q, *cu_k;
  int n_q, n_k, n_seqs, n_heads, n_kv, group, head_dim, causal;
  float scale;
  int window, sinks;  // window 0: none
  int head_shift;     // a window's: log2 of the query heads that a block takes
  opattr_diag *diag;
  Rows dout, dq, dk, dv;
  // the gradient's workspace: pairs (lse in binary digits, D)
  // [heads][n_q]; largest norms [n_heads + n_kv][norm_slots] (float16); the splits' dk and dv
  float *rows, *part;
  uint32_t *norms;
  int norm_slots;
  int splits, split_steps;
  // key tiles of a sequence with sinks; where blocks share them, the log2 of a block's
  // steps and how many share one at most; such blocks and tiles of the call at most
  int sink_tiles, sink_shift, sink_most, sink_slots, sink_sums;
};

// Query heads of a key head that a block takes, as a power of two: a block passes over
// the keys that any of its rows sees, window + rows - 1 of them, so that fewer rows of
// more heads waste fewer (24 prompts of up to 4099 tokens, 32 heads on 8 of 128, window
// 512: 194 us by 128 rows of one head, 159 by 32 of four).
inline int window_heads(int group) { return group % 4 == 0 ? 2 : group % 2 == 0 ? 1 : 0; }

// Blocks that share a key tile of the gradient at most, and the steps of 32 queries
// that each is to have, or fewer; through a window, what PromptArgs has of the sinks'.
struct GradSplits {
  int most, steps, sink_tiles, sink_shift, sink_most, sink_slots, sink_sums;
};
GradSplits grad_splits(int64_t n_q, int64_t n_k, int n_seqs, int n_heads, int n_kv, int window,
                       int sinks);
// Pieces of rows whose largest norms a gradient in float16 looks up, of a head.
int64_t norm_slots(int64_t n_q, int64_t n_k, int n_seqs);
// Key tiles' parts that the blocks leave for the sums: of 128 keys of a key head, at most.
int64_t grad_parts(const GradSplits &x, int64_t n_k, int n_seqs);

struct PagedArgs {
  const uint16_t *k, *v;
  int64_t ps, ts, hs;  // page, token and head strides in elements
  int n_pages, shift, slots;  // log2 of the page size; tokens the table can name
  const int32_t *table;
  int n_seqs, width, n_kv, group, n_heads, head_dim;
  Rows q, out;
  const int32_t *lens;
  float scale;
  float *lse;
  float *part;  // partial results
  opattr_diag *diag;
  int window, sinks;  // window 0: none
  int most;           // tokens of a sequence that its query can see
  int32_t *shares;    // [n_seqs][2] behind the partial results, for their join
};

// The cache of 8 bits; strides (those of PagedArgs too) in bytes.
struct ScaledArgs : PagedArgs {
  const uint8_t *k_codes, *v_codes, *k_scale, *v_scale;
  int64_t sps, sbs, shs;  // the scales' page, block and head strides
  // (most: places, as they are counted through by runs of 16)
  int block_shift;        // log2 of the tokens with one scale
};

struct AppendScaledArgs {
  uint8_t *k, *v, *k_scale, *v_scale;
  int64_t ps, ts, hs, sps, sbs, shs;
  int n_pages, shift, slots, block_shift;
  const int32_t *table;
  int n_seqs, width, n_kv, head_dim, n_new;
  const int32_t *cu, *lens;
  Rows kn, vn;
  int32_t *lens_out;
  opattr_diag *diag;
};

struct AppendArgs {
  uint16_t *k, *v;
  int64_t ps, ts, hs;
  int n_pages, shift, slots;
  const int32_t *table;
  int n_seqs, width, n_kv, head_dim, n_new;
  const int32_t *cu, *lens;
  Rows kn, vn;
  int32_t *lens_out;
  opattr_diag *diag;
};

struct PagesArgs {
  char *data;
  int64_t plane, page;  // strides in bytes
  int n_planes, n_pages, bytes, size;  // size: tokens a page
  const int32_t *held;
  const int32_t *table, *lens, *parent, *room;
  int n_rows, width, n_out;
  int32_t *table_out, *lens_out, *refs, *moved, *live;
  opattr_diag *diag;
  // workspace: a bit a page, the set bits before each word, each row's requests
  uint32_t *words;
  int32_t *sums, *row_at;
  int give, copy_planes;  // blocks that write tables; blocks a row that copy
};

void run_paged(const PagedArgs &a, int dtype, hipStream_t s);
// Bytes of the partial results; the sequences' shares come behind them.
size_t paged_parts(int n_seqs, int n_kv, int n_heads, int most);
size_t scaled_parts(int n_seqs, int n_kv, int n_heads, int most);
void run_paged_scaled(const ScaledArgs &a, int dtype, hipStream_t s);
void run_append_scaled(const AppendScaledArgs &a, int dtype, hipStream_t s);
// blocks of tokens that n_new new ones of n_seqs sequences touch, at most
int64_t append_units(int64_t n_new, int n_seqs, int block_shift);
void run_append(const AppendArgs &a, hipStream_t s);
void run_fork(const PagesArgs &a, hipStream_t s);
void run_compact(const PagesArgs &a, hipStream_t s);
void run_check(const PromptArgs &a, hipStream_t s);
void run_prompt(const PromptArgs &a, int dtype, hipStream_t s);
void run_prompt_grad(const PromptArgs &a, int dtype, hipStream_t s);

}  // namespace opa
