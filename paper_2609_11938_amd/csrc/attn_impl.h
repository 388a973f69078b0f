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
  Rows q, k, v, out, dout, dq, dk, dv;
  float *lse;  // [heads][n_q]
  const int32_t *cu_q, *cu_k;
  int n_q, n_k, n_seqs, n_heads, n_kv, group, head_dim, causal;
  float scale;
  opattr_diag *diag;
  // the gradient's workspace: pairs (lse in binary digits, D)
  // [heads][n_q]; bounds [n_seqs][n_heads + n_kv] (float16); the splits' dk and dv
  float *rows, *part;
  uint32_t *norms;
  int splits, split_steps;
};

// Blocks that share a key tile of the gradient at most, and the steps of 32 queries
// that each is to have, or fewer.
struct GradSplits {
  int most, steps;
};
GradSplits grad_splits(int64_t n_q, int64_t n_k, int n_seqs, int n_heads, int n_kv);

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
size_t paged_workspace(int n_seqs, int n_kv, int n_heads, int slots);
void run_append(const AppendArgs &a, hipStream_t s);
void run_fork(const PagesArgs &a, hipStream_t s);
void run_compact(const PagesArgs &a, hipStream_t s);
void run_check(const PromptArgs &a, hipStream_t s);
void run_prompt(const PromptArgs &a, int dtype, hipStream_t s);
void run_prompt_grad(const PromptArgs &a, int dtype, hipStream_t s);

}  // namespace opa
