// C entry points of the attention operators: argument checks, workspace.
#include <math.h>

#include <algorithm>

#include "attn_impl.h"

namespace opa {

constexpr int64_t kMaxTokenStride = 1 << 22;
constexpr int64_t kMaxHeadStride = (int64_t)1 << 40;
// a launch takes fewer than 2^32 threads: blocks of 256
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

static bool ok_type(int t) { return t == OPATTR_BF16 || t == OPATTR_F16; }

static bool ok_heads(int n_heads, int n_kv, int head_dim) {
  return n_kv > 0 && n_heads > 0 && n_heads <= 4096 && n_heads % n_kv == 0 && head_dim > 0 &&
         head_dim <= 128 && head_dim % 8 == 0;
}

// `n` rows (none: the tensor is not read)
static bool ok_rows(const opattr_rows *r, int64_t n, int head_dim) {
  if (!r) return false;
  if (n == 0) return true;
  return r->p && ((uintptr_t)r->p & 15) == 0 && r->token_stride % 8 == 0 &&
         r->head_stride % 8 == 0 && r->token_stride >= head_dim &&
         r->token_stride <= kMaxTokenStride && r->head_stride >= 0 &&
         r->head_stride <= kMaxHeadStride;
}

struct Steps {
  int64_t n, stride;  // the stride not negative
};
// Whether two of the pieces of `each` values at i x + j y + k z (strides; i, j, k below
// their counts) share a value.
static bool overlap(Steps x, Steps y, Steps z, int64_t each) {
  typedef __int128 wide;
  if (x.n < 1 || y.n < 1 || z.n < 1) return false;
  Steps d[3] = {x, y, z};
  std::sort(d, d + 3, [](const Steps &a, const Steps &b) { return a.stride < b.stride; });
  // each dimension's step past all of those below it: any order of a dense tensor's
  // dimensions, and slices of it
  wide extent = each;
  bool nested = true;
  for (const Steps &s : d) {
    if (s.n > 1 && s.stride < each) return true;
    nested = nested && (s.n == 1 || s.stride >= extent);
    extent += (wide)(s.n - 1) * s.stride;
  }
  if (nested) return false;
  // a difference nearer to 0 than `each`: for all of two dimensions, the nearest two
  // of the longest
  std::sort(d, d + 3, [](const Steps &a, const Steps &b) { return a.n < b.n; });
  const wide step = d[2].stride, most = d[2].n - 1;
  for (int64_t i = 0; i < d[0].n; ++i)
    for (int64_t j = 1 - d[1].n; j < d[1].n; ++j) {
      const wide at = (wide)i * d[0].stride + (wide)j * d[1].stride;
      const wide to = at < 0 ? -at : at;
      const wide k = to / step < most ? to / step : most;
      if (((i || j || k) && to - k * step < each) || (k < most && (k + 1) * step - to < each))
        return true;
    }
  return false;
}

// Rows that are written.
static bool ok_out(const opattr_rows *r, int64_t n, int heads, int head_dim) {
  return ok_rows(r, n, head_dim) &&
         !overlap({n, r->token_stride}, {heads, r->head_stride}, {1, 0}, head_dim);
}

static Rows rows(const opattr_rows *r) {
  return {static_cast<uint16_t *>(r->p), r->token_stride, r->head_stride};
}

static bool ok_shape(const opattr_attn_shape *a) {
  if (!a || a->n_q < 0 || a->n_k < 0 || a->n_q >= (int64_t)1 << 30 ||
      a->n_k >= (int64_t)1 << 30 || a->n_seqs < 0 || a->n_seqs >= 1 << 20 ||
      !ok_type(a->dtype) || (a->causal != 0 && a->causal != 1) ||
      !ok_heads(a->n_heads, a->n_kv_heads, a->head_dim) || !isfinite(a->scale))
    return false;
  if (a->n_seqs > 0 && (!a->cu_q || !a->cu_k)) return false;
  // one block for every tile of 128 rows at most
  return ((a->n_q > a->n_k ? a->n_q : a->n_k) / 128 + a->n_seqs) * a->n_heads <= kMaxGrid;
}

// A window of a causal mask. No sequence has 2^30 tokens: what is past them says
// nothing, and sums of the two stay in 32 bits.
constexpr int32_t kMostWindow = (1 << 30) - 1;
static bool ok_window(int32_t window, int32_t sinks) { return window >= 1 && sinks >= 0; }
static int32_t at_most(int32_t x) { return std::min(x, kMostWindow); }

// Of whole prompts: a token's place and a window past it stay in 32 bits. (A block of
// several heads has as many fewer rows: one launch takes them where it takes ok_shape's.)
constexpr int64_t kMostWindowTokens = (int64_t)1 << 29;
static bool ok_window_shape(const opattr_attn_shape *a, int32_t window, int32_t sinks) {
  return ok_shape(a) && a->causal && ok_window(window, sinks) && a->n_q < kMostWindowTokens &&
         a->n_k < kMostWindowTokens;
}

static PromptArgs prompt_args(const opattr_attn_shape *a, int32_t window, int32_t sinks,
                              opattr_diag *diag) {
  PromptArgs p{};
  p.cu_q = a->cu_q;
  p.cu_k = a->cu_k;
  p.n_q = (int)a->n_q;
  p.n_k = (int)a->n_k;
  p.n_seqs = a->n_seqs;
  p.n_heads = a->n_heads;
  p.n_kv = a->n_kv_heads;
  p.group = a->n_heads / a->n_kv_heads;
  p.head_dim = a->head_dim;
  p.causal = a->causal;
  p.window = (int)std::min<int64_t>(window, kMostWindowTokens);
  p.sinks = at_most(sinks);
  p.head_shift = window ? window_heads(p.group) : 0;
  p.scale = a->scale;
  p.diag = diag;
  return p;
}

// float16: the largest norms
static size_t norms_bytes(const opattr_attn_shape *a) {
  return a->dtype == OPATTR_F16
             ? align256((size_t)norm_slots(a->n_q, a->n_k, a->n_seqs) *
                        (a->n_heads + a->n_kv_heads) * 4)
             : 0;
}

static bool ok_ws(const void *ws, size_t have, size_t need) {
  return need == 0 || (ws && ((uintptr_t)ws & 255) == 0 && have >= need);
}

static bool ok_pages(const opattr_kv_pages *c) {
  if (!c || c->n_pages < 0 || c->n_seqs < 0 || c->n_seqs >= 1 << 20 || c->table_stride < 0 ||
      c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) ||
      !ok_type(c->dtype) || !ok_heads(c->n_kv_heads, c->n_kv_heads, c->head_dim))
    return false;
  if (c->n_seqs > 0 && c->table_stride > 0 && !c->table) return false;
  if ((int64_t)c->table_stride * c->page_size >= (int64_t)1 << 30) return false;
  if (c->n_pages == 0) return true;
  const int64_t most = (int64_t)1 << 40;
  return c->k && c->v && (((uintptr_t)c->k | (uintptr_t)c->v) & 15) == 0 &&
         (c->page_stride | c->token_stride | c->head_stride) % 8 == 0 && c->page_stride >= 0 &&
         c->page_stride <= most && c->token_stride >= 0 && c->token_stride <= most &&
         c->head_stride >= 0 && c->head_stride <= most;
}

// Pages that are written.
static bool ok_pages_out(const opattr_kv_pages *c) {
  return ok_pages(c) && !overlap({c->n_pages, c->page_stride}, {c->page_size, c->token_stride},
                                 {c->n_kv_heads, c->head_stride}, c->head_dim);
}

// Tokens of a sequence that its query sees, at most; of the cache of 8 bits by whole runs
// of 16 at the sinks' end and the window's begin.
static int most_seen(const opattr_kv_pages *c, int32_t window, int32_t sinks) {
  const int slots = c->table_stride * c->page_size;
  return window ? std::min(slots, at_most(window) + at_most(sinks)) : slots;
}
static int most_seen(const opattr_kv_scaled *c, int32_t window, int32_t sinks) {
  const int64_t slots = (int64_t)c->table_stride * c->page_size;
  const int64_t seen = (int64_t)at_most(window) + 15 + (at_most(sinks) + 15) / 16 * 16;
  return (int)std::min(slots, seen);
}

// The cache of 8 bits: as above, in bytes.
static bool ok_scaled(const opattr_kv_scaled *c) {
  if (!c || c->n_pages < 0 || c->n_seqs < 0 || c->n_seqs >= 1 << 20 || c->table_stride < 0 ||
      c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) ||
      c->block_size < 1 || c->block_size > c->page_size || (c->block_size & (c->block_size - 1)) ||
      !ok_type(c->dtype) || !ok_heads(c->n_kv_heads, c->n_kv_heads, c->head_dim) ||
      c->head_dim % 16)
    return false;
  if (c->n_seqs > 0 && c->table_stride > 0 && !c->table) return false;
  if ((int64_t)c->table_stride * c->page_size >= (int64_t)1 << 30) return false;
  if (c->n_pages == 0) return true;
  if (!c->k || !c->v || (((uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0 || !c->k_scale ||
      !c->v_scale || (c->page_stride | c->token_stride | c->head_stride) % 16 != 0)
    return false;
  const int64_t most = (int64_t)1 << 40;
  for (int64_t s : {c->page_stride, c->token_stride, c->head_stride, c->scale_page_stride,
                    c->scale_block_stride, c->scale_head_stride})
    if (s < 0 || s > most) return false;
  return true;
}
static bool ok_scaled_out(const opattr_kv_scaled *c) {
  return ok_scaled(c) &&
         !overlap({c->n_pages, c->page_stride}, {c->page_size, c->token_stride},
                  {c->n_kv_heads, c->head_stride}, c->head_dim) &&
         !overlap({c->n_pages, c->scale_page_stride},
                  {c->page_size / c->block_size, c->scale_block_stride},
                  {c->n_kv_heads, c->scale_head_stride}, 1);
}

static int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

// The partial results of the attention of one token a sequence, and with what their join
// has to know.
static size_t parts_of(const opattr_kv_pages *c, int32_t n_heads, int most) {
  return align256(paged_parts(c->n_seqs, c->n_kv_heads, n_heads, most));
}
static size_t parts_of(const opattr_kv_scaled *c, int32_t n_heads, int most) {
  return align256(scaled_parts(c->n_seqs, c->n_kv_heads, n_heads, most));
}
template <class Cache>
static size_t parts_and_shares(const Cache *c, int32_t n_heads, int most) {
  const size_t parts = parts_of(c, n_heads, most);
  return parts ? parts + align256((size_t)c->n_seqs * 8) : 0;
}

// What the attention of one token a sequence takes of a cache, of either kind.
template <class Cache>
static void paged_args(PagedArgs &a, const Cache *c, int32_t n_heads, int32_t window,
                       int32_t sinks, const opattr_rows *q, const int32_t *lens, float scale,
                       const opattr_rows *out, float *lse, opattr_diag *diag, void *ws) {
  a.ps = c->page_stride;
  a.ts = c->token_stride;
  a.hs = c->head_stride;
  a.n_pages = c->n_pages;
  a.shift = log2_of(c->page_size);
  a.slots = c->table_stride * c->page_size;
  a.window = at_most(window);
  a.sinks = at_most(sinks);
  a.most = most_seen(c, window, sinks);
  a.table = c->table;
  a.n_seqs = c->n_seqs;
  a.width = c->table_stride;
  a.n_kv = c->n_kv_heads;
  a.group = n_heads / c->n_kv_heads;
  a.n_heads = n_heads;
  a.head_dim = c->head_dim;
  a.q = rows(q);
  a.out = rows(out);
  a.lens = lens;
  a.scale = scale;
  a.lse = lse;
  a.diag = diag;
  const size_t parts = parts_of(c, n_heads, a.most);
  if (parts == 0) return;
  a.part = static_cast<float *>(ws);
  a.shares = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + parts);
}

constexpr int kMaxPages = 1 << 24;

static bool ok_pool(const opattr_page_pool *p) {
  if (!p || p->n_planes < 0 || p->n_planes > 65536 || p->n_pages < 0 || p->n_pages > kMaxPages ||
      p->page_size < 1 || p->page_bytes < 0 || p->page_bytes % 16)
    return false;
  if (p->n_planes == 0 || p->n_pages == 0 || p->page_bytes == 0) return true;
  return p->data && ((uintptr_t)p->data & 15) == 0 && p->plane_stride % 16 == 0 &&
         p->page_stride % 16 == 0 && p->plane_stride >= 0 && p->page_stride >= p->page_bytes &&
         !overlap({p->n_pages, p->page_stride}, {p->n_planes, p->plane_stride}, {1, 0},
                  p->page_bytes);
}

// rows x width entries of a page table
static bool ok_table(int64_t rows, int64_t width) {
  return rows >= 0 && rows < 1 << 20 && width >= 0 && rows * width < (int64_t)1 << 31;
}

// a bit a page, and the set bits before each word and in all
static size_t bits_bytes(int n_pages) {
  return align256((size_t)(n_pages / 32 + 1) * 4) + align256((size_t)(n_pages / 32 + 2) * 4);
}

static PagesArgs pages_args(const opattr_page_pool *p, opattr_diag *diag) {
  PagesArgs a{};
  a.data = static_cast<char *>(p->data);
  a.plane = p->plane_stride;
  a.page = p->page_stride;
  a.n_planes = p->page_bytes ? p->n_planes : 0;
  a.n_pages = p->n_pages;
  a.bytes = p->page_bytes;
  a.size = p->page_size;
  a.held = p->held;
  a.diag = diag;
  return a;
}

// the next `n` integers of a workspace
static int32_t *take(char *&at, size_t n) {
  int32_t *p = reinterpret_cast<int32_t *>(at);
  at += align256(n * 4);
  return p;
}

static int launched() { return hipGetLastError() == hipSuccess ? OPATTR_OK : OPATTR_ERR_HIP; }

// The forward pass and the gradient; window 0: none.
static int prompt(const opattr_attn_shape *a, int32_t window, int32_t sinks, const opattr_rows *q,
                  const opattr_rows *k, const opattr_rows *v, const opattr_rows *out, float *lse,
                  opattr_diag *diag, void *stream) {
  if (!ok_shape(a) || !ok_rows(q, a->n_q, a->head_dim) || !ok_rows(k, a->n_k, a->head_dim) ||
      !ok_rows(v, a->n_k, a->head_dim) || !ok_out(out, a->n_q, a->n_heads, a->head_dim))
    return OPATTR_ERR_INVALID_ARG;
  PromptArgs p = prompt_args(a, window, sinks, diag);
  p.q = rows(q);
  p.k = rows(k);
  p.v = rows(v);
  p.out = rows(out);
  p.lse = lse;
  run_prompt(p, a->dtype, (hipStream_t)stream);
  return launched();
}

static size_t grad_workspace(const opattr_attn_shape *a, int32_t window, int32_t sinks) {
  if (!ok_shape(a)) return 0;
  const size_t dp = a->head_dim <= 64 ? 64 : 128;
  const PromptArgs p = prompt_args(a, window, sinks, nullptr);
  const GradSplits x = grad_splits(a->n_q, a->n_k, a->n_seqs, a->n_heads, a->n_kv_heads, p.window,
                                   p.sinks);
  return align256((size_t)a->n_q * a->n_heads * 8) + norms_bytes(a) +
         (size_t)grad_parts(x, a->n_k, a->n_seqs) * 128 * a->n_kv_heads * 2 * dp * 4;
}

static int prompt_grad(const opattr_attn_shape *a, int32_t window, int32_t sinks,
                       const opattr_rows *dout, const opattr_rows *q, const opattr_rows *k,
                       const opattr_rows *v, const opattr_rows *out, const float *lse,
                       const opattr_rows *dq, const opattr_rows *dk, const opattr_rows *dv,
                       opattr_diag *diag, void *ws, size_t ws_bytes, void *stream) {
  if (!ok_shape(a) || !ok_rows(dout, a->n_q, a->head_dim) || !ok_rows(q, a->n_q, a->head_dim) ||
      !ok_rows(k, a->n_k, a->head_dim) || !ok_rows(v, a->n_k, a->head_dim) ||
      !ok_rows(out, a->n_q, a->head_dim) || !ok_out(dq, a->n_q, a->n_heads, a->head_dim) ||
      !ok_out(dk, a->n_k, a->n_kv_heads, a->head_dim) ||
      !ok_out(dv, a->n_k, a->n_kv_heads, a->head_dim) || (a->n_q > 0 && !lse))
    return OPATTR_ERR_INVALID_ARG;
  if (!ok_ws(ws, ws_bytes, grad_workspace(a, window, sinks))) return OPATTR_ERR_WORKSPACE;
  PromptArgs p = prompt_args(a, window, sinks, diag);
  p.dout = rows(dout);
  p.q = rows(q);
  p.k = rows(k);
  p.v = rows(v);
  p.out = rows(out);
  p.lse = const_cast<float *>(lse);
  p.dq = rows(dq);
  p.dk = rows(dk);
  p.dv = rows(dv);
  char *at = static_cast<char *>(ws);
  p.rows = reinterpret_cast<float *>(at);
  at += align256((size_t)a->n_q * a->n_heads * 8);
  if (a->dtype == OPATTR_F16) p.norms = reinterpret_cast<uint32_t *>(at);
  p.norm_slots = (int)norm_slots(a->n_q, a->n_k, a->n_seqs);
  p.part = reinterpret_cast<float *>(at + norms_bytes(a));
  const GradSplits x = grad_splits(a->n_q, a->n_k, a->n_seqs, a->n_heads, a->n_kv_heads, p.window,
                                   p.sinks);
  p.splits = x.most;
  p.split_steps = x.steps;
  p.sink_tiles = x.sink_tiles;
  p.sink_shift = x.sink_shift;
  p.sink_most = x.sink_most;
  p.sink_slots = x.sink_slots;
  p.sink_sums = x.sink_sums;
  run_prompt_grad(p, a->dtype, (hipStream_t)stream);
  return launched();
}

static size_t paged_bytes(const opattr_kv_pages *c, int32_t n_heads, int32_t window,
                          int32_t sinks) {
  if (!ok_pages(c) || !ok_heads(n_heads, c->n_kv_heads, c->head_dim)) return 0;
  return parts_and_shares(c, n_heads, most_seen(c, window, sinks));
}

template <class Cache>
static bool ok_paged_call(const Cache *c, int32_t n_heads, const opattr_rows *q,
                          const int32_t *lens, float scale, const opattr_rows *out) {
  return ok_heads(n_heads, c->n_kv_heads, c->head_dim) && n_heads / c->n_kv_heads <= 16 &&
         isfinite(scale) && ok_rows(q, c->n_seqs, c->head_dim) &&
         ok_out(out, c->n_seqs, n_heads, c->head_dim) && (c->n_seqs == 0 || lens) &&
         (int64_t)c->n_seqs * n_heads <= kMaxGrid / 2;
}

static int paged(const opattr_kv_pages *c, int32_t n_heads, int32_t window, int32_t sinks,
                 const opattr_rows *q, const int32_t *lens, float scale, const opattr_rows *out,
                 float *lse, opattr_diag *diag, void *ws, size_t ws_bytes, void *stream) {
  if (!ok_pages(c) || !ok_paged_call(c, n_heads, q, lens, scale, out))
    return OPATTR_ERR_INVALID_ARG;
  if (!ok_ws(ws, ws_bytes, paged_bytes(c, n_heads, window, sinks))) return OPATTR_ERR_WORKSPACE;
  PagedArgs a{};
  paged_args(a, c, n_heads, window, sinks, q, lens, scale, out, lse, diag, ws);
  a.k = static_cast<const uint16_t *>(c->k);
  a.v = static_cast<const uint16_t *>(c->v);
  run_paged(a, c->dtype, (hipStream_t)stream);
  return launched();
}

}  // namespace opa

using namespace opa;

extern "C" {

int opattr_attn_prompt(const opattr_attn_shape *a, const opattr_rows *q, const opattr_rows *k,
                       const opattr_rows *v, const opattr_rows *out, float *lse,
                       opattr_diag *diag, void *stream) {
  return prompt(a, 0, 0, q, k, v, out, lse, diag, stream);
}

int opattr_attn_prompt_window(const opattr_attn_shape *a, int32_t window, int32_t sinks,
                              const opattr_rows *q, const opattr_rows *k, const opattr_rows *v,
                              const opattr_rows *out, float *lse, opattr_diag *diag,
                              void *stream) {
  if (!ok_window_shape(a, window, sinks)) return OPATTR_ERR_INVALID_ARG;
  return prompt(a, window, sinks, q, k, v, out, lse, diag, stream);
}

size_t opattr_attn_prompt_grad_workspace_bytes(const opattr_attn_shape *a) {
  return grad_workspace(a, 0, 0);
}

size_t opattr_attn_prompt_window_grad_workspace_bytes(const opattr_attn_shape *a, int32_t window,
                                                      int32_t sinks) {
  if (!ok_window_shape(a, window, sinks)) return 0;
  return grad_workspace(a, window, sinks);
}

int opattr_attn_prompt_grad(const opattr_attn_shape *a, const opattr_rows *dout,
                            const opattr_rows *q, const opattr_rows *k, const opattr_rows *v,
                            const opattr_rows *out, const float *lse, const opattr_rows *dq,
                            const opattr_rows *dk, const opattr_rows *dv, opattr_diag *diag,
                            void *ws, size_t ws_bytes, void *stream) {
  return prompt_grad(a, 0, 0, dout, q, k, v, out, lse, dq, dk, dv, diag, ws, ws_bytes, stream);
}

int opattr_attn_prompt_window_grad(const opattr_attn_shape *a, int32_t window, int32_t sinks,
                                   const opattr_rows *dout, const opattr_rows *q,
                                   const opattr_rows *k, const opattr_rows *v,
                                   const opattr_rows *out, const float *lse,
                                   const opattr_rows *dq, const opattr_rows *dk,
                                   const opattr_rows *dv, opattr_diag *diag, void *ws,
                                   size_t ws_bytes, void *stream) {
  if (!ok_window_shape(a, window, sinks)) return OPATTR_ERR_INVALID_ARG;
  return prompt_grad(a, window, sinks, dout, q, k, v, out, lse, dq, dk, dv, diag, ws, ws_bytes,
                     stream);
}

size_t opattr_attn_paged_workspace_bytes(const opattr_kv_pages *c, int32_t n_heads) {
  return paged_bytes(c, n_heads, 0, 0);
}

size_t opattr_attn_paged_window_workspace_bytes(const opattr_kv_pages *c, int32_t n_heads,
                                                int32_t window, int32_t sinks) {
  return ok_window(window, sinks) ? paged_bytes(c, n_heads, window, sinks) : 0;
}

int opattr_attn_paged(const opattr_kv_pages *c, int32_t n_heads, const opattr_rows *q,
                      const int32_t *lens, float scale, const opattr_rows *out, float *lse,
                      opattr_diag *diag, void *ws, size_t ws_bytes, void *stream) {
  return paged(c, n_heads, 0, 0, q, lens, scale, out, lse, diag, ws, ws_bytes, stream);
}

int opattr_attn_paged_window(const opattr_kv_pages *c, int32_t n_heads, int32_t window,
                             int32_t sinks, const opattr_rows *q, const int32_t *lens, float scale,
                             const opattr_rows *out, float *lse, opattr_diag *diag, void *ws,
                             size_t ws_bytes, void *stream) {
  if (!ok_window(window, sinks)) return OPATTR_ERR_INVALID_ARG;
  return paged(c, n_heads, window, sinks, q, lens, scale, out, lse, diag, ws, ws_bytes, stream);
}

size_t opattr_attn_paged_scaled_workspace_bytes(const opattr_kv_scaled *c, int32_t n_heads,
                                                int32_t window, int32_t sinks) {
  if (!ok_scaled(c) || !ok_heads(n_heads, c->n_kv_heads, c->head_dim) ||
      !ok_window(window, sinks))
    return 0;
  return parts_and_shares(c, n_heads, most_seen(c, window, sinks));
}

int opattr_attn_paged_scaled(const opattr_kv_scaled *c, int32_t n_heads, int32_t window,
                             int32_t sinks, const opattr_rows *q, const int32_t *lens, float scale,
                             const opattr_rows *out, float *lse, opattr_diag *diag, void *ws,
                             size_t ws_bytes, void *stream) {
  if (!ok_window(window, sinks) || !ok_scaled(c) ||
      !ok_paged_call(c, n_heads, q, lens, scale, out))
    return OPATTR_ERR_INVALID_ARG;
  if (!ok_ws(ws, ws_bytes, opattr_attn_paged_scaled_workspace_bytes(c, n_heads, window, sinks)))
    return OPATTR_ERR_WORKSPACE;
  ScaledArgs a{};
  paged_args(a, c, n_heads, window, sinks, q, lens, scale, out, lse, diag, ws);
  a.k_codes = static_cast<const uint8_t *>(c->k);
  a.v_codes = static_cast<const uint8_t *>(c->v);
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.sps = c->scale_page_stride;
  a.sbs = c->scale_block_stride;
  a.shs = c->scale_head_stride;
  a.block_shift = log2_of(c->block_size);
  run_paged_scaled(a, c->dtype, (hipStream_t)stream);
  return launched();
}

int opattr_kv_append_scaled(const opattr_kv_scaled *c, int64_t n_new, const int32_t *cu,
                            const opattr_rows *k_new, const opattr_rows *v_new,
                            const int32_t *lens, int32_t *lens_out, opattr_diag *diag,
                            void *stream) {
  if (!ok_scaled_out(c) || n_new < 0 || n_new > kMaxGrid * 4 ||
      !ok_rows(k_new, n_new, c->head_dim) || !ok_rows(v_new, n_new, c->head_dim) ||
      (c->n_seqs > 0 && (!cu || !lens)) || (lens_out && lens_out == lens) ||
      append_units(n_new, c->n_seqs, log2_of(c->block_size)) * c->n_kv_heads * 2 > kMaxGrid * 4)
    return OPATTR_ERR_INVALID_ARG;
  AppendScaledArgs a{};
  a.k = static_cast<uint8_t *>(c->k);
  a.v = static_cast<uint8_t *>(c->v);
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.ps = c->page_stride;
  a.ts = c->token_stride;
  a.hs = c->head_stride;
  a.sps = c->scale_page_stride;
  a.sbs = c->scale_block_stride;
  a.shs = c->scale_head_stride;
  a.n_pages = c->n_pages;
  a.shift = log2_of(c->page_size);
  a.slots = c->table_stride * c->page_size;
  a.block_shift = log2_of(c->block_size);
  a.table = c->table;
  a.n_seqs = c->n_seqs;
  a.width = c->table_stride;
  a.n_kv = c->n_kv_heads;
  a.head_dim = c->head_dim;
  a.n_new = (int)n_new;
  a.cu = cu;
  a.lens = lens;
  a.kn = rows(k_new);
  a.vn = rows(v_new);
  a.lens_out = lens_out;
  a.diag = diag;
  run_append_scaled(a, c->dtype, (hipStream_t)stream);
  return launched();
}

int opattr_kv_append(const opattr_kv_pages *c, int64_t n_new, const int32_t *cu,
                     const opattr_rows *k_new, const opattr_rows *v_new, const int32_t *lens,
                     int32_t *lens_out, opattr_diag *diag, void *stream) {
  if (!ok_pages_out(c) || n_new < 0 || n_new > kMaxGrid * 4 ||
      !ok_rows(k_new, n_new, c->head_dim) || !ok_rows(v_new, n_new, c->head_dim) ||
      (c->n_seqs > 0 && (!cu || !lens)) || (lens_out && lens_out == lens))
    return OPATTR_ERR_INVALID_ARG;
  AppendArgs a{};
  a.k = static_cast<uint16_t *>(c->k);
  a.v = static_cast<uint16_t *>(c->v);
  a.ps = c->page_stride;
  a.ts = c->token_stride;
  a.hs = c->head_stride;
  a.n_pages = c->n_pages;
  a.shift = log2_of(c->page_size);
  a.slots = c->table_stride * c->page_size;
  a.table = c->table;
  a.n_seqs = c->n_seqs;
  a.width = c->table_stride;
  a.n_kv = c->n_kv_heads;
  a.head_dim = c->head_dim;
  a.n_new = (int)n_new;
  a.cu = cu;
  a.lens = lens;
  a.kn = rows(k_new);
  a.vn = rows(v_new);
  a.lens_out = lens_out;
  a.diag = diag;
  run_append(a, (hipStream_t)stream);
  return launched();
}

size_t opattr_pages_fork_workspace_bytes(int32_t n_rows, int32_t n_out, int32_t width,
                                         int32_t n_pages) {
  if (!ok_table(n_rows, width) || !ok_table(n_out, width) || n_pages < 0 || n_pages > kMaxPages)
    return 0;
  return bits_bytes(n_pages) + align256(((size_t)n_out + 1) * 4);
}

int opattr_pages_fork(const opattr_page_pool *p, const int32_t *table, const int32_t *lens,
                      int32_t n_rows, int32_t width, const int32_t *parent, const int32_t *room,
                      int32_t n_out, int32_t *table_out, int32_t *lens_out, int32_t *refs,
                      opattr_diag *diag, void *ws, size_t ws_bytes, void *stream) {
  if (!ok_pool(p) || !ok_table(n_rows, width) || !ok_table(n_out, width) ||
      (n_rows > 0 && (!lens || (width > 0 && !table))) ||
      (n_out > 0 && (!parent || !lens_out || (width > 0 && !table_out))) ||
      (table_out && table_out == table) || (lens_out && lens_out == lens) ||
      (refs && refs == p->held))
    return OPATTR_ERR_INVALID_ARG;
  if (!ok_ws(ws, ws_bytes, opattr_pages_fork_workspace_bytes(n_rows, n_out, width, p->n_pages)))
    return OPATTR_ERR_WORKSPACE;
  PagesArgs a = pages_args(p, diag);
  a.table = table;
  a.lens = lens;
  a.parent = parent;
  a.room = room;
  a.n_rows = n_rows;
  a.width = width;
  a.n_out = n_out;
  a.table_out = table_out;
  a.lens_out = lens_out;
  a.refs = refs;
  char *at = static_cast<char *>(ws);
  a.words = reinterpret_cast<uint32_t *>(take(at, p->n_pages / 32 + 1));
  a.sums = take(at, p->n_pages / 32 + 2);
  a.row_at = take(at, (size_t)n_out + 1);
  run_fork(a, (hipStream_t)stream);
  return launched();
}

size_t opattr_pages_compact_workspace_bytes(int32_t n_pages) {
  if (n_pages < 0 || n_pages > kMaxPages) return 0;
  return bits_bytes(n_pages);
}

int opattr_pages_compact(const opattr_page_pool *p, const int32_t *table, int32_t n_rows,
                         int32_t width, int32_t *table_out, int32_t *moved, int32_t *live,
                         opattr_diag *diag, void *ws, size_t ws_bytes, void *stream) {
  if (!ok_pool(p) || !ok_table(n_rows, width) ||
      ((int64_t)n_rows * width > 0 && (!table || !table_out)) || (p->n_pages > 0 && !moved) ||
      (moved && moved == p->held))
    return OPATTR_ERR_INVALID_ARG;
  if (!ok_ws(ws, ws_bytes, opattr_pages_compact_workspace_bytes(p->n_pages)))
    return OPATTR_ERR_WORKSPACE;
  PagesArgs a = pages_args(p, diag);
  a.table = table;
  a.n_rows = n_rows;
  a.width = width;
  a.table_out = table_out;
  a.moved = moved;
  a.live = live;
  char *at = static_cast<char *>(ws);
  a.words = reinterpret_cast<uint32_t *>(take(at, p->n_pages / 32 + 1));
  a.sums = take(at, p->n_pages / 32 + 2);
  run_compact(a, (hipStream_t)stream);
  return launched();
}

}  // extern "C"
