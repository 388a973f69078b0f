// Pages of the key-value cache: new tokens into their pages (opattr_kv_append),
// the next page table (opattr_pages_fork), pages in use to the front
// (opattr_pages_compact). All whole numbers and copies: moved bytes bound the
// large calls, launches the small ones.
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

// --------------------------------------------------------------------------
// append: one wave a token, 16 bytes a lane. 40 sequences' 55k tokens, 8 heads of
// 128: 90 us, 5.0 TB/s read and written; a few tokens: the launch. Narrow tokens leave
// lanes without a piece: 2 heads of 64 17 us, 3.3 TB/s, one head 16 us, 1.7 TB/s
// --------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  const int lane = lane_id();
  if (blockIdx.x == 0) {
    check_spans(a.cu, a.n_seqs, a.n_new, a.diag, blockDim.x);
    if (a.lens_out)
      for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
        a.lens_out[b] = a.lens[b] + span_of(a.cu, b, a.n_new).count;
  }
  const int t = blockIdx.x * 4 + wave_id();
  if (t >= a.n_new) return;
  const int per = a.head_dim / 8, n = a.n_kv * per;
  const uint16_t *kr = a.kn.p + t * a.kn.ts, *vr = a.vn.p + t * a.vn.ts;
  // the first pieces' loads, before the place they go to is known
  int g = lane / per, c = (lane - g * per) * 8;
  u32x4 x = (u32x4)(0u), y = (u32x4)(0u);
  if (lane < n) {
    x = *reinterpret_cast<const u32x4 *>(kr + g * a.kn.hs + c);
    y = *reinterpret_cast<const u32x4 *>(vr + g * a.vn.hs + c);
  }
  // its sequence: as many as end at or before it
  int seq = 0;
  for (int base = 0; base < a.n_seqs; base += OPA_WAVE) {
    const int b = base + lane;
    const uint64_t m = __ballot(b < a.n_seqs && a.cu[b + 1] <= t);
    seq += __popcll(m);
    if (m != ~0ull) break;
  }
  if (seq >= a.n_seqs) return;
  const int first = clamp_to(a.cu[seq], 0, a.n_new);
  const int64_t at = (int64_t)a.lens[seq] + (t - first);
  if (t < first) return;  // offsets that decrease
  int page = -1;
  if (at >= 0 && at < a.slots) page = a.table[(int64_t)seq * a.width + (at >> a.shift)];
  if (page < 0 || page >= a.n_pages) {
    if (lane == 0) report(a.diag, OPATTR_F_DATA, 1);
    return;
  }
  const int64_t to = page * a.ps + (at & ((1 << a.shift) - 1)) * a.ts;
  for (int i = lane; i < n; i += OPA_WAVE) {
    *reinterpret_cast<u32x4 *>(a.k + to + g * a.hs + c) = x;
    *reinterpret_cast<u32x4 *>(a.v + to + g * a.hs + c) = y;
    if (i + OPA_WAVE >= n) break;
    g = (i + OPA_WAVE) / per;
    c = (i + OPA_WAVE - g * per) * 8;
    x = *reinterpret_cast<const u32x4 *>(kr + g * a.kn.hs + c);
    y = *reinterpret_cast<const u32x4 *>(vr + g * a.vn.hs + c);
  }
}

void run_append(const AppendArgs &a, hipStream_t s) {
  if (a.n_seqs == 0) return;
  const int blocks = a.n_new > 0 ? (a.n_new + 3) / 4 : 1;
  hipLaunchKernelGGL(k_kv_append, dim3(blocks), dim3(256), 0, s, a);
}

// --------------------------------------------------------------------------
// Which pages are in use: a bit each, and the set bits before each word. With
// both, the pages before one, the r-th free page and the r-th page in use are
// found by any thread at any time, so that one launch plans, writes the tables
// and copies, each block for itself. The rest of a call is how the bits come
// about (kHow):
//   kSelf   every block sets them in LDS from the table: one launch, for small
//           tables (8 sequences, 176 entries: a fork of 8 us where five
//           launches took 20 and their gaps; a table of 160 sequences, 41k
//           entries, would be 166 KB for every block to read)
//   kWords  a launch before sets them in memory, each block sums them in LDS
//   kSums   so does the sum, by a launch of its own: pools past kLdsPages pages
//           or tables past kLdsRows rows
// --------------------------------------------------------------------------
enum { kSelf, kWords, kSums };
constexpr int kSelfPages = 4096, kSelfEntries = 8192, kSelfRows = 256;
constexpr int kLdsPages = 65536, kLdsRows = 4096;
constexpr int kThreads = 256;

// Exclusive sum over the threads of a block of kT, and the total.
template <int kT>
__device__ __forceinline__ int block_scan(int x, int &total) {
  __shared__ int part[kT / OPA_WAVE];
  const int lane = lane_id(), wave = wave_id();
  const int inc = wave_sums(x);
  if (lane == OPA_WAVE - 1) part[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kT / OPA_WAVE; ++w) {
    const int p = part[w];
    if (w < wave) before += p;
    all += p;
  }
  __syncthreads();
  total = all;
  return before + inc - x;
}

// to[i] = sum of f(0 .. i-1), i = 0 .. n, by a block of kT threads; ends with a
// barrier. `to` may be where f reads.
template <int kT, class F>
__device__ __forceinline__ void prefix(int *to, int n, F f) {
  int base = 0;
  for (int i0 = 0; i0 < n; i0 += kT) {
    const int i = i0 + threadIdx.x;
    int total;
    const int at = block_scan<kT>(i < n ? f(i) : 0, total);
    if (i < n) to[i] = base + at;
    base += total;
  }
  if (threadIdx.x == 0) to[n] = base;
  __syncthreads();
}

struct Bits {
  const uint32_t *word;  // a set bit: in use, or past the last page
  const int *sum;        // set bits before each word
  int words, pages;
};

__device__ __forceinline__ int words_of(int pages) { return (pages + 31) / 32; }
// Word w's bits past the last page.
__device__ __forceinline__ uint32_t past(int w, int pages) {
  const int n = pages - 32 * w;
  return n >= 32 ? 0u : ~0u << n;
}
__device__ __forceinline__ int free_pages(const Bits &b) { return 32 * b.words - b.sum[b.words]; }
__device__ __forceinline__ int used_before(const Bits &b, int x) {
  return x >= 32 * b.words ? b.sum[b.words]
                           : b.sum[x >> 5] + __popc(b.word[x >> 5] & ((1u << (x & 31)) - 1));
}
// The r-th set bit of a word.
__device__ __forceinline__ int nth_bit(uint32_t w, int r) {
  for (int k = 0; k < r; ++k) w &= w - 1;
  return __ffs(w) - 1;
}
// The r-th page in use (kSet) or free; there are more than r.
template <bool kSet>
__device__ __forceinline__ int nth_page(const Bits &b, int r) {
  int lo = 0, hi = b.words;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((kSet ? b.sum[mid] : 32 * mid - b.sum[mid]) <= r) lo = mid; else hi = mid;
  }
  const int before = kSet ? b.sum[lo] : 32 * lo - b.sum[lo];
  return 32 * lo + nth_bit(kSet ? b.word[lo] : ~b.word[lo], r - before);
}

__device__ __forceinline__ void set_bit(uint32_t *words, int x) {
  atomicOr(&words[x >> 5], 1u << (x & 31));
}

// The words before anything of the table is in: pages held from outside, and
// bits past the last page.
__device__ __forceinline__ uint32_t first_word(const PagesArgs &a, int w) {
  uint32_t v = past(w, a.n_pages);
  if (a.held)
    for (int i = 0; i < 32; ++i) {
      const int x = 32 * w + i;
      if (x < a.n_pages && a.held[x] > 0) v |= 1u << i;
    }
  return v;
}

__global__ __launch_bounds__(kThreads) void k_pages_start(PagesArgs a) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < words_of(a.n_pages)) a.words[i] = first_word(a, i);
  if (a.refs && i < a.n_pages) a.refs[i] = a.held ? a.held[i] : 0;
}

// kSums: the sums of the words, and the requests before each row.
__global__ __launch_bounds__(1024) void k_pages_sums(PagesArgs a) {
  prefix<1024>(a.sums, words_of(a.n_pages), [&](int w) { return __popc(a.words[w]); });
  if (a.row_at) prefix<1024>(a.row_at, a.n_out, [&](int i) { return a.row_at[i]; });
}

// Page x of plane l copied to page y, by the block.
__device__ __forceinline__ void copy_page(const PagesArgs &a, int plane, int x, int y) {
  const u32x4 *from = reinterpret_cast<const u32x4 *>(a.data + plane * a.plane + x * a.page);
  u32x4 *to = reinterpret_cast<u32x4 *>(a.data + plane * a.plane + y * a.page);
  const int n = a.bytes / 16;
  int i = threadIdx.x;
  for (; i + 3 * kThreads < n; i += 4 * kThreads) {
    const u32x4 w0 = from[i], w1 = from[i + kThreads], w2 = from[i + 2 * kThreads],
                w3 = from[i + 3 * kThreads];
    to[i] = w0;
    to[i + kThreads] = w1;
    to[i + 2 * kThreads] = w2;
    to[i + 3 * kThreads] = w3;
  }
  for (; i < n; i += kThreads) to[i] = from[i];
}

// --------------------------------------------------------------------------
// fork
// --------------------------------------------------------------------------
struct ForkRow {
  int parent;    // -1: none
  int n, full;   // tokens, full pages
  bool part;     // a last page filled in part
  int want;      // pages in all, as the table can hold them
};

__device__ __forceinline__ ForkRow fork_row(const PagesArgs &a, int i) {
  ForkRow r{-1, 0, 0, false, 0};
  const int p = a.parent[i];
  if (p >= 0 && p < a.n_rows) r.parent = p;
  const int64_t most = (int64_t)a.width * a.size;
  int64_t n = r.parent >= 0 ? a.lens[r.parent] : 0;
  n = n < 0 ? 0 : n > most ? most : n;
  int64_t room = a.room ? a.room[i] : n;
  room = room < n ? n : room > most ? most : room;
  r.n = (int)n;
  r.full = r.n / a.size;
  r.part = r.n % a.size != 0;
  r.want = (int)((room + a.size - 1) / a.size);
  return r;
}

// What of row i is out of range.
__device__ __forceinline__ int fork_row_bad(const PagesArgs &a, int i, const ForkRow &r) {
  const int64_t most = (int64_t)a.width * a.size;
  const int p = a.parent[i];
  int bad = p < -1 || p >= a.n_rows;
  if (r.parent >= 0) bad += a.lens[r.parent] < 0 || a.lens[r.parent] > most;
  if (a.room) bad += a.room[i] > most;
  return bad;
}

// A page that row i keeps from its parent; -1: the entry is out of range.
__device__ __forceinline__ int kept_page(const PagesArgs &a, const ForkRow &r, int slot) {
  const int id = a.table[(int64_t)r.parent * a.width + slot];
  return id >= 0 && id < a.n_pages ? id : -1;
}

// kWords, kSums: a block a row marks what the row keeps and counts it in refs;
// row_at[i] = the new pages that it asks for.
__global__ __launch_bounds__(kThreads) void k_fork_keep(PagesArgs a) {
  const int i = blockIdx.x;
  const ForkRow r = fork_row(a, i);
  int e = 0;
  if (r.part)
    for (int j = threadIdx.x; j < i; j += kThreads) e |= a.parent[j] == r.parent;
  const int kept = r.full + (r.part && !__syncthreads_or(e));
  int bad = 0;
  for (int s = threadIdx.x; s < kept; s += kThreads) {
    const int id = kept_page(a, r, s);
    if (id < 0) {
      ++bad;
      continue;
    }
    set_bit(a.words, id);
    if (a.refs) atomicAdd(&a.refs[id], 1);
  }
  if (threadIdx.x == 0) {
    a.row_at[i] = r.want - kept;
    bad += fork_row_bad(a, i, r);
  }
  if (bad) report(a.diag, OPATTR_F_DATA, bad);
}

// Request k of the rows' (row by row) takes the k-th free page. The first
// a.give blocks write the tables; the others copy: row (block / planes), planes
// in turn.
template <int kHow>
__global__ __launch_bounds__(kThreads) void k_fork(PagesArgs a) {
  constexpr int kMost = kHow == kSelf ? kSelfPages : kLdsPages;
  constexpr int kRows = kHow == kSelf ? kSelfRows : kLdsRows;
  __shared__ uint32_t words[kHow == kSums ? 1 : kMost / 32];
  __shared__ int sums[kHow == kSums ? 1 : kMost / 32 + 1];
  __shared__ int rows[kHow == kSums ? 1 : kRows + 1];
  __shared__ int refs[kHow == kSelf ? kMost : 1];
  __shared__ ForkRow row_info[kHow == kSelf ? kRows : 1];
  const auto row_of = [&](int i) { return kHow == kSelf ? row_info[i] : fork_row(a, i); };
  if (kHow == kSelf) {  // every row's facts, once
    for (int i = threadIdx.x; i < a.n_out; i += kThreads) row_info[i] = fork_row(a, i);
    __syncthreads();
  }
  const bool copier = (int)blockIdx.x >= a.give;
  const int mine = copier ? ((int)blockIdx.x - a.give) / a.copy_planes : 0;
  if (copier) {  // a row without a part-filled page, or the first of its parent, copies none
    const ForkRow r = row_of(mine);
    if (!r.part) return;
    int e = 0;
    if (kHow == kSelf) {
      for (int j = threadIdx.x; j < mine; j += kThreads) e |= row_info[j].parent == r.parent;
      e = __syncthreads_or(e);
    } else {
      const int asks = kHow == kSums ? a.row_at[mine + 1] - a.row_at[mine] : a.row_at[mine];
      e = r.want - asks == r.full;
    }
    if (!e) return;
  }
  const int nw = words_of(a.n_pages);
  Bits b{words, sums, nw, a.n_pages};
  const int *row_at = rows;
  const bool count = kHow == kSelf && blockIdx.x == 0;
  if (kHow == kSums) {
    b.word = a.words;
    b.sum = a.sums;
    row_at = a.row_at;
  } else {
    if (kHow == kSelf) {
      for (int w = threadIdx.x; w < nw; w += kThreads) words[w] = first_word(a, w);
      if (count)
        for (int x = threadIdx.x; x < a.n_pages; x += kThreads) refs[x] = a.held ? a.held[x] : 0;
      for (int i = threadIdx.x; i < a.n_out; i += kThreads) {
        const ForkRow r = row_info[i];
        bool e = false;
        if (r.part)
          for (int j = 0; j < i; ++j) e |= row_info[j].parent == r.parent;
        rows[i] = r.want - r.full - (r.part && !e);
        if (count) {
          const int bad = fork_row_bad(a, i, r);
          if (bad) report(a.diag, OPATTR_F_DATA, bad);
        }
      }
      __syncthreads();
      int bad = 0;
      for (int i = threadIdx.x / OPA_WAVE; i < a.n_out; i += kThreads / OPA_WAVE) {
        const ForkRow r = row_of(i);
        for (int s = lane_id(); s < r.want - rows[i]; s += OPA_WAVE) {
          const int id = kept_page(a, r, s);
          if (id < 0) {
            ++bad;
            continue;
          }
          set_bit(words, id);
          if (count) atomicAdd(&refs[id], 1);
        }
      }
      if (count && bad) report(a.diag, OPATTR_F_DATA, bad);
    } else {
      for (int w = threadIdx.x; w < nw; w += kThreads) words[w] = a.words[w];
    }
    __syncthreads();
    prefix<kThreads>(sums, nw, [&](int w) { return __popc(words[w]); });
    prefix<kThreads>(rows, a.n_out, [&](int i) { return kHow == kSelf ? rows[i] : a.row_at[i]; });
  }
  const int free = free_pages(b), wanted = row_at[a.n_out];
  if (copier) {
    const ForkRow r = row_of(mine);
    if (row_at[mine] >= free) return;
    const int x = kept_page(a, r, r.full), y = nth_page<false>(b, row_at[mine]);
    if (x < 0) return;
    for (int l = ((int)blockIdx.x - a.give) % a.copy_planes; l < a.n_planes; l += a.copy_planes)
      copy_page(a, l, x, y);
    return;
  }
  const int64_t step = (int64_t)a.give * kThreads;
  const int64_t from = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t at = from; at < (int64_t)a.n_out * a.width; at += step) {
    const int i = (int)(at / a.width), s = (int)(at - (int64_t)i * a.width);
    const ForkRow r = row_of(i);
    const int kept = r.want - (row_at[i + 1] - row_at[i]), k = row_at[i] + s - kept;
    a.table_out[at] = s < kept                  ? kept_page(a, r, s)
                      : s < r.want && k < free ? nth_page<false>(b, k)
                                               : -1;
  }
  for (int64_t i = from; i < a.n_out; i += step) {
    const ForkRow r = row_of((int)i);
    const bool copy = r.part && r.want - (row_at[i + 1] - row_at[i]) == r.full;
    a.lens_out[i] = copy && row_at[i] >= free ? r.full * a.size : r.n;
  }
  if (a.refs && kHow != kSelf)  // a page given has no other reference
    for (int64_t k = from; k < wanted && k < free; k += step) a.refs[nth_page<false>(b, (int)k)] = 1;
  if (a.refs && count) {
    for (int x = threadIdx.x; x < a.n_pages; x += kThreads) {
      const bool f = !((words[x >> 5] >> (x & 31)) & 1);
      a.refs[x] = f ? x - used_before(b, x) < wanted : refs[x];
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && wanted > free)
    report(a.diag, OPATTR_F_LIMIT, wanted - free);
}

static int blocks_for(int64_t n, int most) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return b < 1 ? 1 : b > most ? most : (int)b;
}

// a launch takes fewer than 2^32 threads
constexpr int kMaxCopiers = 1 << 23;

void run_fork(const PagesArgs &args, hipStream_t s) {
  PagesArgs a = args;
  const int64_t entries = (int64_t)a.n_out * a.width;
  if (a.n_out == 0 && !a.refs) return;
  const bool self = a.n_pages <= kSelfPages && a.n_out <= kSelfRows && entries <= kSelfEntries;
  const bool lds = a.n_pages <= kLdsPages && a.n_out <= kLdsRows;
  // a table writer's setup is worth some entries; planes are shared out so that
  // a copy of many pages is many blocks, and its setup is paid a few times only
  a.give = blocks_for(entries / (self ? 2 : 4), self ? 16 : 256);
  const int each = a.n_out > 1 << 18 ? kMaxCopiers / a.n_out : 32;
  a.copy_planes = a.n_planes < each ? a.n_planes : each;
  const int64_t blocks = a.give + (a.n_pages > 0 ? (int64_t)a.n_out * a.copy_planes : 0);
  if (!self) {
    hipLaunchKernelGGL(k_pages_start, dim3((a.n_pages + kThreads) / kThreads), dim3(kThreads), 0,
                       s, a);
    if (a.n_out > 0) hipLaunchKernelGGL(k_fork_keep, dim3(a.n_out), dim3(kThreads), 0, s, a);
    if (!lds) hipLaunchKernelGGL(k_pages_sums, dim3(1), dim3(1024), 0, s, a);
  }
  const dim3 grid((uint32_t)blocks), block(kThreads);
  if (self)
    hipLaunchKernelGGL(k_fork<kSelf>, grid, block, 0, s, a);
  else if (lds)
    hipLaunchKernelGGL(k_fork<kWords>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(k_fork<kSums>, grid, block, 0, s, a);
}

// --------------------------------------------------------------------------
// compact
// --------------------------------------------------------------------------
// kWords, kSums: the pages that the table names.
__global__ __launch_bounds__(kThreads) void k_compact_mark(PagesArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  bool bad = false;
  if (i < (int64_t)a.n_rows * a.width) {
    const int id = a.table[i];
    if (id >= 0 && id < a.n_pages)
      set_bit(a.words, id);
    else
      bad = id != -1;
  }
  const int wrong = __popcll(__ballot(bad));
  if (wrong && lane_id() == 0) report(a.diag, OPATTR_F_DATA, wrong);
}

// m pages are in use. The j-th of those at or above m takes the j-th free place
// below m; there are as many of one as of the other.
// Bound by the copies: 160 sequences of up to 4096 tokens, 8 planes of 8192 pages of 32
// KB: 206 us of a turn's 239 (1.04 GB read and written in all).
template <int kHow>
__global__ __launch_bounds__(kThreads) void k_compact(PagesArgs a) {
  constexpr int kMost = kHow == kSelf ? kSelfPages : kLdsPages;
  __shared__ uint32_t words[kHow == kSums ? 1 : kMost / 32];
  __shared__ int sums[kHow == kSums ? 1 : kMost / 32 + 1];
  const int nw = words_of(a.n_pages);
  const int64_t entries = (int64_t)a.n_rows * a.width;
  Bits b{words, sums, nw, a.n_pages};
  if (kHow == kSums) {
    b.word = a.words;
    b.sum = a.sums;
  } else {
    if (kHow == kSelf) {
      for (int w = threadIdx.x; w < nw; w += kThreads) words[w] = first_word(a, w);
      __syncthreads();
      int bad = 0;
      for (int i = threadIdx.x; i < entries; i += kThreads) {
        const int id = a.table[i];
        if (id >= 0 && id < a.n_pages)
          set_bit(words, id);
        else
          bad += id != -1;
      }
      if (blockIdx.x == 0 && bad) report(a.diag, OPATTR_F_DATA, bad);
    } else {
      for (int w = threadIdx.x; w < nw; w += kThreads) words[w] = a.words[w];
    }
    __syncthreads();
    prefix<kThreads>(sums, nw, [&](int w) { return __popc(words[w]); });
  }
  const int m = a.n_pages - free_pages(b), low = used_before(b, m), n = m - low;
  const auto place = [&](int x) {
    return x < m ? x : nth_page<false>(b, used_before(b, x) - low);
  };
  const int64_t jobs = (int64_t)n * a.n_planes;
  for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
    const int at = (int)(j / a.n_planes), plane = (int)(j - (int64_t)at * a.n_planes);
    copy_page(a, plane, nth_page<true>(b, low + at), nth_page<false>(b, at));
  }
  const int64_t step = (int64_t)gridDim.x * kThreads;
  const int64_t from = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t i = from; i < entries; i += step) {
    const int id = a.table[i];
    a.table_out[i] = id >= 0 && id < a.n_pages ? place(id) : -1;
  }
  for (int64_t x = from; x < a.n_pages; x += step)
    a.moved[x] = (b.word[x >> 5] >> (x & 31)) & 1 ? place((int)x) : -1;
  if (a.live && blockIdx.x == 0 && threadIdx.x == 0) *a.live = m;
}

void run_compact(const PagesArgs &a, hipStream_t s) {
  const int64_t entries = (int64_t)a.n_rows * a.width;
  // in place, no block may read the table after another has written it
  const bool self = a.n_pages <= kSelfPages && entries <= kSelfEntries && a.table_out != a.table;
  const bool lds = a.n_pages <= kLdsPages;
  if (!self) {
    hipLaunchKernelGGL(k_pages_start, dim3((a.n_pages + kThreads) / kThreads), dim3(kThreads), 0,
                       s, a);
    if (entries > 0)
      hipLaunchKernelGGL(k_compact_mark, dim3((uint32_t)((entries + kThreads - 1) / kThreads)),
                         dim3(kThreads), 0, s, a);
    if (!lds) hipLaunchKernelGGL(k_pages_sums, dim3(1), dim3(1024), 0, s, a);
  }
  const dim3 block(kThreads);
  if (self)
    hipLaunchKernelGGL(k_compact<kSelf>, dim3(512), block, 0, s, a);
  else if (lds)
    hipLaunchKernelGGL(k_compact<kWords>, dim3(2048), block, 0, s, a);
  else
    hipLaunchKernelGGL(k_compact<kSums>, dim3(2048), block, 0, s, a);
}

}  // namespace opa
