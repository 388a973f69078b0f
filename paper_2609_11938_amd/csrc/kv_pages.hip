// Pages of the key-value cache: new tokens into their pages (opattr_kv_append),
// the next page table (opattr_pages_fork), pages in use to the front
// (opattr_pages_compact). All whole numbers and copies: moved bytes bound the
// large calls, launches the small ones.
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

// --------------------------------------------------------------------------
// append: one wave a token, 16 bytes a lane
// --------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  const int lane = lane_id();
  if (blockIdx.x == 0) {
    check_spans(a.cu, a.n_seqs, a.n_new, a.diag);
    if (a.lens_out)
      for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x)
        a.lens_out[b] = a.lens[b] + span_of(a.cu, b, a.n_new).count;
  }
  const int t = blockIdx.x * 4 + wave_id();
  if (t >= a.n_new) return;
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
  const int per = a.head_dim / 8, n = a.n_kv * per;
  for (int i = lane; i < n; i += OPA_WAVE) {
    const int g = i / per, c = (i - g * per) * 8;
    const u32x4 x = *reinterpret_cast<const u32x4 *>(a.kn.p + t * a.kn.ts + g * a.kn.hs + c);
    const u32x4 y = *reinterpret_cast<const u32x4 *>(a.vn.p + t * a.vn.ts + g * a.vn.hs + c);
    *reinterpret_cast<u32x4 *>(a.k + to + g * a.hs + c) = x;
    *reinterpret_cast<u32x4 *>(a.v + to + g * a.hs + c) = y;
  }
}

void run_append(const AppendArgs &a, hipStream_t s) {
  if (a.n_seqs == 0) return;
  const int blocks = a.n_new > 0 ? (a.n_new + 3) / 4 : 1;
  hipLaunchKernelGGL(k_kv_append, dim3(blocks), dim3(256), 0, s, a);
}

// --------------------------------------------------------------------------
// scans over a block of 1024 threads
// --------------------------------------------------------------------------
constexpr int kScan = 1024;

// Exclusive sum over the block's threads, and the total. Ends with a barrier
// before `part` may be used again.
__device__ __forceinline__ int block_scan(int x, int *part, int &total) {
  const int lane = lane_id(), wave = wave_id();
  int inc = x;
#pragma unroll
  for (int d = 1; d < OPA_WAVE; d <<= 1) {
    const int o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  if (lane == OPA_WAVE - 1) part[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kScan / OPA_WAVE; ++w) {
    const int p = part[w];
    if (w < wave) before += p;
    all += p;
  }
  __syncthreads();
  total = all;
  return before + inc - x;
}

// Sum of x over the block, for every thread.
__device__ __forceinline__ int block_sum(int x, int *part) {
  int total;
  block_scan(x, part, total);
  return total;
}

__global__ void k_pages_zero(int32_t *p, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0;
}

// Page x of plane l copied to page y, by the block.
__device__ __forceinline__ void copy_page(const PagesArgs &a, int plane, int x, int y) {
  const u32x4 *from = reinterpret_cast<const u32x4 *>(a.data + plane * a.plane + x * a.page);
  u32x4 *to = reinterpret_cast<u32x4 *>(a.data + plane * a.plane + y * a.page);
  for (int i = threadIdx.x; i < a.bytes / 16; i += blockDim.x) to[i] = from[i];
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

// A block a row: the entries it keeps, counted in `used`; row_at[i] = new pages
// it asks for.
__global__ __launch_bounds__(256) void k_fork_keep(PagesArgs a) {
  const int i = blockIdx.x;
  const ForkRow r = fork_row(a, i);
  __shared__ int earlier;
  if (threadIdx.x == 0) earlier = 0;
  __syncthreads();
  if (r.parent >= 0 && r.part) {
    bool e = false;
    for (int j = threadIdx.x; j < i; j += blockDim.x) e |= a.parent[j] == r.parent;
    if (e) earlier = 1;
  }
  __syncthreads();
  const int kept = r.full + (r.part && !earlier);
  int bad = 0;
  for (int s = threadIdx.x; s < a.width; s += blockDim.x) {
    int id = -1;
    if (s < kept) {
      id = a.table[(int64_t)r.parent * a.width + s];
      if (id < 0 || id >= a.n_pages) {
        id = -1;
        ++bad;
      } else {
        atomicAdd(&a.used[id], 1);
      }
    }
    a.table_out[(int64_t)i * a.width + s] = id;
  }
  if (threadIdx.x == 0) {
    a.row_at[i] = r.want - kept;
    a.lens_out[i] = r.n;
    const int p = a.parent[i];
    bad += p < -1 || p >= a.n_rows;
    if (r.parent >= 0)
      bad += a.lens[r.parent] < 0 || a.lens[r.parent] > (int64_t)a.width * a.size;
    if (a.room) bad += a.room[i] > (int64_t)a.width * a.size;
  }
  if (bad) report(a.diag, OPATTR_F_DATA, bad);
}

__device__ __forceinline__ bool is_free(const PagesArgs &a, int x) {
  return x < a.n_pages && a.used[x] == 0 && !(a.held && a.held[x] > 0);
}

// Free pages of every block of pages; the last block instead turns row_at into
// the requests before each row, row_at[n_out] their total.
__global__ __launch_bounds__(kScan) void k_fork_count(PagesArgs a) {
  __shared__ int part[kScan / OPA_WAVE];
  if (blockIdx.x + 1 == gridDim.x) {
    int base = 0;
    for (int i0 = 0; i0 < a.n_out; i0 += kScan) {
      const int i = i0 + threadIdx.x;
      int total;
      const int at = block_scan(i < a.n_out ? a.row_at[i] : 0, part, total);
      if (i < a.n_out) a.row_at[i] = base + at;
      base += total;
    }
    if (threadIdx.x == 0) a.row_at[a.n_out] = base;
    return;
  }
  int n = 0;
  for (int j = 0; j < kPageBlock / kScan; ++j)
    n += is_free(a, blockIdx.x * kPageBlock + j * kScan + threadIdx.x);
  n = block_sum(n, part);
  if (threadIdx.x == 0) a.count[blockIdx.x] = n;
}

// The free page of rank r answers request r. Requests past the free pages stay
// -1; a row whose copy is among them ends at its full pages.
__global__ __launch_bounds__(kScan) void k_fork_give(PagesArgs a) {
  __shared__ int part[kScan / OPA_WAVE];
  int before = 0;
  for (int j = threadIdx.x; j < (int)blockIdx.x; j += kScan) before += a.count[j];
  before = block_sum(before, part);
  const int wanted = a.row_at[a.n_out];
  for (int j = 0; j < kPageBlock / kScan; ++j) {
    const int x = blockIdx.x * kPageBlock + j * kScan + threadIdx.x;
    const bool f = is_free(a, x);
    int total;
    const int rank = before + block_scan(f, part, total);
    before += total;
    const bool give = f && rank < wanted;
    if (give) {
      int lo = 0, hi = a.n_out;  // the last row with row_at <= rank
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.row_at[mid] <= rank) lo = mid; else hi = mid;
      }
      const ForkRow r = fork_row(a, lo);
      const int slot = r.want - (a.row_at[lo + 1] - a.row_at[lo]) + rank - a.row_at[lo];
      a.table_out[(int64_t)lo * a.width + slot] = x;
    }
    if (a.refs && x < a.n_pages) a.refs[x] = a.used[x] + (a.held ? a.held[x] : 0) + give;
  }
  if (blockIdx.x + 1 == gridDim.x && before < wanted) {
    for (int i = threadIdx.x; i < a.n_out; i += kScan) {
      const ForkRow r = fork_row(a, i);
      const bool copy = r.part && r.want - (a.row_at[i + 1] - a.row_at[i]) == r.full;
      if (copy && a.row_at[i] >= before) a.lens_out[i] = r.full * a.size;
    }
    if (threadIdx.x == 0) report(a.diag, OPATTR_F_LIMIT, wanted - before);
  }
}

__global__ __launch_bounds__(256) void k_fork_copy(PagesArgs a) {
  const int i = blockIdx.x;
  const ForkRow r = fork_row(a, i);
  if (!r.part || r.want - (a.row_at[i + 1] - a.row_at[i]) != r.full) return;
  const int x = a.table[(int64_t)r.parent * a.width + r.full];
  const int y = a.table_out[(int64_t)i * a.width + r.full];
  if (x < 0 || x >= a.n_pages || y < 0) return;
  for (int l = blockIdx.y; l < a.n_planes; l += gridDim.y) copy_page(a, l, x, y);
}

void run_fork(const PagesArgs &a, hipStream_t s) {
  const int blocks = (a.n_pages + kPageBlock - 1) / kPageBlock;
  if (a.n_pages > 0)
    hipLaunchKernelGGL(k_pages_zero, dim3((a.n_pages + 255) / 256), dim3(256), 0, s, a.used,
                       a.n_pages);
  if (a.n_out > 0) hipLaunchKernelGGL(k_fork_keep, dim3(a.n_out), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_fork_count, dim3(blocks + 1), dim3(kScan), 0, s, a);
  hipLaunchKernelGGL(k_fork_give, dim3(blocks > 0 ? blocks : 1), dim3(kScan), 0, s, a);
  if (a.n_out > 0 && a.n_planes > 0 && a.n_pages > 0)
    hipLaunchKernelGGL(k_fork_copy, dim3(a.n_out, a.n_planes < 256 ? a.n_planes : 256),
                       dim3(256), 0, s, a);
}

// --------------------------------------------------------------------------
// compact
// --------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_compact_mark(PagesArgs a) {
  const int64_t n = (int64_t)a.n_rows * a.width;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  bool bad = false;
  if (i < n) {
    const int id = a.table[i];
    if (id >= 0 && id < a.n_pages)
      a.used[id] = 1;
    else
      bad = id != -1;
  }
  const int wrong = __popcll(__ballot(bad));
  if (wrong && lane_id() == 0) report(a.diag, OPATTR_F_DATA, wrong);
}

__device__ __forceinline__ bool in_use(const PagesArgs &a, int x) {
  return x < a.n_pages && (a.used[x] != 0 || (a.held && a.held[x] > 0));
}

__global__ __launch_bounds__(kScan) void k_compact_count(PagesArgs a) {
  __shared__ int part[kScan / OPA_WAVE];
  int n = 0;
  for (int j = 0; j < kPageBlock / kScan; ++j)
    n += in_use(a, blockIdx.x * kPageBlock + j * kScan + threadIdx.x);
  n = block_sum(n, part);
  if (threadIdx.x == 0) a.count[blockIdx.x] = n;
}

// m pages are in use. holes[j]: the j-th free page below m; highs[j]: the j-th
// page in use at or above m; there are as many of one as of the other. moved of
// a high page is its j for now.
__global__ __launch_bounds__(kScan) void k_compact_list(PagesArgs a) {
  __shared__ int part[kScan / OPA_WAVE];
  const int blocks = gridDim.x;
  int before = 0, all = 0;
  for (int j = threadIdx.x; j < blocks; j += kScan) {
    const int c = a.count[j];
    all += c;
    if (j < (int)blockIdx.x) before += c;
  }
  const int m = block_sum(all, part);
  before = block_sum(before, part);
  // pages in use below m: the blocks before m's, and the part of that block
  int low = 0;
  const int mb = m / kPageBlock;
  for (int j = threadIdx.x; j < mb; j += kScan) low += a.count[j];
  for (int x = mb * kPageBlock + threadIdx.x; x < m; x += kScan) low += in_use(a, x);
  low = block_sum(low, part);
  for (int j = 0; j < kPageBlock / kScan; ++j) {
    const int x = blockIdx.x * kPageBlock + j * kScan + threadIdx.x;
    const bool u = in_use(a, x);
    int total;
    const int at = before + block_scan(u, part, total);
    before += total;
    if (x >= a.n_pages) continue;
    if (u) {
      a.moved[x] = x < m ? x : at - low;
      if (x >= m) a.highs[at - low] = x;
    } else {
      a.moved[x] = -1;
      if (x < m) a.holes[x - at] = x;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.total[0] = m;
    a.total[1] = m - low;
    if (a.live) *a.live = m;
  }
}

// Page moves, then entries of the table and of `moved` of the high pages.
__global__ __launch_bounds__(256) void k_compact_move(PagesArgs a) {
  const int m = a.total[0], n = a.total[1];
  const int64_t jobs = (int64_t)n * a.n_planes;
  for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
    const int at = (int)(j / a.n_planes), plane = (int)(j - (int64_t)at * a.n_planes);
    copy_page(a, plane, a.highs[at], a.holes[at]);
  }
  const int64_t entries = (int64_t)a.n_rows * a.width, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += step) {
    const int id = a.table[i];
    int to = -1;
    if (id >= 0 && id < a.n_pages) {
      to = id;
      if (id >= m) {  // its place in `highs`
        int lo = 0, hi = n;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (a.highs[mid] <= id) lo = mid; else hi = mid;
        }
        to = a.holes[lo];
      }
    }
    a.table_out[i] = to;
  }
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < n; j += step)
    a.moved[a.highs[j]] = a.holes[j];
}

void run_compact(const PagesArgs &a, hipStream_t s) {
  const int blocks = (a.n_pages + kPageBlock - 1) / kPageBlock;
  const int64_t entries = (int64_t)a.n_rows * a.width;
  if (a.n_pages > 0)
    hipLaunchKernelGGL(k_pages_zero, dim3((a.n_pages + 255) / 256), dim3(256), 0, s, a.used,
                       a.n_pages);
  if (entries > 0)
    hipLaunchKernelGGL(k_compact_mark, dim3((uint32_t)((entries + 255) / 256)), dim3(256), 0, s,
                       a);
  if (a.n_pages > 0)
    hipLaunchKernelGGL(k_compact_count, dim3(blocks), dim3(kScan), 0, s, a);
  hipLaunchKernelGGL(k_compact_list, dim3(blocks > 0 ? blocks : 1), dim3(kScan), 0, s, a);
  hipLaunchKernelGGL(k_compact_move, dim3(2048), dim3(256), 0, s, a);
}

}  // namespace opa
