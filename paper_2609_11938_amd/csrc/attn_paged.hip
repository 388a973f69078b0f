// Attention of one new token a sequence over a paged cache (opattr_attn_paged).
//
// A block takes a share of one sequence's tokens for one key head, all the
// query heads that read it (at most 16: the columns of a 16x16x32 product),
// and its waves take tiles of 32 tokens in turn. Shares are equal but for a
// sequence's last, of a size that makes about kBlocks blocks of all the work;
// where a sequence has more than one, a second launch joins them in order.
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kPagedWaves = 4;
constexpr int kTile = 32;        // tokens a wave takes at a time
constexpr int kMinShare = 256;   // tokens of the smallest share
constexpr int kBlocks = 1024;

// Tokens of sequence b, as many as its table can name.
__device__ __forceinline__ int paged_len(const PagedArgs &a, int b) {
  return b < a.n_seqs ? clamp_to(a.lens[b], 0, a.slots) : 0;
}

// Tokens of a share; by whole waves.
__device__ __forceinline__ int share_size(const PagedArgs &a) {
  int64_t sum = 0;
  for (int base = 0; base < a.n_seqs; base += OPA_WAVE) sum += paged_len(a, base + lane_id());
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
  const int64_t each = (sum * a.n_kv + kBlocks - 1) / kBlocks;
  const int64_t c = (each + kTile * kPagedWaves - 1) / (kTile * kPagedWaves) *
                    (kTile * kPagedWaves);
  return uniform((int)(c < kMinShare ? kMinShare : c));
}

__device__ __forceinline__ int shares_of(int len, int c) { return len > c ? (len + c - 1) / c : 1; }

// Share `item` of all the sequences' shares: its sequence and which of its
// shares it is; false past the last.
__device__ __forceinline__ bool find_share(const PagedArgs &a, int c, int item, int &seq,
                                           int &part) {
  const int lane = lane_id();
  for (int base = 0; base < a.n_seqs; base += OPA_WAVE) {
    const int b = base + lane;
    const int n = b < a.n_seqs ? shares_of(paged_len(a, b), c) : 0;
    int inc = n;
#pragma unroll
    for (int d = 1; d < OPA_WAVE; d <<= 1) {
      const int o = __shfl_up(inc, d);
      if (lane >= d) inc += o;
    }
    const uint64_t m = __ballot(inc > item);
    if (m) {
      const int w = __ffsll((unsigned long long)m) - 1;
      seq = base + w;
      part = uniform(item - __shfl(inc - n, w));
      return true;
    }
    item -= uniform(__shfl(inc, OPA_WAVE - 1));
  }
  return false;
}

// The first share of sequence seq (as find_share counts them).
__device__ __forceinline__ int first_share(const PagedArgs &a, int c, int seq) {
  int sum = 0;
  for (int b = lane_id(); b < seq; b += OPA_WAVE) sum += shares_of(paged_len(a, b), c);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
  return uniform(sum);
}

// Results of a share: [items][n_heads][DP + 2]: values, then m and l.
template <class E, int DP>
__global__ __launch_bounds__(kPagedWaves * OPA_WAVE, 2) void k_attn_paged(PagedArgs a) {
  constexpr int KS = DP / 32, DB = DP / 16;
  __shared__ __align__(16) uint16_t tv[kPagedWaves][kTile * DP];
  __shared__ float so[kPagedWaves][16][DP + 1], sm[kPagedWaves][16], sl[kPagedWaves][16];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_kv, item = blockIdx.x / a.n_kv;
  const int share = share_size(a);
  int seq, part;
  if (!find_share(a, share, item, seq, part)) return;
  const int len = uniform(paged_len(a, seq));
  const int t0 = part * share, t1 = len < t0 + share ? len : t0 + share;
  const int32_t *table = a.table + (int64_t)seq * a.width;
  if (threadIdx.x == 0 && part == 0 && hk == 0 && a.lens[seq] != len)
    report(a.diag, OPATTR_F_DATA, 1);

  s16x8 qf[KS];
  {
    const uint16_t *qp = a.q.p + seq * a.q.ts + (int64_t)(hk * a.group + r) * a.q.hs;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = (s16x8)(0);
      if (r < a.group && 32 * s + 8 * g < a.head_dim)
        qf[s] = *reinterpret_cast<const s16x8 *>(qp + 32 * s + 8 * g);
    }
  }
  const float c = a.scale * kLog2e;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = (f32x4)(0.f);
  float m = -INFINITY, l = 0.f;
  const int mask = (1 << a.shift) - 1;
  int bad = 0;
  for (int k0 = t0 + wave * kTile; k0 < t1; k0 += kTile * kPagedWaves) {
    // lane t % 32 finds token k0 + t; -1: none
    int64_t at = -1;
    {
      const int tok = k0 + (lane & 31);
      if (tok < t1) {
        const int page = table[tok >> a.shift];
        if (page >= 0 && page < a.n_pages)
          at = page * a.ps + (tok & mask) * a.ts + (int64_t)hk * a.hs;
        else if (lane < 32)
          ++bad;
      }
    }
    // values, a row's chunks side by side, to LDS
    constexpr int C = DP / 8, N = kTile * C / OPA_WAVE;
    s16x8 vr[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane;
      const int64_t p = __shfl(at, id / C);
      vr[i] = (s16x8)(0);
      if (p >= 0 && (id % C) * 8 < a.head_dim)
        vr[i] = *reinterpret_cast<const s16x8 *>(a.v + p + (id % C) * 8);
    }
    f32x4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t p = __shfl(at, 16 * u + r);
      x[u] = (f32x4)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        s16x8 kf = (s16x8)(0);
        if (p >= 0 && 32 * s + 8 * g < a.head_dim)
          kf = *reinterpret_cast<const s16x8 *>(a.k + p + 32 * s + 8 * g);
        x[u] = E::mfma16(kf, qf[s], x[u]);
      }
    }
    const uint64_t there = __ballot(at >= 0);  // tokens in both halves of the wave
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane, row = id / C;
      *reinterpret_cast<s16x8 *>(&tv[wave][row * DP + (((id % C) ^ swz<DP>(row)) << 3)]) = vr[i];
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool ok = (there >> (16 * u + 4 * g + i)) & 1;
        x[u][i] = ok ? x[u][i] * c : -INFINITY;
        top = fmaxf(top, x[u][i]);
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float mn = fmaxf(m, top);
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float old = exp2_fast(m - ref);
    m = mn;
    float sum = 0.f;
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float p0 = exp2_fast(x[u][2 * i] - ref + E::kShift);
        const float p1 = exp2_fast(x[u][2 * i + 1] - ref + E::kShift);
        sum += p0 + p1;
        w[2 * u + i] = E::pack(p0, p1);
      }
    l = l * old + sum;
    const s16x8 pf = __builtin_bit_cast(s16x8, w);
    // the tile's rows were written by this wave
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      typedef s16x4 __attribute__((address_space(3))) * lds4;
      const int i = lane & 15, row = 4 * g + (i >> 2), col = 16 * d + 4 * (i & 3);
      const uint16_t *p0 = &tv[wave][row * DP + (((col >> 3) ^ swz<DP>(row)) << 3) + (col & 4)];
      const uint16_t *p1 = p0 + 16 * DP;  // swz repeats every 16 rows
      const s16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p0);
      const s16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p1);
      const s16x8 vf = __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[d][e] *= old;
      o[d] = E::mfma16(vf, pf, o[d]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  if (hk == 0 && bad) report(a.diag, OPATTR_F_DATA, bad);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) so[wave][r][16 * d + 4 * g + e] = o[d][e];
  if (g == 0) {
    sm[wave][r] = m;
    sl[wave][r] = l;
  }
  __syncthreads();
  const bool whole = shares_of(len, share) == 1;
  for (int i = threadIdx.x; i < a.group * DP; i += kPagedWaves * OPA_WAVE) {
    const int row = i / DP, d = i % DP, head = hk * a.group + row;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, sm[w][row]);
    const float ref = top == -INFINITY ? 0.f : top;
    float v = 0.f, ls = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      const float f = exp2_fast(sm[w][row] - ref);
      v = fmaf(so[w][row][d], f, v);
      ls = fmaf(sl[w][row], f, ls);
    }
    if (whole) {
      const float y = ls == 0.f ? 0.f : v / ls;
      if (d < a.head_dim)
        a.out.p[seq * a.out.ts + (int64_t)head * a.out.hs + d] = (uint16_t)E::pack(y, y);
      if (d == 0 && a.lse)
        a.lse[(int64_t)head * a.n_seqs + seq] =
            ls == 0.f ? -INFINITY : (top + log2f(ls) - E::kShift) * kLn2;
    } else {
      float *p = a.part + ((int64_t)item * a.n_heads + head) * (DP + 2);
      p[d] = v;
      if (d == 0) {
        p[DP] = top;
        p[DP + 1] = ls;
      }
    }
  }
}

// A block a sequence and key head: its shares joined in order.
template <class E, int DP>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  const int hk = blockIdx.x % a.n_kv, seq = blockIdx.x / a.n_kv;
  const int share = share_size(a);
  const int n = shares_of(uniform(paged_len(a, seq)), share);
  if (n == 1) return;
  const int first = first_share(a, share, seq);
  for (int i = threadIdx.x; i < a.group * DP; i += 256) {
    const int row = i / DP, d = i % DP, head = hk * a.group + row;
    const int64_t step = (int64_t)a.n_heads * (DP + 2);
    const float *p = a.part + ((int64_t)first * a.n_heads + head) * (DP + 2);
    float top = -INFINITY;
    for (int k = 0; k < n; ++k) top = fmaxf(top, p[k * step + DP]);
    const float ref = top == -INFINITY ? 0.f : top;
    float v = 0.f, ls = 0.f;
    for (int k = 0; k < n; ++k) {
      const float f = exp2_fast(p[k * step + DP] - ref);
      v = fmaf(p[k * step + d], f, v);
      ls = fmaf(p[k * step + DP + 1], f, ls);
    }
    const float y = ls == 0.f ? 0.f : v / ls;
    if (d < a.head_dim)
      a.out.p[seq * a.out.ts + (int64_t)head * a.out.hs + d] = (uint16_t)E::pack(y, y);
    if (d == 0 && a.lse)
      a.lse[(int64_t)head * a.n_seqs + seq] =
          ls == 0.f ? -INFINITY : (top + log2f(ls) - E::kShift) * kLn2;
  }
}

// Shares at most: sum of ceil(len / c) with c >= kMinShare and c >= sum / (kBlocks
// / n_kv).
static int64_t most_items(int n_seqs, int n_kv, int slots) {
  const int64_t a = (int64_t)kBlocks / n_kv + 1 + n_seqs;
  const int64_t b = (int64_t)n_seqs * (slots > kMinShare ? (slots + kMinShare - 1) / kMinShare : 1);
  return a < b ? a : b;
}

size_t paged_workspace(int n_seqs, int n_kv, int n_heads, int slots) {
  if (slots <= kMinShare) return 0;  // no sequence has two shares
  return (size_t)most_items(n_seqs, n_kv, slots) * n_heads * (128 + 2) * sizeof(float);
}

template <class E, int DP>
static void launch(const PagedArgs &a, hipStream_t s) {
  const int64_t items = most_items(a.n_seqs, a.n_kv, a.slots);
  hipLaunchKernelGGL((k_attn_paged<E, DP>), dim3((uint32_t)(items * a.n_kv)),
                     dim3(kPagedWaves * OPA_WAVE), 0, s, a);
  if (a.slots > kMinShare)
    hipLaunchKernelGGL((k_paged_join<E, DP>), dim3((uint32_t)(a.n_seqs * a.n_kv)), dim3(256), 0,
                       s, a);
}

void run_paged(const PagedArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  if (dtype == OPATTR_BF16) {
    if (a.head_dim <= 64)
      launch<BF16, 64>(a, s);
    else
      launch<BF16, 128>(a, s);
  } else {
    if (a.head_dim <= 64)
      launch<F16, 64>(a, s);
    else
      launch<F16, 128>(a, s);
  }
}

}  // namespace opa
