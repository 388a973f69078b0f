// Attention of one new token a sequence over a paged cache (opattr_attn_paged).
//
// A block takes a share of one sequence's tokens for one key head, all the
// query heads that read it (at most 16: the columns of a 16x16x32 product),
// and its waves take tiles of 32 tokens in turn. Shares are equal but for a
// sequence's last, of a size that makes about kBlocks blocks of all the work;
// where a sequence has more than one, a second launch joins them in order:
// with a share's sums o_s = sum_j 2^(x_j - m_s) v_j, l_s = sum_j 2^(x_j - m_s),
// out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s, m the largest m_s.
//
// Bound by the cache's bytes, each read once, with the next tile's keys and values in
// registers and its pages a tile further: 2 sequences of 131000 tokens, 32 heads on 8
// of 128: 195 us, 5.5 TB/s; 96 of up to 9001: 117 us, 4.7 TB/s, and 5 us for the join.
// 4 of 150, 12 heads of 64: 5.7 us, the chain of length, table, keys and values.
#include "attn_paged_dev.h"

namespace opa {

// A row's result from its values' sum, its weights' sum and reference.
template <class E>
__device__ __forceinline__ void paged_store(const PagedArgs &a, int seq, int head, int d, f32x4 v,
                                            float top, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const u32x2 w = {E::pack(v[0] * inv, v[1] * inv), E::pack(v[2] * inv, v[3] * inv)};
  if (d < a.head_dim)
    *reinterpret_cast<u32x2 *>(a.out.p + seq * a.out.ts + (int64_t)head * a.out.hs + d) = w;
  if (d == 0 && a.lse)
    a.lse[(int64_t)head * a.n_seqs + seq] =
        l == 0.f ? -INFINITY : (top + log2_sum<E>(l)) * kLn2;
}

// Results of a share: [items][n_heads][DP + 4]: values, then reference and sum of
// the weights. W: through a window with sinks; the tokens that the query sees are
// counted through, and what lies between them is never looked at: 64 sequences of up to
// 32000 tokens, window 4096, 4 sinks, 32 heads on 8 of 128: 89 us, 4.7 TB/s of the 418 MB
// that are seen, and 4 us for the join; without a window 234 us.
template <class E, int DP, bool W>
__global__ __launch_bounds__(kPagedWaves * OPA_WAVE, 2) void k_attn_paged(PagedArgs a) {
  constexpr int KS = DP / 32, DB = DP / 16, C = DP / 8, N = kTile * C / OPA_WAVE;
  // each wave's tile of values; at the end the waves' sums
  __shared__ __align__(16) union {
    uint16_t v[kPagedWaves][kTile * DP];
    float o[kPagedWaves][16][DP + 4];
  } t;
  __shared__ float sm[kPagedWaves][16], sl[kPagedWaves][16];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_kv, item = blockIdx.x / a.n_kv;
  Share s;
  if (!find_share(a, item, s)) return;
  if (hk == 0) note_shares(a, s);
  const int seq = s.seq, len = s.len;
  const int t0 = s.part * s.size, t1 = len < t0 + s.size ? len : t0 + s.size;
  const int32_t *table = a.table + (int64_t)seq * a.width;
  const int tokens = W ? uniform(paged_tokens(a, seq)) : len, skip = tokens - len;
  if (a.diag && threadIdx.x == 0 && s.part == 0 && hk == 0 && a.lens[seq] != tokens)
    report(a.diag, OPATTR_F_DATA, 1);

  const uint16_t *qrow = a.q.p + seq * a.q.ts + (int64_t)hk * a.group * a.q.hs;
  s16x8 qf[KS];
#pragma unroll
  for (int e = 0; e < KS; ++e) {
    qf[e] = (s16x8)(0);
    if (r < a.group && 32 * e + 8 * g < a.head_dim)
      qf[e] = *reinterpret_cast<const s16x8 *>(qrow + r * a.q.hs + 32 * e + 8 * g);
  }
  const float c = a.scale * kLog2e;
  const int mask = (1 << a.shift) - 1, last = a.head_dim / 8 - 1;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = (f32x4)(0.f);
  float m = -INFINITY, l = 0.f;
  int bad = 0;

  // The page of token k0 + lane % 32 (kNone past the share's last), and where the
  // token lies; -1: nowhere. The page is only looked at a tile later: its load
  // comes after that tile's and would be waited for with them.
  constexpr int kNone = INT_MIN;
  const auto page_of = [&](int k0) __attribute__((always_inline)) {
    const int tok = k0 + (lane & 31);
    return tok < t1 ? table[(W && tok >= a.sinks ? tok + skip : tok) >> a.shift] : kNone;
  };
  const auto place = [&](int page, int k0) __attribute__((always_inline)) {
    const bool ok = page >= 0 && page < a.n_pages;
    bad += page != kNone && !ok && lane < 32;
    const int tok = k0 + (lane & 31);
    const int64_t at = page * a.ps + ((W && tok >= a.sinks ? tok + skip : tok) & mask) * a.ts +
                       (int64_t)hk * a.hs;
    return ok ? at : (int64_t)-1;
  };
  // A tile's values (a row's chunks side by side) and keys (as A operands).
  // Tokens that are not there read the query instead, chunks past head_dim the
  // last one; neither is used.
  s16x8 vr[N], kr[2][KS];
  const auto load = [&](int64_t at) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane, ch = id % C < last ? id % C : last;
      const int64_t p = __shfl(at, id / C);
      vr[i] = *reinterpret_cast<const s16x8 *>((p >= 0 ? a.v + p : qrow) + ch * 8);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t p = __shfl(at, 16 * u + r);
      const uint16_t *kp = p >= 0 ? a.k + p : qrow;
#pragma unroll
      for (int e = 0; e < KS; ++e) {
        const int ch = 4 * e + g < last ? 4 * e + g : last;
        kr[u][e] = *reinterpret_cast<const s16x8 *>(kp + ch * 8);
      }
    }
  };

  int k0 = t0 + wave * kTile;
  int64_t at = -1;
  int next = kNone;
  if (k0 < t1) {
    at = place(page_of(k0), k0);
    load(at);
    next = page_of(k0 + kTile * kPagedWaves);
  }
  for (; k0 < t1; k0 += kTile * kPagedWaves) {
    const uint64_t there = __ballot(at >= 0);  // the tokens, in both halves
    if (there != ~0ull) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (!((there >> ((i * OPA_WAVE + lane) / C)) & 1)) vr[i] = (s16x8)(0);
    }
    if (a.head_dim < DP) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((i * OPA_WAVE + lane) % C > last) vr[i] = (s16x8)(0);
#pragma unroll
      for (int e = 0; e < KS; ++e)
        if (4 * e + g > last) kr[0][e] = kr[1][e] = (s16x8)(0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane, row = id / C;
      *reinterpret_cast<s16x8 *>(&t.v[wave][row * DP + (((id % C) ^ swz<DP>(row)) << 3)]) = vr[i];
    }
    f32x4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x[u] = (f32x4)(0.f);
#pragma unroll
      for (int e = 0; e < KS; ++e) x[u] = E::mfma16(kr[u][e], qf[e], x[u]);
    }
    // the next tile's loads, before this one's softmax; places one tile further
    if (k0 + kTile * kPagedWaves < t1) {
      at = place(next, k0 + kTile * kPagedWaves);
      load(at);
      next = page_of(k0 + 2 * kTile * kPagedWaves);
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
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      typedef s16x4 __attribute__((address_space(3))) * lds4;
      const int i = lane & 15, row = 4 * g + (i >> 2), col = 16 * d + 4 * (i & 3);
      const uint16_t *p0 = &t.v[wave][row * DP + (((col >> 3) ^ swz<DP>(row)) << 3) + (col & 4)];
      const uint16_t *p1 = p0 + 16 * DP;  // swz repeats every 16 rows
      const s16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p0);
      const s16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p1);
      const s16x8 vf = __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[d][e] *= old;
      o[d] = E::mfma16(vf, pf, o[d]);
    }
  }
  if (hk == 0 && bad) report(a.diag, OPATTR_F_DATA, bad);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  __syncthreads();
#pragma unroll
  for (int d = 0; d < DB; ++d)
    *reinterpret_cast<f32x4 *>(&t.o[wave][r][16 * d + 4 * g]) = o[d];
  if (g == 0) {
    sm[wave][r] = m;
    sl[wave][r] = l;
  }
  __syncthreads();
  const bool whole = shares_of(len, s.size) == 1;
  for (int i = threadIdx.x; i < a.group * (DP / 4); i += kPagedWaves * OPA_WAVE) {
    const int row = i / (DP / 4), d = i % (DP / 4) * 4, head = hk * a.group + row;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) top = fmaxf(top, sm[w][row]);
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 v = (f32x4)(0.f);
    float ls = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      const float f = exp2_fast(sm[w][row] - ref);
      v += *reinterpret_cast<const f32x4 *>(&t.o[w][row][d]) * f;
      ls = fmaf(sl[w][row], f, ls);
    }
    if (whole) {
      paged_store<E>(a, seq, head, d, v, top, ls);
    } else {
      float *p = a.part + ((int64_t)item * a.n_heads + head) * (DP + 4);
      *reinterpret_cast<f32x4 *>(p + d) = v;
      if (d == 0) *reinterpret_cast<f32x4 *>(p + DP) = f32x4{top, ls, 0.f, 0.f};
    }
  }
}

// A block a sequence and head: its shares joined. The weights' factors first,
// then the shares in kJoin interleaved runs, each added in order, and the runs
// in order.
constexpr int kJoin = 8;
template <class E, int DP>
__global__ __launch_bounds__(kJoin * DP / 4) void k_paged_join(PagedArgs a) {
  constexpr int kThreads = kJoin * DP / 4;
  __shared__ float f[kBlocks + 64];  // sized for the most shares of a sequence
  __shared__ __align__(16) f32x4 sums[kJoin][DP / 4];
  __shared__ float wave_top[kThreads / OPA_WAVE], run_l[kJoin];
  const int head = blockIdx.x % a.n_heads, seq = blockIdx.x / a.n_heads;
  const int2 mine = *reinterpret_cast<const int2 *>(a.shares + 2 * seq);
  const int n = mine.y;
  if (n == 1) return;
  const int64_t step = (int64_t)a.n_heads * (DP + 4);
  const float *p = a.part + ((int64_t)mine.x * a.n_heads + head) * (DP + 4);
  float top = -INFINITY;
  for (int k = threadIdx.x; k < n; k += kThreads) {
    f[k] = p[k * step + DP];
    top = fmaxf(top, f[k]);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane_id() == 0) wave_top[wave_id()] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / OPA_WAVE; ++w) top = fmaxf(top, wave_top[w]);
  const float ref = top == -INFINITY ? 0.f : top;
  const int run = threadIdx.x / (DP / 4), d = threadIdx.x % (DP / 4) * 4;
  f32x4 v = (f32x4)(0.f);
  float l = 0.f;
#pragma unroll 4
  for (int k = run; k < n; k += kJoin) {
    const float w = exp2_fast(f[k] - ref);
    v += *reinterpret_cast<const f32x4 *>(p + k * step + d) * w;
    l = fmaf(p[k * step + DP + 1], w, l);
  }
  sums[run][d / 4] = v;
  if (d == 0) run_l[run] = l;
  __syncthreads();
  if (run) return;
#pragma unroll
  for (int k = 1; k < kJoin; ++k) {
    v += sums[k][d / 4];
    l += run_l[k];
  }
  paged_store<E>(a, seq, head, d, v, top, l);
}

static size_t parts(int n_seqs, int n_kv, int n_heads, int most, int blocks) {
  if (most <= kMinShare) return 0;  // no sequence has two shares
  return (size_t)most_items(n_seqs, n_kv, most, blocks) * n_heads * (128 + 4) * sizeof(float);
}

size_t paged_parts(int n_seqs, int n_kv, int n_heads, int most) {
  return parts(n_seqs, n_kv, n_heads, most, kBlocks);
}
size_t scaled_parts(int n_seqs, int n_kv, int n_heads, int most) {
  return parts(n_seqs, n_kv, n_heads, most, kScaledBlocks);
}

template <class E, int DP>
static void launch(const PagedArgs &a, hipStream_t s) {
  const int64_t items = most_items(a.n_seqs, a.n_kv, a.most, kBlocks);
  const dim3 grid((uint32_t)(items * a.n_kv)), block(kPagedWaves * OPA_WAVE);
  if (a.window)
    hipLaunchKernelGGL((k_attn_paged<E, DP, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_attn_paged<E, DP, false>), grid, block, 0, s, a);
  if (a.most > kMinShare)
    hipLaunchKernelGGL((k_paged_join<E, DP>), dim3((uint32_t)(a.n_seqs * a.n_heads)),
                       dim3(kJoin * DP / 4), 0, s, a);
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
