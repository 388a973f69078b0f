// The paged cache of 8 bits: new tokens into it (opattr_kv_append_scaled) and the
// attention of one new token a sequence over it (opattr_attn_paged_scaled).
//
// A value is code * 2^e, the code an e4m3 number, e one byte for a block of tokens
// and head. Scales are powers of two: e4m3 keeps its relative precision under them,
// and a code taken over to a larger scale is the same bits of another exponent.
#include "attn_paged_dev.h"

namespace opa {

// --------------------------------------------------------------------------
// append: a wave a block of tokens, head, and keys or values
// --------------------------------------------------------------------------
constexpr int kAppendWaves = 4;
constexpr int kHeldPieces = 8;  // pieces of 8 values that a lane keeps from one read

__device__ __forceinline__ int scale_word(const u32x4 &x, uint32_t most, uint32_t top) {
  uint32_t m = top;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
    if (lo < most && lo > m) m = lo;
    if (hi < most && hi > m) m = hi;
  }
  return (int)m;
}

// 8 values as codes.
template <class E>
__device__ __forceinline__ u32x2 codes_of(const u32x4 &x, float by) {
  u32x2 c = (u32x2)(0u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = E::widen((uint16_t)x[i]) * by, hi = E::widen((uint16_t)(x[i] >> 16)) * by;
    c[i >> 1] = i & 1 ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, (int)c[i >> 1], true)
                      : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, (int)c[i >> 1], false);
  }
  return c;
}

template <class E>
__global__ __launch_bounds__(kAppendWaves * OPA_WAVE) void k_append_scaled(AppendScaledArgs a) {
  const int lane = lane_id();
  if (blockIdx.x == 0) {
    check_spans(a.cu, a.n_seqs, a.n_new, a.diag);
    int bad = 0;  // tokens before 0 or past the table
    for (int b = threadIdx.x; b < a.n_seqs; b += blockDim.x) {
      const int n = span_of(a.cu, b, a.n_new).count;
      const int64_t first = a.lens[b], last = first + n;
      if (a.lens_out) a.lens_out[b] = a.lens[b] + n;
      const int64_t lo = first < 0 ? 0 : first, hi = last > a.slots ? a.slots : last;
      bad += n - (int)(hi > lo ? hi - lo : 0);
    }
    if (bad) report(a.diag, OPATTR_F_DATA, bad);
  }
  const int item = uniform((int)blockIdx.x * kAppendWaves + wave_id());
  const int which = item & 1, head = (item >> 1) % a.n_kv;
  int unit = (item >> 1) / a.n_kv;
  const int size = 1 << a.block_shift;
  // the sequence, its first new row, and where its first new token goes
  int seq = -1, row = 0, lo = 0, hi = 0;
  for (int base = 0; base < a.n_seqs; base += OPA_WAVE) {
    const int b = base + lane < a.n_seqs ? base + lane : a.n_seqs - 1;
    const Span s = span_of(a.cu, b, a.n_new);
    const int64_t first = a.lens[b], last = first + s.count;
    const int from = (int)(first < 0 ? 0 : first > a.slots ? a.slots : first);
    const int past = (int)(last < from ? from : last > a.slots ? a.slots : last);
    const int n = base + lane < a.n_seqs && past > from
                      ? ((past - 1) >> a.block_shift) - (from >> a.block_shift) + 1
                      : 0;
    const int inc = wave_sums(n);
    const uint64_t m = __ballot(inc > unit);
    if (m) {
      const int w = __ffsll((unsigned long long)m) - 1;
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, w); };
      seq = base + w;
      lo = of(from);
      hi = of(past);
      row = of((int)(s.first + (from - first)));
      unit -= of(inc - n);
      break;
    }
    unit -= __builtin_amdgcn_readlane(inc, OPA_WAVE - 1);
  }
  if (seq < 0) return;
  const int begin = ((lo >> a.block_shift) + unit) << a.block_shift;  // the block's first token
  const int from = begin > lo ? begin : lo, past = begin + size < hi ? begin + size : hi;
  const int kept = from - begin;
  row += from - lo;
  const Rows &x = which ? a.vn : a.kn;
  const uint16_t *src = x.p + (int64_t)row * x.ts + (int64_t)head * x.hs;
  const int per = a.head_dim / 8, pieces = (past - from) * per;
  const auto piece = [&](int i) __attribute__((always_inline)) {
    const int t = i / per;
    return *reinterpret_cast<const u32x4 *>(src + t * x.ts + (i - t * per) * 8);
  };
  u32x4 held[kHeldPieces];
#pragma unroll
  for (int j = 0; j < kHeldPieces; ++j)
    if (j * OPA_WAVE + lane < pieces) held[j] = piece(j * OPA_WAVE + lane);
  const int page = a.table[(int64_t)seq * a.width + (begin >> a.shift)];
  if (page < 0 || page >= a.n_pages) {
    if (lane == 0 && which == 0 && head == 0) report(a.diag, OPATTR_F_DATA, past - from);
    return;
  }
  const int slot = begin & ((1 << a.shift) - 1);
  uint8_t *to = (which ? a.v : a.k) + page * a.ps + slot * a.ts + (int64_t)head * a.hs;
  uint8_t *scale = (which ? a.v_scale : a.k_scale) + page * a.sps +
                   (slot >> a.block_shift) * a.sbs + (int64_t)head * a.shs;
  const int had = kept > 0 ? *scale : 0;
  // the largest finite magnitude, as the type's bits
  constexpr uint32_t kInf = std::is_same<E, BF16>::value ? 0x7f80u : 0x7c00u;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kHeldPieces; ++j)
    if (j * OPA_WAVE + lane < pieces) top = scale_word(held[j], kInf, top);
  for (int i = kHeldPieces * OPA_WAVE + lane; i < pieces; i += OPA_WAVE)
    top = scale_word(piece(i), kInf, top);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const float most = E::widen((uint16_t)uniform((int)top));
  int e = 0;  // the exponent and 127
  if (most > 0.f) {  // most = m 2^x with m in [1/2, 1), 448 = 7/8 2^9
    const int x2 = __builtin_amdgcn_frexp_expf(most);
    e = (__builtin_amdgcn_frexp_mantf(most) <= 0.875f ? x2 - 9 : x2 - 8) + 127;
    e = e < 0 ? 0 : e;
  }
  if (had > e) e = had;
  const float by = ldexpf(1.f, 127 - e);
  uint8_t *put = to + kept * a.ts;
  const auto write = [&](int i, const u32x4 &v) __attribute__((always_inline)) {
    const int t = i / per;
    *reinterpret_cast<u32x2 *>(put + t * a.ts + (i - t * per) * 8) = codes_of<E>(v, by);
  };
#pragma unroll
  for (int j = 0; j < kHeldPieces; ++j)
    if (j * OPA_WAVE + lane < pieces) write(j * OPA_WAVE + lane, held[j]);
  for (int i = kHeldPieces * OPA_WAVE + lane; i < pieces; i += OPA_WAVE) write(i, piece(i));
  if (kept > 0 && e > had) {
    // below 2^-126 everything has become 0 long before
    const float down = ldexpf(1.f, had - e > -126 ? had - e : -126);
    for (int i = lane; i < kept * per; i += OPA_WAVE) {
      const int t = i / per;
      u32x2 *p = reinterpret_cast<u32x2 *>(to + t * a.ts + (i - t * per) * 8);
      u32x2 c = *p;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const f32x2 l = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
        const f32x2 h = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(l[0] * down, l[1] * down, 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(h[0] * down, h[1] * down, v, true);
        c[w] = (uint32_t)v;
      }
      *p = c;
    }
  }
  if (lane == 0) *scale = (uint8_t)e;
}

int64_t append_units(int64_t n_new, int n_seqs, int block_shift) {
  const int64_t n = (n_new >> block_shift) + 2 * (int64_t)n_seqs;
  return n < n_new ? n : n_new;
}

void run_append_scaled(const AppendScaledArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  const int64_t waves = append_units(a.n_new, a.n_seqs, a.block_shift) * a.n_kv * 2;
  const dim3 grid((uint32_t)(waves > 0 ? (waves + kAppendWaves - 1) / kAppendWaves : 1));
  if (dtype == OPATTR_BF16)
    hipLaunchKernelGGL(k_append_scaled<BF16>, grid, dim3(kAppendWaves * OPA_WAVE), 0, s, a);
  else
    hipLaunchKernelGGL(k_append_scaled<F16>, grid, dim3(kAppendWaves * OPA_WAVE), 0, s, a);
}

// --------------------------------------------------------------------------
// attention
// --------------------------------------------------------------------------
// The weights that meet the codes are 2^(x_j + e_j - m'), e_j the value's exponent and
// m' the largest x_j + e_j so far; those of the sum are 2^(x_j - m) as elsewhere. So
// no scale, however large or small, takes a weight past the 16 bits of its product:
// out = 2^(m' - m) sum_j 2^(x_j + e_j - m') c_j / sum_j 2^(x_j - m).

// The two codes of half h of a word as 16-bit values (exact).
template <class E>
__device__ __forceinline__ uint32_t two_values(uint32_t w, bool high) {
  if constexpr (std::is_same<E, BF16>::value) {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
  } else {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
  }
}
template <class E>
__device__ __forceinline__ s16x8 eight_values(uint32_t w0, uint32_t w1) {
  const u32x4 v = {two_values<E>(w0, false), two_values<E>(w0, true), two_values<E>(w1, false),
                   two_values<E>(w1, true)};
  return __builtin_bit_cast(s16x8, v);
}

// A row's result from its values' sum and its weights' sum, with their references.
template <class E>
__device__ __forceinline__ void scaled_store(const PagedArgs &a, int seq, int head, int d, f32x4 v,
                                             float vtop, float top, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  // 2^(vtop - top) as a power within one and a whole exponent
  const float by = l == 0.f ? 0.f : vtop - top;
  const float whole = rintf(by), f = exp2_fast(by - whole) * inv;
  const int n = (int)whole;
  const u32x2 w = {E::pack(ldexpf(v[0] * f, n), ldexpf(v[1] * f, n)),
                   E::pack(ldexpf(v[2] * f, n), ldexpf(v[3] * f, n))};
  if (d < a.head_dim)
    *reinterpret_cast<u32x2 *>(a.out.p + seq * a.out.ts + (int64_t)head * a.out.hs + d) = w;
  if (d == 0 && a.lse)
    a.lse[(int64_t)head * a.n_seqs + seq] =
        l == 0.f ? -INFINITY : (top + log2_sum<E>(l)) * kLn2;
}

// As k_attn_paged, which see; a share's results end in m', m and l. W: a window.
template <class E, int DP>
__global__ __launch_bounds__(kPagedWaves * OPA_WAVE, 2) void k_attn_scaled(ScaledArgs a) {
  constexpr int KS = DP / 32, DB = DP / 16, C = DP / 16, N = kTile * C / OPA_WAVE;
  __shared__ __align__(16) union {
    uint16_t v[kPagedWaves][kTile * DP];
    float o[kPagedWaves][16][DP + 4];
  } t;
  __shared__ __align__(16) int se[kPagedWaves][kTile];  // a tile's exponents, k and v
  __shared__ float sm[kPagedWaves][16], sv[kPagedWaves][16], sl[kPagedWaves][16];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % a.n_kv, item = blockIdx.x / a.n_kv;
  Share s;
  if (!find_share(a, item, s)) return;
  const int seq = s.seq, len = s.len;
  const int t0 = s.part * s.size, t1 = len < t0 + s.size ? len : t0 + s.size;
  const int32_t *table = a.table + (int64_t)seq * a.width;
  const int tokens = uniform(paged_tokens(a, seq)), skip = tokens - len;
  if (a.diag && threadIdx.x == 0 && s.part == 0 && hk == 0 && a.lens[seq] != tokens)
    report(a.diag, OPATTR_F_DATA, 1);

  // Queries as the keys' chunks of 16 come: chunk 4 e + g, its first 8 and its last.
  const uint16_t *qrow = a.q.p + seq * a.q.ts + (int64_t)hk * a.group * a.q.hs;
  const uint8_t *nothing = reinterpret_cast<const uint8_t *>(qrow);
  s16x8 qf[KS];
#pragma unroll
  for (int e = 0; e < KS; ++e) {
    const int d = 64 * (e >> 1) + 16 * g + 8 * (e & 1);
    qf[e] = (s16x8)(0);
    if (r < a.group && d < a.head_dim)
      qf[e] = *reinterpret_cast<const s16x8 *>(qrow + r * a.q.hs + d);
  }
  const float c = a.scale * kLog2e;
  const int mask = (1 << a.shift) - 1, last = a.head_dim / 16 - 1;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = (f32x4)(0.f);
  float m = -INFINITY, mv = -INFINITY, l = 0.f;
  int bad = 0;

  constexpr int kNone = INT_MIN;
  const auto token_of = [&](int k0) __attribute__((always_inline)) {
    const int tok = k0 + (lane & 31);
    return tok >= a.sinks ? tok + skip : tok;
  };
  const auto page_of = [&](int k0) __attribute__((always_inline)) {
    return k0 + (lane & 31) < t1 ? table[token_of(k0) >> a.shift] : kNone;
  };
  // Where the token's codes lie (-1: nowhere), and its two exponents' bytes.
  u32x4 vr[N], kr[KS];
  int ek, ev;
  const auto load = [&](int page, int k0) __attribute__((always_inline)) {
    const bool ok = page >= 0 && page < a.n_pages;
    bad += page != kNone && !ok && lane < 32;
    const int slot = token_of(k0) & mask;
    const int64_t to = page * a.ps + slot * a.ts + (int64_t)hk * a.hs;
    const int64_t at = ok ? to : (int64_t)-1;
    const int64_t es =
        page * a.sps + (slot >> a.block_shift) * a.sbs + (int64_t)hk * a.shs;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane, ch = id % C < last ? id % C : last;
      const int64_t p = __shfl(at, id / C);
      vr[i] = *reinterpret_cast<const u32x4 *>((p >= 0 ? a.v_codes + p : nothing) + ch * 16);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t p = __shfl(at, 16 * u + r);
      const uint8_t *kp = p >= 0 ? a.k_codes + p : nothing;
#pragma unroll
      for (int e = 0; e < KS / 2; ++e) {
        const int ch = 4 * e + g < last ? 4 * e + g : last;
        kr[u * (KS / 2) + e] = *reinterpret_cast<const u32x4 *>(kp + ch * 16);
      }
    }
    ek = *(ok ? a.k_scale + es : nothing);
    ev = *(ok ? a.v_scale + es : nothing);
    return at;
  };

  int k0 = t0 + wave * kTile;
  int64_t at = -1;
  int next = kNone;
  if (k0 < t1) {
    at = load(page_of(k0), k0);
    next = page_of(k0 + kTile * kPagedWaves);
  }
  for (; k0 < t1; k0 += kTile * kPagedWaves) {
    const uint64_t there = __ballot(at >= 0);  // the tokens, in both halves
    const uint64_t nan_k = __ballot(ek == 255), nan_v = __ballot(ev == 255);
    if (lane < 32) se[wave][lane] = ek | ev << 8;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * OPA_WAVE + lane, row = id / C, ch = id % C;
      if (!((there >> row) & 1) || ch > last) vr[i] = (u32x4)(0u);
      uint16_t *p = &t.v[wave][row * DP];
      *reinterpret_cast<s16x8 *>(p + (((2 * ch) ^ swz<DP>(row)) << 3)) =
          eight_values<E>(vr[i][0], vr[i][1]);
      *reinterpret_cast<s16x8 *>(p + (((2 * ch + 1) ^ swz<DP>(row)) << 3)) =
          eight_values<E>(vr[i][2], vr[i][3]);
    }
    f32x4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x[u] = (f32x4)(0.f);
#pragma unroll
      for (int e = 0; e < KS / 2; ++e) {
        u32x4 w = kr[u * (KS / 2) + e];
        if (4 * e + g > last) w = (u32x4)(0u);
        x[u] = E::mfma16(eight_values<E>(w[0], w[1]), qf[2 * e], x[u]);
        x[u] = E::mfma16(eight_values<E>(w[2], w[3]), qf[2 * e + 1], x[u]);
      }
    }
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const i32x4 ex[2] = {*reinterpret_cast<const i32x4 *>(&se[wave][4 * g]),
                         *reinterpret_cast<const i32x4 *>(&se[wave][16 + 4 * g])};
    // the next tile's loads, before this one's softmax; pages one tile further
    if (k0 + kTile * kPagedWaves < t1) {
      at = load(next, k0 + kTile * kPagedWaves);
      next = page_of(k0 + 2 * kTile * kPagedWaves);
    }
    float top = -INFINITY, vtop = -INFINITY;
    f32x4 y[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool ok = (there >> (16 * u + 4 * g + i)) & 1;
        x[u][i] = ok ? ldexpf(x[u][i] * c, (ex[u][i] & 255) - 127) : -INFINITY;
        y[u][i] = x[u][i] + (float)((ex[u][i] >> 8) - 127);
      }
    if ((nan_k | nan_v) & there) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = 16 * u + 4 * g + i;
          if ((nan_k & there) >> tok & 1) x[u][i] = y[u][i] = __builtin_nanf("");
          if ((nan_v & there) >> tok & 1) y[u][i] = __builtin_nanf("");
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top = fmaxf(top, x[u][i]);
        vtop = fmaxf(vtop, y[u][i]);
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    vtop = fmaxf(vtop, __shfl_xor(vtop, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    vtop = fmaxf(vtop, __shfl_xor(vtop, 32));
    const float mn = fmaxf(m, top), mvn = fmaxf(mv, vtop);
    const float ref = mn == -INFINITY ? 0.f : mn, vref = mvn == -INFINITY ? 0.f : mvn;
    const float old = exp2_fast(m - ref), vold = exp2_fast(mv - vref);
    m = mn;
    mv = mvn;
    float sum = 0.f;
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sum += exp2_fast(x[u][2 * i] - ref + E::kShift) +
               exp2_fast(x[u][2 * i + 1] - ref + E::kShift);
        w[2 * u + i] = E::pack(exp2_fast(y[u][2 * i] - vref + E::kShift),
                               exp2_fast(y[u][2 * i + 1] - vref + E::kShift));
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
      for (int e = 0; e < 4; ++e) o[d][e] *= vold;
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
    sv[wave][r] = mv;
    sl[wave][r] = l;
  }
  __syncthreads();
  const bool whole = shares_of(len, s.size) == 1;
  for (int i = threadIdx.x; i < a.group * (DP / 4); i += kPagedWaves * OPA_WAVE) {
    const int row = i / (DP / 4), d = i % (DP / 4) * 4, head = hk * a.group + row;
    float top = -INFINITY, vtop = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      top = fmaxf(top, sm[w][row]);
      vtop = fmaxf(vtop, sv[w][row]);
    }
    const float ref = top == -INFINITY ? 0.f : top, vref = vtop == -INFINITY ? 0.f : vtop;
    f32x4 v = (f32x4)(0.f);
    float ls = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      v += *reinterpret_cast<const f32x4 *>(&t.o[w][row][d]) * exp2_fast(sv[w][row] - vref);
      ls = fmaf(sl[w][row], exp2_fast(sm[w][row] - ref), ls);
    }
    if (whole) {
      scaled_store<E>(a, seq, head, d, v, vtop, top, ls);
    } else {
      float *p = a.part + ((int64_t)item * a.n_heads + head) * (DP + 4);
      *reinterpret_cast<f32x4 *>(p + d) = v;
      if (d == 0) *reinterpret_cast<f32x4 *>(p + DP) = f32x4{vtop, top, ls, 0.f};
    }
  }
}

// A block a sequence and head: its shares joined, in kJoin interleaved runs, each
// added in order, and the runs in order.
constexpr int kJoin = 8;
template <class E, int DP>
__global__ __launch_bounds__(kJoin * DP / 4) void k_scaled_join(ScaledArgs a) {
  constexpr int kThreads = kJoin * DP / 4;
  __shared__ float f[kBlocks + 64], fv[kBlocks + 64];  // the most shares of a sequence
  __shared__ __align__(16) f32x4 sums[kJoin][DP / 4];
  __shared__ float wave_top[kThreads / OPA_WAVE][2], run_l[kJoin];
  const int head = blockIdx.x % a.n_heads, seq = blockIdx.x / a.n_heads;
  const Share s = shares_at(a, seq);
  const int n = shares_of(s.len, s.size);
  if (n == 1) return;
  const int64_t step = (int64_t)a.n_heads * (DP + 4);
  const float *p = a.part + ((int64_t)s.first * a.n_heads + head) * (DP + 4);
  float top = -INFINITY, vtop = -INFINITY;
  for (int k = threadIdx.x; k < n; k += kThreads) {
    fv[k] = p[k * step + DP];
    f[k] = p[k * step + DP + 1];
    vtop = fmaxf(vtop, fv[k]);
    top = fmaxf(top, f[k]);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    top = fmaxf(top, __shfl_xor(top, d));
    vtop = fmaxf(vtop, __shfl_xor(vtop, d));
  }
  if (lane_id() == 0) {
    wave_top[wave_id()][0] = top;
    wave_top[wave_id()][1] = vtop;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / OPA_WAVE; ++w) {
    top = fmaxf(top, wave_top[w][0]);
    vtop = fmaxf(vtop, wave_top[w][1]);
  }
  const float ref = top == -INFINITY ? 0.f : top, vref = vtop == -INFINITY ? 0.f : vtop;
  const int run = threadIdx.x / (DP / 4), d = threadIdx.x % (DP / 4) * 4;
  f32x4 v = (f32x4)(0.f);
  float l = 0.f;
#pragma unroll 4
  for (int k = run; k < n; k += kJoin) {
    v += *reinterpret_cast<const f32x4 *>(p + k * step + d) * exp2_fast(fv[k] - vref);
    l = fmaf(p[k * step + DP + 2], exp2_fast(f[k] - ref), l);
  }
  sums[run][d / 4] = v;
  if (d == 0) run_l[run] = l;
  __syncthreads();
  if (run) return;
  l = run_l[0];
#pragma unroll
  for (int k = 1; k < kJoin; ++k) {
    v += sums[k][d / 4];
    l += run_l[k];
  }
  scaled_store<E>(a, seq, head, d, v, vtop, top, l);
}

template <class E, int DP>
static void launch(const ScaledArgs &a, hipStream_t s) {
  const int64_t items = most_items(a.n_seqs, a.n_kv, a.most);
  hipLaunchKernelGGL((k_attn_scaled<E, DP>), dim3((uint32_t)(items * a.n_kv)),
                     dim3(kPagedWaves * OPA_WAVE), 0, s, a);
  if (a.most > kMinShare)
    hipLaunchKernelGGL((k_scaled_join<E, DP>), dim3((uint32_t)(a.n_seqs * a.n_heads)),
                       dim3(kJoin * DP / 4), 0, s, a);
}

void run_paged_scaled(const ScaledArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  if (dtype == OPATTR_BF16)
    a.head_dim <= 64 ? launch<BF16, 64>(a, s) : launch<BF16, 128>(a, s);
  else
    a.head_dim <= 64 ? launch<F16, 64>(a, s) : launch<F16, 128>(a, s);
}

}  // namespace opa
