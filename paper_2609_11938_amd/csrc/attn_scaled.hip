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
// e = the least exponent with max |x| <= 448 2^e: with max |x| = f 2^x, f in [1/2, 1),
// x - 9 if f <= 7/8 (448 = 7/8 2^9), else x - 8. The maximum is of the values' own bits,
// whose order is that of the magnitudes. One wave sees a whole block, so its scale needs
// no second launch, no atomic and no memory; a block's rows are read once, kept in
// registers until the scale is known, and written.
//
// Bound by the bytes: 55000 tokens of 8 heads of 128 in bfloat16, blocks of 16, 341 MB
// read and written: 69 us, 4.9 TB/s, as a large copy has; in float16 79 us, of blocks of
// 64 tokens 72 us. A wave finds its sequence, its page and its old scale before its
// rows' maximum: one token for each of 96 sequences 5 us, for 4 of them 3 us.
constexpr int kAppendWaves = 4;

// The largest magnitude below `most` of 8 values, as their type's bits, and `top`.
__device__ __forceinline__ uint32_t largest(const u32x4 &x, uint32_t most, uint32_t top) {
  uint32_t m = top;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
    if (lo < most && lo > m) m = lo;
    if (hi < most && hi > m) m = hi;
  }
  return m;
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

// kHeld: pieces of 8 values that a lane keeps from their first read; what a block has
// beyond is read again. 4 where a block has no more, 16 else: with 16 for blocks of 16
// tokens of 128 the 55000 take 92 us and not 69 (86 and not 79 in float16), as fewer
// waves fit; with 4 for blocks of 32 they take 79 us and not 70, of 64 92 us and not 72.
template <class E, int kHeld>
__global__ __launch_bounds__(kAppendWaves * OPA_WAVE) void k_append_scaled(AppendScaledArgs a) {
  const int lane = lane_id();
  if (blockIdx.x == 0) {
    check_spans(a.cu, a.n_seqs, a.n_new, a.diag, kAppendWaves * OPA_WAVE);
    int bad = 0;  // tokens before 0 or past the table
    for (int b = threadIdx.x; b < a.n_seqs; b += kAppendWaves * OPA_WAVE) {
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
  // pieces of 8 values, a row's side by side on 2^ls lanes, rows `apart` on in each pass
  const int per = a.head_dim / 8, ls = per > 8 ? 4 : per > 4 ? 3 : per > 2 ? 2 : 1;
  const int n = past - from, apart = OPA_WAVE >> ls, t = lane >> ls;
  const int col = (lane & ((1 << ls) - 1)) * 8;
  const int rows = col < a.head_dim ? n : 0;  // this lane's: none where a row has no piece
  const uint16_t *src = x.p + (int64_t)(row + t) * x.ts + (int64_t)head * x.hs + col;
  u32x4 held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    held[j] = (u32x4)(0u);
    if (j * apart < n && t + j * apart < rows)
      held[j] = *reinterpret_cast<const u32x4 *>(src + j * apart * x.ts);
  }
  const int page = a.table[(int64_t)seq * a.width + (begin >> a.shift)];
  if (page < 0 || page >= a.n_pages) {
    if (lane == 0 && which == 0 && head == 0) report(a.diag, OPATTR_F_DATA, n);
    return;
  }
  const int slot = begin & ((1 << a.shift) - 1);
  uint8_t *to = (which ? a.v : a.k) + page * a.ps + (slot + t) * a.ts + (int64_t)head * a.hs + col;
  uint8_t *scale = (which ? a.v_scale : a.k_scale) + page * a.sps +
                   (slot >> a.block_shift) * a.sbs + (int64_t)head * a.shs;
  const int had = kept > 0 ? *scale : 0;
  // the largest finite magnitude, as the type's bits
  constexpr uint32_t kInf = std::is_same<E, BF16>::value ? 0x7f80u : 0x7c00u;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) top = largest(held[j], kInf, top);
  for (int i = kHeld * apart; i < n; i += apart)
    if (t + i < rows) top = largest(*reinterpret_cast<const u32x4 *>(src + i * x.ts), kInf, top);
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
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (j * apart < n && t + j * apart < rows)
      *reinterpret_cast<u32x2 *>(put + j * apart * a.ts) = codes_of<E>(held[j], by);
  for (int i = kHeld * apart; i < n; i += apart)
    if (t + i < rows)
      *reinterpret_cast<u32x2 *>(put + i * a.ts) =
          codes_of<E>(*reinterpret_cast<const u32x4 *>(src + i * x.ts), by);
  if (kept > 0 && e > had) {
    // below 2^-126 everything has become 0 long before
    const float down = ldexpf(1.f, had - e > -126 ? had - e : -126);
    for (int i = 0; i < kept; i += apart) {
      if (t + i >= kept || col >= a.head_dim) continue;
      u32x2 *p = reinterpret_cast<u32x2 *>(to + i * a.ts);
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
  const dim3 block(kAppendWaves * OPA_WAVE);
  // rows that the lanes take at once: 4 of 128 values, 8 of 64
  const int at_once = a.head_dim > 64 ? 4 : a.head_dim > 32 ? 8 : a.head_dim > 16 ? 16 : 32;
  const bool few = 1 << a.block_shift <= 4 * at_once;
  if (dtype == OPATTR_BF16 && few)
    hipLaunchKernelGGL((k_append_scaled<BF16, 4>), grid, block, 0, s, a);
  else if (dtype == OPATTR_BF16)
    hipLaunchKernelGGL((k_append_scaled<BF16, 16>), grid, block, 0, s, a);
  else if (few)
    hipLaunchKernelGGL((k_append_scaled<F16, 4>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_append_scaled<F16, 16>), grid, block, 0, s, a);
}

// --------------------------------------------------------------------------
// attention
// --------------------------------------------------------------------------
// The weights that meet the codes are 2^((x_j - m) + (e_j - n)), e_j the value's exponent and
// n a whole number near the largest x_j + e_j so far, less m; those of the sum are
// 2^(x_j - m) as elsewhere. So no scale, however large or small, takes a weight past the 16
// bits of its product, and exponents are added to differences of scores, never to
// scores, whose size would round them:
// out = 2^n sum_j 2^((x_j - m) + (e_j - n)) c_j / sum_j 2^(x_j - m).
//
// Bound by the cache's bytes, half of those of 16 bits: 2 sequences of 131000 tokens, 32
// heads on 8 of 128: 108 us, 537 MB at 5.0 TB/s, and 6 us to join the shares; 96 of up to
// 9001, 275 MB: 65 us, 4.2 TB/s, and 5 us; 64 of up to 32000 through a window of 4096 with 4
// sinks, 210 MB: 51 us, 4.1 TB/s, and 4 us (127 and 6 without a window). At half the bytes a
// tile's conversions, softmax and products are no longer hidden by themselves, so the work
// is what the loop looks after: codes become 16-bit values only as operands, an exponent is
// added and not multiplied, a run's addresses and exponents are scalars.

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

// A row's result from its values' sum, of 2^n, and its weights' sum and reference.
template <class E>
__device__ __forceinline__ void scaled_store(const PagedArgs &a, int seq, int head, int d, f32x4 v,
                                             float n, float top, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int by = (int)n;
  const u32x2 w = {E::pack(ldexpf(v[0] * inv, by), ldexpf(v[1] * inv, by)),
                   E::pack(ldexpf(v[2] * inv, by), ldexpf(v[3] * inv, by))};
  if (d < a.head_dim)
    *reinterpret_cast<u32x2 *>(a.out.p + seq * a.out.ts + (int64_t)head * a.out.hs + d) = w;
  if (d == 0 && a.lse)
    a.lse[(int64_t)head * a.n_seqs + seq] =
        l == 0.f ? -INFINITY : (top + log2_sum<E>(l)) * kLn2;
}

// Largest over the lanes that hold the same column: 16 and 32 lanes apart.
__device__ __forceinline__ float column_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return half_max(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}

// Values' codes of a tile in LDS: rows of DP bytes in chunks of 16, chunk c at place
// c ^ code_swz(row), so that the 32 lanes of a read, 16 rows' pieces of one chunk, meet
// each bank once.
template <int DP>
__device__ __forceinline__ int code_swz(int row) {
  return DP == 128 ? ((row >> 1) & 3) | ((row >> 4) & 1) << 2
                   : ((row >> 2) & 1) | ((row >> 4) & 1) << 1;
}

// As k_attn_paged, which see; a share's results end in n, m and l. Keys' codes come to
// registers, values' straight to LDS, from where the transposing read gives a lane the
// codes of one column of the 8 tokens whose weights it holds: they become 16-bit values
// only as operands. The references follow the maxima only when those have passed them
// by 8 binary digits: until then weights are at most 2^(8 + kShift).
//
// R: pages and blocks of 16 tokens or more. A run of 16 then has one page and one scale:
// its addresses are scalars and a lane's own offsets, its exponents scalars. Otherwise
// each token has its own (ts of any size too). 2 sequences of 131000 tokens: 108 us by
// runs, 111 us otherwise; 96 of up to 9001: 65 and 68 us; 4 of 300 through a window of 64,
// heads of 64: 4.5 and 5.7 us.
//
// Three waves a SIMD for heads of 128: the registers of four hold a tile's loads no more
// (2 of 131000: 112 us and not 108; 64 of up to 32000: 131 and not 127; 96 of up to 9001:
// 65 us either way).
//
// Blocks go round the 8 chiplets: a share's key heads lie 8 blocks apart, on one chiplet,
// so that a token's heads, side by side in memory, are read through one cache.
template <class E, int DP, bool R>
__global__ __launch_bounds__(kPagedWaves * OPA_WAVE, DP == 64 ? 4 : 3) void k_attn_scaled(
    ScaledArgs a) {
  constexpr int KS = DP / 32, DB = DP / 16, C = DP / 16, N = kTile * C / OPA_WAVE;
  constexpr int kBytes = kTile * DP;  // a wave's tile
  // the tiles of the waves, two in turn; at the end the waves' sums, two waves' in each
  __shared__ __align__(16) uint8_t v0[kPagedWaves * kBytes], v1[kPagedWaves * kBytes];
  static_assert(kPagedWaves * kBytes == 2 * 16 * DP * 4, "sums of two waves");
  __shared__ __align__(16) int se[R ? 1 : kPagedWaves][kTile];  // a tile's exponents, k and v
  __shared__ float sm[kPagedWaves][16], sv[kPagedWaves][16], sl[kPagedWaves][16];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x / 8 % a.n_kv, item = blockIdx.x % 8 + blockIdx.x / 8 / a.n_kv * 8;
  Share s;
  if (!find_share(a, item, s)) return;
  if (hk == 0) note_shares(a, s);
  const int seq = s.seq, len = s.len;
  const int t0 = s.part * s.size, t1 = len < t0 + s.size ? len : t0 + s.size;
  const int32_t *table = a.table + (int64_t)seq * a.width;
  const int tokens = uniform(paged_tokens(a, seq));
  const Seen seen = seen_of(a, tokens);
  if (a.diag && threadIdx.x == 0 && s.part == 0 && hk == 0 && a.lens[seq] != tokens)
    report(a.diag, OPATTR_F_DATA, 1);

  // Queries as the keys' chunks of 16 come: chunk 4 e + g, its first 8 and its last.
  const uint16_t *qrow = a.q.p + seq * a.q.ts + (int64_t)hk * a.group * a.q.hs;
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
  float m = -INFINITY, l = 0.f;  // the weights' reference, and this lane's sum
  float n = 0.f;                 // the values' reference is 2^n beside it
  int bad = 0;

  constexpr int kNone = INT_MIN;
  const auto token_at = [&](int place) __attribute__((always_inline)) {
    return place >= seen.front ? place + seen.skip : place;
  };
  const auto is_seen = [&](int place) __attribute__((always_inline)) {
    return place < t1 && !(place >= seen.hide && place < seen.shown);
  };
  // This lane's place of a tile: of a token, or the first of its run.
  const int mine = R ? lane & 16 : lane & 31;
  const auto page_of = [&](int k0) __attribute__((always_inline)) {
    return (R ? k0 + mine < t1 : is_seen(k0 + mine)) ? table[token_at(k0 + mine) >> a.shift]
                                                     : kNone;
  };
  // The loads of the tile at k0: keys to registers, values to `to`, the bytes of the
  // exponents. `here`: this lane's token (run) is there; what is not there leaves what
  // was in its place.
  u32x4 kr[KS] = {};
  int ek = 0, ev = 0;  // R: ev's byte is in the lanes' other half
  bool here = false;
  const auto load = [&](uint8_t *to, int page, int k0) __attribute__((always_inline)) {
    here = page >= 0 && page < a.n_pages;
    if constexpr (R) {
      if (page != kNone && !here && lane < 32)
        for (int i = 0; lane == mine && i < 16; ++i) bad += is_seen(k0 + mine + i);
      const int slot = token_at(k0 + mine) & mask;
      if (here) {
        const int64_t es =
            page * a.sps + (slot >> a.block_shift) * a.sbs + (int64_t)hk * a.shs;
        ek = (fresh(lane) < 32 ? a.k_scale : a.v_scale)[es];
      }
      // A lane's part of the addresses, rows 8 i of a run besides where a load has 8:
      // again each time (held over the loop, or kept as addresses, they take registers
      // from the waves that a SIMD has).
      const uint32_t id = fresh(lane), ts = (uint32_t)a.ts;
      const uint32_t k_row = (id & 15) * ts, v_row = id / C * ts;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int p = __builtin_amdgcn_readlane(page, 16 * u);
        if (p < 0 || p >= a.n_pages) continue;
        const int64_t base = p * a.ps + (token_at(k0 + 16 * u) & mask) * a.ts + (int64_t)hk * a.hs;
        const uint8_t *kb = a.k_codes + base, *vb = a.v_codes + base;
        const int vc = (int)(id % C) ^ code_swz<DP>(16 * u + (int)(id / C));
        const uint32_t v_at = v_row + (vc < last ? vc : last) * 16;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)  // (8 rows on, the swizzle is the same)
          __builtin_amdgcn_global_load_lds(
              (const __attribute__((address_space(1))) void *)(vb + i * 8 * a.ts + v_at),
              (__attribute__((address_space(3))) void *)(to + wave * kBytes +
                                                         (u * (N / 2) + i) * OPA_WAVE * 16),
              16, 0, 0);
#pragma unroll
        for (int e = 0; e < KS / 2; ++e) {
          const int ch = 4 * e + (int)(id >> 4);
          kr[u * (KS / 2) + e] = *reinterpret_cast<const u32x4 *>(
              kb + (k_row + (uint32_t)(ch < last ? ch : last) * 16));
        }
      }
    } else {
      bad += page != kNone && !here && lane < 32;
      const int slot = token_at(k0 + mine) & mask;
      const uint8_t *nothing = reinterpret_cast<const uint8_t *>(qrow);
      const int64_t at =
          here ? page * a.ps + slot * a.ts + (int64_t)hk * a.hs : (int64_t)-1;
      const int64_t es = page * a.sps + (slot >> a.block_shift) * a.sbs + (int64_t)hk * a.shs;
      const uint32_t id = fresh(lane);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (i * OPA_WAVE + id) / C, ch = (id % C) ^ code_swz<DP>(row);
        const int64_t p = __shfl(at, row);
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void *)((p >= 0 ? a.v_codes + p : nothing) +
                                                             (ch < last ? ch : last) * 16),
            (__attribute__((address_space(3))) void *)(to + wave * kBytes + i * OPA_WAVE * 16),
            16, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t p = __shfl(at, 16 * u + (id & 15));
        const uint8_t *kp = p >= 0 ? a.k_codes + p : nothing;
#pragma unroll
        for (int e = 0; e < KS / 2; ++e) {
          const int ch = 4 * e + (int)(id >> 4);
          kr[u * (KS / 2) + e] =
              *reinterpret_cast<const u32x4 *>(kp + (ch < last ? ch : last) * 16);
        }
      }
      ek = *(here ? a.k_scale + es : nothing);
      ev = *(here ? a.v_scale + es : nothing);
    }
  };

  // The transposing read: of 16 lanes, lanes 2 k and 2 k + 1 name the two halves of a
  // chunk of row k, and lane i gets column i of the 8 rows, here the tokens of its weights.
  // The chunks differ in bits that the swizzle leaves to an exclusive or.
  const int k = r >> 1, row = k < 4 ? 4 * g + k : 12 + 4 * g + k;
  const int place = row * DP + (code_swz<DP>(row) << 4) + (r & 1) * 8;
  constexpr int kNext = kTile * kPagedWaves;
  int k0 = t0 + wave * kTile, next = kNone;
  // One tile, from `v`, with the next one's loads on their way to `after`.
  const auto step = [&](uint8_t *v, uint8_t *after) __attribute__((always_inline)) {
    // the tokens that are seen, in both halves
    uint64_t there = ~0ull, nan_k = 0, nan_v = 0;
    int xk[2];
    float xv[2];  // R: the exponent of the run's values
    if constexpr (R) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        xk[u] = __builtin_amdgcn_readlane(ek, 16 * u);
        xv[u] = (float)(__builtin_amdgcn_readlane(ek, 16 * u + 32) - 127);
      }
      const uint64_t runs = __ballot(here);
      if (runs != ~0ull || k0 + kTile > t1 || (k0 < seen.shown && k0 + kTile > seen.hide))
        there = __ballot(here && is_seen(k0 + (lane & 31)));
      if (xk[0] == 255 || xk[1] == 255 || xv[0] == 128.f || xv[1] == 128.f) {
        const uint64_t run[2] = {0xffffull, 0xffff0000ull};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (xk[u] == 255) nan_k |= run[u] & there;
          if (xv[u] == 128.f) xv[u] = run[u] & there ? __builtin_nanf("") : 0.f;
        }
      }
    } else {
      there = __ballot(here);
      nan_k = __ballot(here && ek == 255);
      nan_v = __ballot(here && ev == 255);
      if (lane < 32) se[wave][lane] = ek | ev << 8;
    }
    if (there != ~0ull) {  // a weight of 0 times what is not finite is no 0
      const uint32_t id = fresh(lane);
      const u32x4 zero = {(uint32_t)fresh(0), 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (!((there >> ((i * OPA_WAVE + id) / C)) & 1))
          *reinterpret_cast<u32x4 *>(v + wave * kBytes + (i * OPA_WAVE + id) * 16) = zero;
    }
    if (a.head_dim < DP) {
#pragma unroll
      for (int i = 0; i < KS; ++i)
        if (4 * (i % (KS / 2)) + g > last) kr[i] = (u32x4)(0u);
    }
    f32x4 x[2], y[R ? 1 : 2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x[u] = (f32x4)(0.f);
#pragma unroll
      for (int e = 0; e < KS / 2; ++e) {
        const u32x4 w = kr[u * (KS / 2) + e];
        x[u] = E::mfma16(eight_values<E>(w[0], w[1]), qf[2 * e], x[u]);
        x[u] = E::mfma16(eight_values<E>(w[2], w[3]), qf[2 * e + 1], x[u]);
      }
    }
    // the next tile's loads, before this one's softmax; pages one tile further
    if (k0 + kNext < t1) {
      load(after, next, k0 + kNext);
      next = page_of(k0 + 2 * kNext);
    }
    typedef int i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      i32x4 ex;
      if constexpr (!R) ex = *reinterpret_cast<const i32x4 *>(&se[wave][16 * u + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[u][i] = __builtin_amdgcn_ldexpf(x[u][i] * c, (R ? xk[u] : ex[i] & 255) - 127);
        if constexpr (!R) y[u][i] = (float)((ex[i] >> 8) - 127);
      }
    }
    if (there != ~0ull || (nan_k | nan_v)) {
      const int shift = 4 * (fresh(lane) >> 4 & 3);
      const uint32_t seen4 = (uint32_t)there >> shift, nk = (uint32_t)nan_k >> shift,
                     nv = (uint32_t)nan_v >> shift;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bit = 1u << (16 * u + i);
          if (nk & bit) x[u][i] = __builtin_nanf("");
          if (!(seen4 & bit)) x[u][i] = -INFINITY;
          if constexpr (!R) {
            if ((nk | nv) & bit) y[u][i] = __builtin_nanf("");
            if (!(seen4 & bit)) y[u][i] = -INFINITY;
          }
        }
    }
    // a value's exponent
    const auto value_e = [&](int u, int i) __attribute__((always_inline)) {
      return R ? xv[u] : y[R ? 0 : u][i];
    };
    float top = -INFINITY, vtop = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        t = fmaxf(t, x[u][i]);
        if (!R) vtop = fmaxf(vtop, x[u][i] + value_e(u, i));
      }
      top = fmaxf(top, t);
      if (R) vtop = fmaxf(vtop, t + xv[u]);
    }
    if (__any(top > m + 8.f || vtop > m + n + 8.f)) {
      const float mn = fmaxf(m, column_max(top)), both = fmaxf(m + n, column_max(vtop));
      const float to = both == -INFINITY ? 0.f : rintf(both - mn);
      const float by = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
      const float vby = mn == -INFINITY ? 1.f : exp2_fast((m - mn) + (n - to));
      l *= by;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][e] *= vby;
      m = mn;
      n = to;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float p0 = x[u][2 * i] - ref, p1 = x[u][2 * i + 1] - ref;
        sum += exp2_fast(p0 + E::kShift) + exp2_fast(p1 + E::kShift);
        w[2 * u + i] = E::pack(exp2_fast(p0 + (value_e(u, 2 * i) + (E::kShift - n))),
                               exp2_fast(p1 + (value_e(u, 2 * i + 1) + (E::kShift - n))));
      }
    l += sum;
    const s16x8 pf = __builtin_bit_cast(s16x8, w);
    const int at = fresh(place);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      typedef int i32x2 __attribute__((ext_vector_type(2)));
      typedef i32x2 __attribute__((address_space(3))) * lds8;
      const i32x2 codes =
          __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(v + wave * kBytes + (at ^ (d << 4))));
      o[d] = E::mfma16(eight_values<E>((uint32_t)codes[0], (uint32_t)codes[1]), pf, o[d]);
    }
    k0 += kNext;
  };
  if (k0 < t1) {
    load(v0, page_of(k0), k0);
    next = page_of(k0 + kNext);
  }
  while (k0 < t1) {
    wait_loads();
    step(v0, v1);
    if (k0 >= t1) break;
    wait_loads();
    step(v1, v0);
  }
  if (hk == 0 && bad) report(a.diag, OPATTR_F_DATA, bad);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  __syncthreads();
  // a wave's row r of sums, piece p of four values at place p ^ r
  const auto sums = [&](int w, int row, int p) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4 *>(w < 2 ? v0 : v1) +
           (((w & 1) * 16 + row) * (DP / 4) + (p ^ row));
  };
#pragma unroll
  for (int d = 0; d < DB; ++d) *sums(wave, r, 4 * d + g) = o[d];
  if (g == 0) {
    sm[wave][r] = m;
    sv[wave][r] = n;
    sl[wave][r] = l;
  }
  __syncthreads();
  const bool whole = shares_of(len, s.size) == 1;
  for (int i = threadIdx.x; i < a.group * (DP / 4); i += kPagedWaves * OPA_WAVE) {
    const int row = i / (DP / 4), p = i % (DP / 4), head = hk * a.group + row;
    float top = -INFINITY, vtop = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      top = fmaxf(top, sm[w][row]);
      vtop = fmaxf(vtop, sm[w][row] + sv[w][row]);
    }
    const float ref = top == -INFINITY ? 0.f : top;
    const float to = vtop == -INFINITY ? 0.f : rintf(vtop - ref);
    f32x4 v = (f32x4)(0.f);
    float ls = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      v += *sums(w, row, p) * exp2_fast((sm[w][row] - ref) + (sv[w][row] - to));
      ls = fmaf(sl[w][row], exp2_fast(sm[w][row] - ref), ls);
    }
    if (whole) {
      scaled_store<E>(a, seq, head, 4 * p, v, to, top, ls);
    } else {
      float *part = a.part + ((int64_t)item * a.n_heads + head) * (DP + 4);
      *reinterpret_cast<f32x4 *>(part + 4 * p) = v;
      if (p == 0) *reinterpret_cast<f32x4 *>(part + DP) = f32x4{to, top, ls, 0.f};
    }
  }
}

// A block a sequence and head: its shares joined, in kJoin interleaved runs, each
// added in order, and the runs in order.
constexpr int kJoin = 8;
template <class E, int DP>
__global__ __launch_bounds__(kJoin * DP / 4) void k_scaled_join(ScaledArgs a) {
  constexpr int kThreads = kJoin * DP / 4;
  __shared__ float f[kScaledBlocks + 64], fv[kScaledBlocks + 64];  // the most shares of a sequence
  __shared__ __align__(16) f32x4 sums[kJoin][DP / 4];
  __shared__ float wave_top[kThreads / OPA_WAVE][2], run_l[kJoin];
  const int head = blockIdx.x % a.n_heads, seq = blockIdx.x / a.n_heads;
  const int2 mine = *reinterpret_cast<const int2 *>(a.shares + 2 * seq);
  const int n = mine.y;
  if (n == 1) return;
  const int64_t step = (int64_t)a.n_heads * (DP + 4);
  const float *p = a.part + ((int64_t)mine.x * a.n_heads + head) * (DP + 4);
  float top = -INFINITY, vtop = -INFINITY;
  for (int k = threadIdx.x; k < n; k += kThreads) {
    fv[k] = p[k * step + DP];
    f[k] = p[k * step + DP + 1];
    vtop = fmaxf(vtop, f[k] + fv[k]);
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
  const float ref = top == -INFINITY ? 0.f : top;
  const float to = vtop == -INFINITY ? 0.f : rintf(vtop - ref);
  const int run = threadIdx.x / (DP / 4), d = threadIdx.x % (DP / 4) * 4;
  f32x4 v = (f32x4)(0.f);
  float l = 0.f;
#pragma unroll 4
  for (int k = run; k < n; k += kJoin) {
    v += *reinterpret_cast<const f32x4 *>(p + k * step + d) *
         exp2_fast((f[k] - ref) + (fv[k] - to));
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
  scaled_store<E>(a, seq, head, d, v, to, top, l);
}

constexpr int64_t kMaxRunStride = 1 << 26;  // 16 tokens within 2^31 bytes

template <class E, int DP>
static void launch(const ScaledArgs &a, hipStream_t s) {
  const int64_t items = (most_items(a.n_seqs, a.n_kv, a.most, kScaledBlocks) + 7) / 8 * 8;
  const dim3 grid((uint32_t)(items * a.n_kv)), block(kPagedWaves * OPA_WAVE);
  if (a.shift >= 4 && a.block_shift >= 4 && a.ts <= kMaxRunStride)
    hipLaunchKernelGGL((k_attn_scaled<E, DP, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_attn_scaled<E, DP, false>), grid, block, 0, s, a);
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
