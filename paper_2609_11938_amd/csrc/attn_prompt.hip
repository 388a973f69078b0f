// Attention over whole prompts (opattr_attn_prompt).
//
// out_i = sum_j w_ij v_j / sum_j w_ij with w_ij = 2^(c (q_i.k_j - m_i)), c = scale
// log2 e, in one pass over the keys: m_i is a reference near the maximum so far, and
// what has been added is rescaled when it moves. A wave holds 32 queries and takes
// tiles of 64 keys, two in LDS: one for the products, one on its way. The scores are
// K Q^T, so that a lane holds the scores of one query: its maximum and sum are the
// lane's own but for one exchange between the halves, and the weights are where the
// second product takes them.
//
// 24 prompts of up to 4099 tokens, 32 heads on 8 of 128: 358 us, 867 TFLOP/s counted
// (what is seen), the matrix units busy 52% of the time; one of 16384, 16 heads on 4:
// 1071 us, 1.03 PFLOP/s. In a wave the phases of a tile follow one another, and two
// waves a SIMD hide little of that: products alone (softmax left out) 680 us, softmax
// 140 and the reads of fragments from LDS 260 add up to the whole. 64 queries a wave,
// with half those reads, leave one wave a SIMD: twice the time. head_dim 72 to 120
// costs nearly what 128 does (24 prompts of 80: 313 us, of 96: 323).
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kWaves = 4;       // waves a block, 32 queries each
constexpr int kRowsQ = 32 * kWaves;
constexpr int kRowsK = 64;      // keys a tile

// (one sequence of 6000, 4 heads, 192 blocks: 107 us with one group, 85 with two;
// 3 of 1500, 16 heads, 608 blocks: 48 and 55; 4 of 128, where there is a tile for
// each group: 6.9 and 7.6)
constexpr int kFewBlocks = 384, kManyKeys = 768;

// G groups of kWaves waves take the key tiles in turn and join their sums at the
// end: the waves that a few rows would leave a compute unit without.
template <class E, int DP, int G>
__global__ __launch_bounds__(G * kWaves * OPA_WAVE, 2) void k_attn_prompt(PromptArgs a) {
  constexpr int KS = DP / 16, DB = DP / 32;
  constexpr int kTile = kRowsK * DP;
  // a group's two tiles of keys, two of values; its sums at the end
  __shared__ __align__(16) uint16_t tk0[G][kTile], tk1[G][kTile], tv0[G][kTile], tv1[G][kTile];
  const int lane = lane_id(), all = uniform(wave_id()), wave = all % kWaves, group = all / kWaves;
  const int r = lane & 31, h = lane >> 5;
  // a block's key head goes by its index modulo the key heads
  int id = blockIdx.x;
  const int hk = id % a.n_kv;
  id /= a.n_kv;
  const int head = hk * a.group + id % a.group;
  if (blockIdx.x == 0) {
    check_spans(a.cu_q, a.n_seqs, a.n_q, a.diag);
    check_spans(a.cu_k, a.n_seqs, a.n_k, a.diag);
  }
  Span sq, sk;
  int part;
  if (!find_tile(a.cu_q, a.n_q, a.cu_k, a.n_k, a.n_seqs, kRowsQ, id / a.group, sq, sk, part))
    return;
  // the sequence's last queries, which see the most keys, first
  const int q0 = ((sq.count + kRowsQ - 1) / kRowsQ - 1 - part) * kRowsQ;
  const int lead = sk.count - sq.count;
  const int qrow = q0 + wave * 32 + r;  // this lane's query
  const bool live = qrow < sq.count;
  const int last = (q0 + kRowsQ < sq.count ? q0 + kRowsQ : sq.count) - 1;
  const int keys = a.causal ? clamp_to(last + lead + 1, 0, sk.count) : sk.count;
  const int tiles = (keys + kRowsK - 1) / kRowsK;
  // keys below `whole` are seen by every query of this wave
  const int whole = a.causal ? clamp_to(q0 + wave * 32 + lead + 1, 0, sk.count) : sk.count;
  const int seen = live ? (a.causal ? clamp_to(qrow + lead + 1, 0, sk.count) : sk.count) : 0;

  // scores in units of 1 / c, c > 0: a negative scale turns the queries round
  const float c = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-120f);
  s16x8 qf[KS];
  {
    const uint16_t *qp = a.q.p + (int64_t)(sq.first + (live ? qrow : 0)) * a.q.ts +
                         (int64_t)head * a.q.hs;
    const s16x8 turn = (s16x8)(a.scale < 0.f ? (short)0x8000 : (short)0);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = (s16x8)(0);
      if (live && 16 * s + 8 * h < a.head_dim)
        qf[s] = *reinterpret_cast<const s16x8 *>(qp + 16 * s + 8 * h) ^ turn;
    }
  }
  const uint16_t *kp = a.k.p + (int64_t)sk.first * a.k.ts + (int64_t)hk * a.k.hs;
  const uint16_t *vp = a.v.p + (int64_t)sk.first * a.v.ts + (int64_t)hk * a.v.hs;
  f32x16 o[DB];
  float m, l;  // the reference of the weights, in scores, and this half's sum

  const int nat0 = nat_place<DP>(), tr0 = tr_place<DP>();

  const auto load = [&](uint16_t *k, uint16_t *v, int k0) __attribute__((always_inline)) {
    tile_load<DP, kRowsK, kWaves>(k, kp + k0 * a.k.ts, a.k.ts, sk.count - k0, a.head_dim, wave);
    tile_load<DP, kRowsK, kWaves>(v, vp + k0 * a.v.ts, a.v.ts, sk.count - k0, a.head_dim, wave);
  };
  const auto step = [&](auto careful, const uint16_t *k, const uint16_t *v,
                        int k0) __attribute__((always_inline)) {
    const int nat = fresh(nat0), tr = fresh(tr0);
    f32x16 x[2];
    x[0] = x[1] = (f32x16)(0.f);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        x[kb] = E::mfma(nat_frag<DP>(k, nat, 32 * kb, s), qf[s], x[kb]);
    const bool cut = k0 + kRowsK > whole;
    if (cut) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (k0 + 32 * kb + 8 * (i >> 2) + 4 * h + (i & 3) >= seen) x[kb][i] = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
    // The weights' reference follows the maximum only when that has passed it by
    // 8 binary digits: until then they are at most 2^(8 + kShift), and sums and
    // outputs need no new scale.
    if (__any(top > m + 8.f / c)) {
      const float to = half_max(top);
      const float by = to == -INFINITY ? 1.f : exp2_fast((m - to) * c);
      m = to;
      l *= by;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= by;
    }
    const float ref = E::kShift - (m == -INFINITY ? 0.f : m * c);
    s16x8 pf[4];
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = exp2_fast(fmaf(x[kb][8 * s + 2 * i], c, ref));
          const float p1 = exp2_fast(fmaf(x[kb][8 * s + 2 * i + 1], c, ref));
          sum += p0 + p1;
          w[i] = E::pack(p0, p1);
        }
        pf[2 * kb + s] = __builtin_bit_cast(s16x8, w);
      }
    l += sum;
    if (decltype(careful)::value && cut) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll 1
        for (int n = 0; n < 16; ++n) {  // slot n % 8 of half n / 8
          u32x4 only;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            only[i] = h == n >> 3 && i == (n & 7) >> 1 ? (n & 1 ? 0xffff0000u : 0xffffu) : 0u;
          const bool sees = k0 + 16 * s + 8 * ((n & 7) >> 2) + 4 * (n >> 3) + (n & 3) < seen;
          const s16x8 pn = __builtin_bit_cast(s16x8, __builtin_bit_cast(u32x4, pf[s]) & only);
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const u32x4 w = __builtin_bit_cast(u32x4, tr_frag<DP>(v, tr, 16 * s, d)) & only;
            const f32x16 with = E::mfma(__builtin_bit_cast(s16x8, w), pn, o[d]);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = sees ? with[i] : o[d][i];
          }
        }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = E::mfma(tr_frag<DP>(v, tr, 16 * s, d), pf[s], o[d]);
    }
  };
  // The second group's sums, through LDS, into the first's, whose lanes hold the
  // same queries: half of o in the place of each pair of key tiles.
  const auto join = [&]() __attribute__((always_inline)) {
    static_assert(G <= 2, "one other group");
    const int t = threadIdx.x % (kWaves * OPA_WAVE);
    f32x4 *const so[2] = {reinterpret_cast<f32x4 *>(tk0[0]), reinterpret_cast<f32x4 *>(tk1[0])};
    f32x2 *const sm = reinterpret_cast<f32x2 *>(tv0[0]);
    block_sync();
    if (group) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          so[2 * d / DB][((d % (DB / 2)) * 4 + i) * kWaves * OPA_WAVE + t] =
              f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      sm[t] = f32x2{m, l};
    }
    block_sync();
    if (group == 0) {
      const f32x2 other = sm[t];
      const float to = fmaxf(m, other[0]);
      const float by = to == -INFINITY ? 1.f : exp2_fast((m - to) * c);
      const float with = to == -INFINITY ? 1.f : exp2_fast((other[0] - to) * c);
      m = to;
      l = l * by + other[1] * with;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 v = so[2 * d / DB][((d % (DB / 2)) * 4 + i) * kWaves * OPA_WAVE + t];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * i + e] = o[d][4 * i + e] * by + v[e] * with;
        }
    }
  };
  const auto start = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = (f32x16)(0.f);
    m = -INFINITY;
    l = 0.f;
  };
  start();
  run_tiles(
      (tiles + G - 1) / G,
      [&](auto i, int t) __attribute__((always_inline)) {
        load(i == 0 ? tk0[group] : tk1[group], i == 0 ? tv0[group] : tv1[group],
             (t * G + group) * kRowsK);
      },
      [&](auto i, int t) __attribute__((always_inline)) {
        step(std::false_type{}, i == 0 ? tk0[group] : tk1[group],
             i == 0 ? tv0[group] : tv1[group], (t * G + group) * kRowsK);
      });
  if constexpr (G > 1) join();
  // A weight of 0 times a value that is not finite is no 0: where a sum is not
  // finite, a second pass adds the values of a tile that not every query of the
  // wave sees key by key, and only to the queries that see the key.
  if (a.causal) {
    float zero = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) zero = fmaf(o[d][i], 0.f, zero);
    if (__syncthreads_or(group == 0 && !(zero == 0.f))) {
      start();
      for (int k0 = group * kRowsK; k0 < tiles * kRowsK + group * kRowsK; k0 += G * kRowsK) {
        load(tk0[group], tv0[group], k0);
        wait_loads();
        block_sync();
        step(std::true_type{}, tk0[group], tv0[group], k0);
        block_sync();
      }
      if constexpr (G > 1) join();
    }
  }
  l = half_sum(l);
  block_sync();  // the tiles' last readers are done
  if (group) return;
  store_rows<E, DP>((wave < 2 ? tk0[0] : tk1[0]) + wave % 2 * (kTile / 2), o,
                    l == 0.f ? 0.f : 1.f / l,
                    a.out.p + (int64_t)(sq.first + q0 + wave * 32) * a.out.ts +
                        (int64_t)head * a.out.hs,
                    a.out.ts, sq.count - q0 - wave * 32, a.head_dim);
  if (a.lse && live && h == 0)
    a.lse[(int64_t)head * a.n_q + sq.first + qrow] =
        l == 0.f ? -INFINITY : (m * c + log2_sum<E>(l)) * kLn2;
}

template <class E, int DP>
static void launch(const PromptArgs &a, hipStream_t s) {
  const int64_t blocks = ((int64_t)a.n_q / kRowsQ + a.n_seqs) * a.n_heads;
  if (blocks <= kFewBlocks && a.n_k >= (int64_t)kManyKeys * a.n_seqs)
    hipLaunchKernelGGL((k_attn_prompt<E, DP, 2>), dim3((uint32_t)blocks),
                       dim3(2 * kWaves * OPA_WAVE), 0, s, a);
  else
    hipLaunchKernelGGL((k_attn_prompt<E, DP, 1>), dim3((uint32_t)blocks),
                       dim3(kWaves * OPA_WAVE), 0, s, a);
}

// The offsets alone, for calls whose kernels have no queries to start from.
__global__ __launch_bounds__(256) void k_attn_check(PromptArgs a) {
  check_spans(a.cu_q, a.n_seqs, a.n_q, a.diag);
  check_spans(a.cu_k, a.n_seqs, a.n_k, a.diag);
}

void run_check(const PromptArgs &a, hipStream_t s) {
  if (a.diag) hipLaunchKernelGGL(k_attn_check, dim3(1), dim3(256), 0, s, a);
}

void run_prompt(const PromptArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  if (a.n_q == 0) {
    run_check(a, s);
    return;
  }
  if (dtype == OPATTR_BF16)
    a.head_dim <= 64 ? launch<BF16, 64>(a, s) : launch<BF16, 128>(a, s);
  else
    a.head_dim <= 64 ? launch<F16, 64>(a, s) : launch<F16, 128>(a, s);
}

}  // namespace opa
