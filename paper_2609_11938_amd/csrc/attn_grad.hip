// Gradient of attention over whole prompts (opattr_attn_prompt_grad).
//
// Two passes, each recomputing the weights p from lse; every sum has one owner
// and one order, so runs repeat bit for bit.
//   k_attn_dq   a wave holds 32 queries and passes over their keys: dq, and the
//               rows' D = sum_j p_j dp_j for the second pass
//   k_attn_dkv  a wave holds 32 keys of one key head, and their dk and dv, and
//               passes over the queries that see them, of every query head of
//               the group; where key tiles are few, a tile's passes are split
//               over several blocks and added up by k_dkv_sum
// Ten products where seven are needed (with the forward pass): the scores and dp
// are computed by both passes, because adding dq in the second needs float32 atomics,
// whose order changes the result; and sum_j p_j k_j, which takes the rounding of
// `out` out of dq, is one more.
//
// Products, exponentials and fragment reads follow one another in a wave, as in the
// forward pass: 12 documents of up to 4001 tokens, 16 heads on 4 of 128: dq 346 us, dk
// and dv 346, their sums 39, the matrix units busy 54% and 52% of the first two; with
// the forward pass 887 us, in float16 (two launches more, which read dout and v once
// more: 25 us) 961. 8 sequences of 512, 8 heads of 64: 16 and 18 us, one round of
// blocks; a training pass 43 us, in float16 53. head_dim 72 to 120 costs nearly what 128
// does.
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kGradWaves = 4;
constexpr int kHeld = 32 * kGradWaves;  // keys (queries) a block holds
// Keys a tile of the first pass, queries a tile of the second. Registers hold the
// scores of 32 at a time of head_dim 128.
constexpr int kStep(int dp) { return dp <= 64 ? 64 : 32; }

// Weights and their gradients are rounded to 16 bits for the products. For
// float16 both are scaled by powers of two first: the weights by 2^kWeight, and
// ds by 2^e with |ds| <= 2 |dout_i| |v_j|, so that its largest stays below
// 2^15 and small ones keep their bits. The largest are those of one sequence, of
// the n query heads from `head` on and key head hk: what is large, or not finite,
// in one sequence says nothing of another, and dq's of one head nothing of the next.
template <class E>
struct Scales {
  static constexpr float kWeight = 0.f;
  static __device__ __forceinline__ float ds(const PromptArgs &, int, int, int, int) {
    return 1.f;
  }
};
template <>
struct Scales<F16> {
  static constexpr float kWeight = 10.f;
  static __device__ __forceinline__ float ds(const PromptArgs &a, int seq, int head, int n,
                                             int hk) {
    const uint32_t *norms = a.norms + (int64_t)seq * (a.n_heads + a.n_kv);
    uint32_t dout = norms[head];
    if (n > 1) {
      for (int i = lane_id(); i < n; i += OPA_WAVE) dout = max(dout, norms[head + i]);
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) dout = max(dout, (uint32_t)__shfl_xor((int)dout, d));
      dout = (uint32_t)uniform((int)dout);
    }
    const float most = sqrtf(__uint_as_float(dout)) *
                       sqrtf(__uint_as_float(norms[a.n_heads + hk]));
    if (!(most > 0.f) || !(most < 1e30f)) return 1.f;
    int e;
    frexpf(most, &e);  // most < 2^e
    return ldexpf(1.f, clamp_to(14 - e, -100, 100));
  }
};

// float16: the largest squared norms of dout's and v's rows, of each sequence and
// head (the bits of non-negative floats order as integers, so the maximum is the same
// in any order). A block takes kNormRows rows of a sequence and one head: blockIdx.y
// is a query head, and past those a key head. 4 lanes a row.
constexpr int kNormRows = 512;
__global__ __launch_bounds__(256) void k_attn_norms(PromptArgs a) {
  __shared__ float most[4];
  const int sub = threadIdx.x & 3;
  const bool q = (int)blockIdx.y < a.n_heads;
  const int head = q ? blockIdx.y : blockIdx.y - a.n_heads;
  const int n = q ? a.n_q : a.n_k;
  const Rows x = q ? a.dout : a.v;
  const int32_t *cu = q ? a.cu_q : a.cu_k;
  Span s, same;
  int part, seq;
  if (!find_tile(cu, n, cu, n, a.n_seqs, kNormRows, blockIdx.x, s, same, part, &seq)) return;
  float top = 0.f;
  for (int t = part * kNormRows + (threadIdx.x >> 2); t < s.count && t < (part + 1) * kNormRows;
       t += 64) {
    const uint16_t *px = x.p + (int64_t)(s.first + t) * x.ts + (int64_t)head * x.hs;
    float norm = 0.f;
    for (int c = sub * 8; c < a.head_dim; c += 32) {
      const s16x8 u = *reinterpret_cast<const s16x8 *>(px + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = F16::widen((uint16_t)u[i]);
        norm = fmaf(f, f, norm);
      }
    }
    norm += __shfl_xor(norm, 1);
    norm += __shfl_xor(norm, 2);
    top = fmaxf(top, norm);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane_id() == 0) most[wave_id()] = top;
  __syncthreads();
  if (threadIdx.x == 0)
    atomicMax(&a.norms[(int64_t)seq * (a.n_heads + a.n_kv) + blockIdx.y],
              __float_as_uint(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]))));
}

__global__ void k_attn_zero(uint32_t *p, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0;
}

// Two groups of waves share the keys where the blocks are this few (one sequence
// of 6000, 4 heads, 192 blocks: a training pass of 378 us with one, 340 with two).
constexpr int kFewBlocks = 256, kManyKeys = 768;

// dq of 32 queries a wave: S^T = K Q^T with the wave's queries as columns;
// dS^T then is the B operand of dq^T = K^T dS^T. The pass goes by D' = dout . out,
// which out's 16 bits make inexact; D - D' = sum_j p_j (dp_j - D') is summed beside
// it, and with kp = sum_j p_j k_j, dq = sum_j p_j (dp_j - D') k_j - (D - D') kp puts
// that right (a product more; the error of a training pass against 64 bits, in that of
// the plain form rounded to 16 bits once: 1.65 without, 1.4 to 1.5 with). The exact D
// goes to the second pass with the scaled lse.
template <class E, int DP, int G>
__global__ __launch_bounds__(G * kGradWaves * OPA_WAVE, 2) void k_attn_dq(PromptArgs a) {
  constexpr int KS = DP / 16, DB = DP / 32;
  constexpr int kStepK = kStep(DP), kTile = kStepK * DP;
  // a group's two tiles of keys, two of values; the second's sums at the end
  __shared__ __align__(16) uint16_t tk0[G][kTile], tk1[G][kTile], tv0[G][kTile], tv1[G][kTile];
  // of head_dim 128, dout's fragments, which the registers have no room for
  constexpr bool kHeldHere = DP <= 64;
  __shared__ s16x8 held[kHeldHere ? 1 : kGradWaves * KS * OPA_WAVE];
  const int lane = lane_id(), all = uniform(wave_id());
  const int wave = all % kGradWaves, group = all / kGradWaves;
  s16x8 *const mine = held + (kHeldHere ? 0 : wave * KS * OPA_WAVE + lane);
  const int r = lane & 31, h = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % a.n_kv;
  id /= a.n_kv;
  const int head = hk * a.group + id % a.group;
  if (blockIdx.x == 0) {
    check_spans(a.cu_q, a.n_seqs, a.n_q, a.diag);
    check_spans(a.cu_k, a.n_seqs, a.n_k, a.diag);
  }
  Span sq, sk;
  int part, seq;
  if (!find_tile(a.cu_q, a.n_q, a.cu_k, a.n_k, a.n_seqs, kHeld, id / a.group, sq, sk, part, &seq))
    return;
  const int q0 = ((sq.count + kHeld - 1) / kHeld - 1 - part) * kHeld;
  const int lead = sk.count - sq.count;
  const int qrow = q0 + wave * 32 + r;
  const bool live = qrow < sq.count;
  const int last = (q0 + kHeld < sq.count ? q0 + kHeld : sq.count) - 1;
  const int keys = a.causal ? clamp_to(last + lead + 1, 0, sk.count) : sk.count;
  const int tiles = (keys + kStepK - 1) / kStepK;
  const int whole = a.causal ? clamp_to(q0 + wave * 32 + lead + 1, 0, sk.count) : sk.count;
  const int seen = live ? (a.causal ? clamp_to(qrow + lead + 1, 0, sk.count) : sk.count) : 0;
  s16x8 qf[KS], df[kHeldHere ? KS : 1];
  float L = INFINITY, D = 0.f, off = 0.f;
  {
    const int64_t tok = sq.first + (live ? qrow : 0);
    const uint16_t *qp = a.q.p + tok * a.q.ts + (int64_t)head * a.q.hs;
    const uint16_t *dp = a.dout.p + tok * a.dout.ts + (int64_t)head * a.dout.hs;
    const uint16_t *op = a.out.p + tok * a.out.ts + (int64_t)head * a.out.hs;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      s16x8 d = (s16x8)(0);
      qf[s] = (s16x8)(0);
      if (live && 16 * s + 8 * h < a.head_dim) {
        qf[s] = *reinterpret_cast<const s16x8 *>(qp + 16 * s + 8 * h);
        d = *reinterpret_cast<const s16x8 *>(dp + 16 * s + 8 * h);
        const s16x8 of = *reinterpret_cast<const s16x8 *>(op + 16 * s + 8 * h);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          D = fmaf(E::widen((uint16_t)d[i]), E::widen((uint16_t)of[i]), D);
      }
      if constexpr (kHeldHere)
        df[s] = d;
      else if (group == 0)
        mine[s * OPA_WAVE] = d;
    }
    D = half_sum(D);
    if (live) {
      // a query that sees nothing has weights 0: exp2(x - inf)
      const float lse = a.lse[(int64_t)head * a.n_q + tok] * kLog2e;
      L = lse == -INFINITY ? INFINITY : lse - Scales<E>::kWeight;
    }
  }
  const uint16_t *k0p = a.k.p + (int64_t)sk.first * a.k.ts + (int64_t)hk * a.k.hs;
  const uint16_t *v0p = a.v.p + (int64_t)sk.first * a.v.ts + (int64_t)hk * a.v.hs;
  const float c = a.scale * kLog2e;
  const float up = Scales<E>::ds(a, seq, head, 1, hk);
  const float fw = exp2_fast(-Scales<E>::kWeight), upw = up * fw;
  const int nat0 = nat_place<DP>(), tr0 = tr_place<DP>();
  f32x16 dq[DB], kp[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dq[d] = kp[d] = (f32x16)(0.f);

  const auto load = [&](uint16_t *k, uint16_t *v, int k0) __attribute__((always_inline)) {
    tile_load<DP, kStepK, kGradWaves>(k, k0p + k0 * a.k.ts, a.k.ts, sk.count - k0, a.head_dim,
                                     wave);
    tile_load<DP, kStepK, kGradWaves>(v, v0p + k0 * a.v.ts, a.v.ts, sk.count - k0, a.head_dim,
                                     wave);
  };
  const auto step = [&](const uint16_t *k, const uint16_t *v, int k0)
                        __attribute__((always_inline)) {
    const bool cut = k0 + kStepK > whole;
    const int nat = fresh(nat0), tr = fresh(tr0);
#pragma unroll
    for (int kb = 0; kb < kStepK / 32; ++kb) {
      f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        x = E::mfma(nat_frag<DP>(k, nat, 32 * kb, s), qf[s], x);
        y = E::mfma(nat_frag<DP>(v, nat, 32 * kb, s),
                    kHeldHere ? df[kHeldHere ? s : 0] : mine[s * OPA_WAVE], y);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = exp2_fast(fmaf(x[e], c, -L));
        y[e] = x[e] * (y[e] - D) * upw;
      }
      if (cut) {  // both: of a hidden key either may be past float32
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 32 * kb + 8 * (e >> 2) + 4 * h + (e & 3) >= seen) x[e] = y[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 16; e += 4) off += (y[e] + y[e + 1]) + (y[e + 2] + y[e + 3]);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 wp, ws;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          wp[i] = E::pack(x[8 * s + 2 * i], x[8 * s + 2 * i + 1]);
          ws[i] = E::pack(y[8 * s + 2 * i], y[8 * s + 2 * i + 1]);
        }
        const s16x8 pf = __builtin_bit_cast(s16x8, wp), sf = __builtin_bit_cast(s16x8, ws);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const s16x8 kt = tr_frag<DP>(k, tr, 32 * kb + 16 * s, d);
          dq[d] = E::mfma(kt, sf, dq[d]);
          kp[d] = E::mfma(kt, pf, kp[d]);
        }
      }
    }
  };
  run_tiles(
      (tiles + G - 1) / G,
      [&](auto i, int t) __attribute__((always_inline)) {
        load(i == 0 ? tk0[group] : tk1[group], i == 0 ? tv0[group] : tv1[group],
             (t * G + group) * kStepK);
      },
      [&](auto i, int t) __attribute__((always_inline)) {
        step(i == 0 ? tk0[group] : tk1[group], i == 0 ? tv0[group] : tv1[group],
             (t * G + group) * kStepK);
      });
  off = half_sum(off);
  const int t = threadIdx.x % (kGradWaves * OPA_WAVE);
  if constexpr (G > 1) {  // of both groups' keys
    static_assert(G == 2, "one other group");
    __shared__ float sum[G][kGradWaves * OPA_WAVE];
    sum[group][t] = off;
    block_sync();
    off = sum[0][t] + sum[1][t];
  }
  const float f = 1.f / up;
  off *= f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[d][i] = a.scale * (dq[d][i] * f - off * fw * kp[d][i]);
  if constexpr (G > 1) {
    // the second group's dq to the first's: a part in each of the four tiles' places
    constexpr int kEach = G * kTile * 2 / 16 / (kGradWaves * OPA_WAVE);  // pieces a lane
    static_assert(4 * kEach >= DB * 4, "they fit");
    f32x4 *const at[4] = {reinterpret_cast<f32x4 *>(tk0[0]), reinterpret_cast<f32x4 *>(tk1[0]),
                          reinterpret_cast<f32x4 *>(tv0[0]), reinterpret_cast<f32x4 *>(tv1[0])};
    if (group) {
#pragma unroll
      for (int i = 0; i < DB * 4; ++i)
        at[i / kEach][i % kEach * kGradWaves * OPA_WAVE + t] =
            f32x4{dq[i / 4][i % 4 * 4], dq[i / 4][i % 4 * 4 + 1], dq[i / 4][i % 4 * 4 + 2],
                  dq[i / 4][i % 4 * 4 + 3]};
    }
    block_sync();
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < DB * 4; ++i) {
        const f32x4 v = at[i / kEach][i % kEach * kGradWaves * OPA_WAVE + t];
#pragma unroll
        for (int e = 0; e < 4; ++e) dq[i / 4][i % 4 * 4 + e] += v[e];
      }
    }
  }
  if (group == 0 && live && h == 0) {
    const int64_t at = (int64_t)head * a.n_q + sq.first + qrow;
    *reinterpret_cast<f32x2 *>(a.rows + 2 * at) = f32x2{L, D + off};
  }
  block_sync();  // the tiles' last readers are done
  if (group) return;
  constexpr int kFit = G * kTile / (32 * DP);  // waves' rows in one tile's place
  uint16_t *const place = wave / kFit == 0 ? tk0[0]
                          : wave / kFit == 1 ? tk1[0]
                          : wave / kFit == 2 ? tv0[0]
                                             : tv1[0];
  store_rows<E, DP>(place + wave % kFit * 32 * DP, dq, 1.f,
                    a.dq.p + (int64_t)(sq.first + q0 + wave * 32) * a.dq.ts +
                        (int64_t)head * a.dq.hs,
                    a.dq.ts, sq.count - q0 - wave * 32, a.head_dim);
}

// 32 pairs (lse, D) from p to LDS, past `left` of them zero; by a whole wave.
__device__ __forceinline__ void row_load(float *to, const float *p, int left) {
  const int n = left < 0 ? 0 : left > 32 ? 32 : left;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float *>(reinterpret_cast<const float *>(
          uniform(reinterpret_cast<const uint16_t *>(p)))),
      (short)0, uniform(n * 8), 0x00027000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)to, 4,
                                           lane_id() * 4, 0, 0, 0);
}

// Tiles of queries that key tile `part` of a sequence meets: the first, and how many.
template <int DP>
__device__ __forceinline__ Span tile_queries(const PromptArgs &a, const Span &sq, const Span &sk,
                                             int part) {
  const int begin =
      a.causal ? clamp_to(part * kHeld - (sk.count - sq.count), 0, sq.count) : 0;
  const int first = begin / kStep(DP), end = (sq.count + kStep(DP) - 1) / kStep(DP);
  return {first, end - first};
}
// Blocks that share the tile: as many as bring each to a.split_steps steps of 32
// queries or fewer, at most a.splits.
template <int DP>
__device__ __forceinline__ int tile_splits(const PromptArgs &a, const Span &sq, const Span &sk,
                                           int part) {
  const int steps = tile_queries<DP>(a, sq, sk, part).count * a.group * (kStep(DP) / 32);
  return clamp_to((steps + a.split_steps - 1) / a.split_steps, 1, a.splits);
}

// Where a wave of one of a tile's blocks leaves its dk and dv, as its registers hold
// them: [splits][tiles][n_kv][waves][dk, dv][DP / 8][64 lanes] of four values.
template <int DP>
__device__ __forceinline__ f32x4 *part_of(const PromptArgs &a, int split, int tile, int hk,
                                          int wave) {
  const int64_t tiles = a.n_k / kHeld + a.n_seqs;
  const int64_t at = ((split * tiles + tile) * a.n_kv + hk) * kGradWaves + wave;
  return reinterpret_cast<f32x4 *>(a.part) + at * (2 * DP / 8 * OPA_WAVE) + lane_id();
}

// dk and dv of 32 keys a wave: S = Q K^T with the wave's keys as columns, so
// that a lane holds one key; P and dS then are the B operands of
// dv^T = dout^T P and dk^T = q^T dS.
template <class E, int DP>
__global__ __launch_bounds__(kGradWaves * OPA_WAVE, 2) void k_attn_dkv(PromptArgs a) {
  constexpr int KS = DP / 16, DB = DP / 32;
  constexpr int kStepQ = kStep(DP), kTile = kStepQ * DP, kQB = kStepQ / 32;
  __shared__ __align__(16) uint16_t tq0[kTile], tq1[kTile], td0[kTile], td1[kTile];
  __shared__ __align__(16) float ts0[2 * kStepQ], ts1[2 * kStepQ];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 31, h = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % a.n_kv;
  id /= a.n_kv;
  const int split = id % a.splits;
  Span sq, sk;
  int part, seq;
  if (!find_tile(a.cu_k, a.n_k, a.cu_q, a.n_q, a.n_seqs, kHeld, id / a.splits, sk, sq, part, &seq))
    return;
  const int lead = sk.count - sq.count;
  const int key0 = part * kHeld + wave * 32, key = key0 + r;
  const bool live = key < sk.count;
  // the first query that sees every key of this wave, and the first that sees
  // this lane's
  const int whole = key0 + 32 > sk.count ? sq.count
                                         : a.causal ? clamp_to(key0 + 31 - lead, 0, sq.count) : 0;
  const int from = live ? (a.causal ? clamp_to(key - lead, 0, sq.count) : 0) : sq.count;
  const Span met = tile_queries<DP>(a, sq, sk, part);
  const int t0 = met.first, per = met.count;
  // this block's steps of the tile's: a head's queries, then the next head's
  const int splits = tile_splits<DP>(a, sq, sk, part), all = per * a.group;
  if (split >= splits) return;
  const int first = (int)((int64_t)all * split / splits);
  const int steps = (int)((int64_t)all * (split + 1) / splits);
  s16x8 kf[KS], vf[KS];
  {
    const int64_t tok = sk.first + (live ? key : 0);
    const uint16_t *kp = a.k.p + tok * a.k.ts + (int64_t)hk * a.k.hs;
    const uint16_t *vp = a.v.p + tok * a.v.ts + (int64_t)hk * a.v.hs;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kf[s] = (s16x8)(0);
      vf[s] = (s16x8)(0);
      if (live && 16 * s + 8 * h < a.head_dim) {
        kf[s] = *reinterpret_cast<const s16x8 *>(kp + 16 * s + 8 * h);
        vf[s] = *reinterpret_cast<const s16x8 *>(vp + 16 * s + 8 * h);
      }
    }
  }
  const float c = a.scale * kLog2e;
  const float up = Scales<E>::ds(a, seq, hk * a.group, a.group, hk);
  const float fv = exp2_fast(-Scales<E>::kWeight), upw = up * fv;
  const int nat0 = nat_place<DP>(), tr0 = tr_place<DP>();
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = dv[d] = (f32x16)(0.f);

  // Queries past the sequence's last, and tiles past this block's last, come as
  // zero rows with lse and D zero: they add zeros.
  const auto load = [&](uint16_t *q, uint16_t *dout, float *rows, int t)
                        __attribute__((always_inline)) {
    const int g = t / per, q0 = (t0 + t - g * per) * kStepQ, head = hk * a.group + g;
    const int left = t < steps ? sq.count - q0 : 0;
    const int64_t tok = sq.first + q0;
    tile_load<DP, kStepQ, kGradWaves>(q, a.q.p + tok * a.q.ts + (int64_t)head * a.q.hs, a.q.ts,
                                      left, a.head_dim, wave);
    tile_load<DP, kStepQ, kGradWaves>(dout,
                                      a.dout.p + tok * a.dout.ts + (int64_t)head * a.dout.hs,
                                      a.dout.ts, left, a.head_dim, wave);
#pragma unroll
    for (int b = 0; b < kQB; ++b)
      if (wave == b)
        row_load(rows + 64 * b, a.rows + ((int64_t)head * a.n_q + tok + 32 * b) * 2, left - 32 * b);
  };
  const auto step = [&](const uint16_t *q, const uint16_t *dout, const float *rows, int t)
                        __attribute__((always_inline)) {
    const int q0 = (t0 + t % per) * kStepQ;
    const int nat = fresh(nat0), tr = fresh(tr0);
#pragma unroll
    for (int qb = 0; qb < kQB; ++qb) {
      f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        x = E::mfma(nat_frag<DP>(q, nat, 32 * qb, s), kf[s], x);
        y = E::mfma(nat_frag<DP>(dout, nat, 32 * qb, s), vf[s], y);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 r0 = *reinterpret_cast<const f32x4 *>(rows + 64 * qb + 2 * (8 * g + 4 * h));
        const f32x4 r1 = *reinterpret_cast<const f32x4 *>(rows + 64 * qb + 2 * (8 * g + 4 * h) + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 4 * g + i;
          const float p = exp2_fast(fmaf(x[e], c, -(i < 2 ? r0[2 * i] : r1[2 * i - 4])));
          y[e] = p * (y[e] - (i < 2 ? r0[2 * i + 1] : r1[2 * i - 3])) * upw;
          x[e] = p;
        }
      }
      if (q0 < whole) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (q0 + 32 * qb + 8 * (e >> 2) + 4 * h + (e & 3) < from) x[e] = y[e] = 0.f;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 wp, ws;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          wp[i] = E::pack(x[8 * s + 2 * i], x[8 * s + 2 * i + 1]);
          ws[i] = E::pack(y[8 * s + 2 * i], y[8 * s + 2 * i + 1]);
        }
        const s16x8 pf = __builtin_bit_cast(s16x8, wp), sf = __builtin_bit_cast(s16x8, ws);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          dv[d] = E::mfma(tr_frag<DP>(dout, tr, 32 * qb + 16 * s, d), pf, dv[d]);
          dk[d] = E::mfma(tr_frag<DP>(q, tr, 32 * qb + 16 * s, d), sf, dk[d]);
        }
      }
    }
  };
  run_tiles(
      steps - first,
      [&](auto i, int t) __attribute__((always_inline)) {
        load(i == 0 ? tq0 : tq1, i == 0 ? td0 : td1, i == 0 ? ts0 : ts1, first + t);
      },
      [&](auto i, int t) __attribute__((always_inline)) {
        step(i == 0 ? tq0 : tq1, i == 0 ? td0 : td1, i == 0 ? ts0 : ts1, first + t);
      });
  const float fk = a.scale / up;
  if (splits > 1) {
    f32x4 *p = part_of<DP>(a, split, id / a.splits, hk, wave);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 x, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = dk[d][4 * g + i] * fk;
          y[i] = dv[d][4 * g + i] * fv;
        }
        p[(4 * d + g) * OPA_WAVE] = x;
        p[(4 * DB + 4 * d + g) * OPA_WAVE] = y;
      }
    return;
  }
  block_sync();  // the tiles' last readers are done
  constexpr int kFit = kTile / (32 * DP);  // waves' rows in one tile's place
  uint16_t *const place = (wave / kFit == 0 ? tq0 : wave / kFit == 1 ? tq1
                                                  : wave / kFit == 2 ? td0
                                                                     : td1) +
                          wave % kFit * 32 * DP;
  const int64_t tok = sk.first + key0;
  store_rows<E, DP>(place, dk, fk, a.dk.p + tok * a.dk.ts + (int64_t)hk * a.dk.hs, a.dk.ts,
                    sk.count - key0, a.head_dim);
  store_rows<E, DP>(place, dv, fv, a.dv.p + tok * a.dv.ts + (int64_t)hk * a.dv.hs, a.dv.ts,
                    sk.count - key0, a.head_dim);
}

// A key tile's dk and dv from those of its blocks, added in order; a tile of one
// block is done already. A wave takes dk or dv of 32 keys.
template <class E, int DP>
__global__ __launch_bounds__(2 * kGradWaves * OPA_WAVE) void k_dkv_sum(PromptArgs a) {
  constexpr int DB = DP / 32;
  __shared__ __align__(16) uint16_t rows[2 * kGradWaves][32 * DP];
  const int hk = blockIdx.x % a.n_kv, tile = blockIdx.x / a.n_kv;
  const int all = uniform(wave_id()), wave = all / 2, which = all % 2;
  Span sq, sk;
  int part;
  if (!find_tile(a.cu_k, a.n_k, a.cu_q, a.n_q, a.n_seqs, kHeld, tile, sk, sq, part)) return;
  const int splits = tile_splits<DP>(a, sq, sk, part);
  const int key0 = part * kHeld + wave * 32;
  if (splits == 1 || key0 >= sk.count) return;
  f32x16 sum[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) sum[d] = (f32x16)(0.f);
  for (int k = 0; k < splits; ++k) {
    const f32x4 *p = part_of<DP>(a, k, tile, hk, wave) + which * 4 * DB * OPA_WAVE;
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      const f32x4 v = p[i * OPA_WAVE];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[i / 4][i % 4 * 4 + e] += v[e];
    }
  }
  const Rows &o = which ? a.dv : a.dk;
  store_rows<E, DP>(rows[all], sum, 1.f,
                    o.p + (int64_t)(sk.first + key0) * o.ts + (int64_t)hk * o.hs, o.ts,
                    sk.count - key0, a.head_dim);
}

template <class E, int DP>
static void launch(const PromptArgs &a, hipStream_t s) {
  const int64_t kt = (int64_t)a.n_k / kHeld + a.n_seqs, qt = (int64_t)a.n_q / kHeld + a.n_seqs;
  const dim3 block(kGradWaves * OPA_WAVE);
  const dim3 rows((uint32_t)(qt * a.n_heads));
  if (a.n_q > 0 && qt * a.n_heads <= kFewBlocks && a.n_k >= (int64_t)kManyKeys * a.n_seqs)
    hipLaunchKernelGGL((k_attn_dq<E, DP, 2>), rows, dim3(2 * kGradWaves * OPA_WAVE), 0, s, a);
  else if (a.n_q > 0)
    hipLaunchKernelGGL((k_attn_dq<E, DP, 1>), rows, block, 0, s, a);
  if (a.n_k == 0) return;
  hipLaunchKernelGGL((k_attn_dkv<E, DP>), dim3((uint32_t)(kt * a.n_kv * a.splits)), block, 0, s,
                     a);
  if (a.splits > 1)
    hipLaunchKernelGGL((k_dkv_sum<E, DP>), dim3((uint32_t)(kt * a.n_kv)),
                       dim3(2 * kGradWaves * OPA_WAVE), 0, s, a);
}

template <class E>
static void grad(const PromptArgs &a, hipStream_t s) {
  if (a.norms) {
    const int n = a.n_seqs * (a.n_heads + a.n_kv);
    hipLaunchKernelGGL(k_attn_zero, dim3((n + 63) / 64), dim3(64), 0, s, a.norms, n);
    const int most = a.n_k > a.n_q ? a.n_k : a.n_q;
    const dim3 grid(most / kNormRows + a.n_seqs, a.n_heads + a.n_kv);
    if (most > 0) hipLaunchKernelGGL(k_attn_norms, grid, dim3(256), 0, s, a);
  }
  if (a.head_dim <= 64)
    launch<E, 64>(a, s);
  else
    launch<E, 128>(a, s);
}

// Blocks of a key tile at most. A tile's steps go one after another, and a causal
// sequence's first tile has the most: about 2048 blocks keep the chip full to
// the end (12 packed documents of up to 4001, 512 blocks without: 1110 us, 2048:
// 900 us, 4096: 1000 us). By the mean length: blocks that find their tile not
// split cost what the others gain (8 sequences of 512: 46 us unsplit, 57 us with
// six blocks a tile that do nothing). Where the tiles leave compute units without a
// block, a block takes fewer steps (4 sequences of 512, 8 heads on 4 of 128, 64 tiles
// of up to 32 steps: a training pass of 85 us unsplit, 69 us by 8 steps, of which the
// sums take 10; of 20 steps 48 and 47: not below 24).
// The mean is what a batch of like sequences wants; a long one beside many short ones
// is split less than alone: 4000 tokens, 8 heads on 2 of 128, a training pass of 268
// us, with 30 sequences of one token beside it 797.
constexpr int kSplitSteps = 24, kFewSteps = 8, kFewTiles = 192;
GradSplits grad_splits(int64_t n_q, int64_t n_k, int n_seqs, int n_heads, int n_kv) {
  GradSplits x{1, kSplitSteps};
  if (n_seqs == 0 || n_k == 0) return x;
  const int64_t blocks = (n_k / kHeld + n_seqs) * n_kv;
  const int64_t steps = n_q * (n_heads / n_kv) / 32 / n_seqs;
  if (blocks <= kFewTiles && steps >= kSplitSteps) x.steps = kFewSteps;
  int64_t n = (2048 + blocks - 1) / blocks;
  if (n > steps / x.steps) n = steps / x.steps;
  x.most = n < 1 ? 1 : n > 16 ? 16 : (int)n;
  return x;
}

void run_prompt_grad(const PromptArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  if (a.n_q == 0) run_check(a, s);
  if (dtype == OPATTR_BF16)
    grad<BF16>(a, s);
  else
    grad<F16>(a, s);
}

}  // namespace opa
