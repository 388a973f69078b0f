// Gradient of attention over whole prompts (opattr_attn_prompt_grad).
//
// Two passes, each recomputing the weights p from lse; every sum has one owner
// and one order, so runs repeat bit for bit.
//   k_attn_dq   a wave holds 32 queries and passes over their keys: dq, and the
//               rows' D = sum_j p_j dp_j for the second pass
//   k_attn_dkv  a wave holds 32 keys of one key head, and their dk and dv, and
//               passes over the queries that see them, of every query head of
//               the group; where key tiles are few, a tile's passes are split
//               over several blocks and added up by k_dkv_sum (k_window_sum)
// Ten products where seven are needed (with the forward pass): the scores and dp
// are computed by both passes, because adding dq in the second needs float32 atomics,
// whose order changes the result; and sum_j p_j k_j, which takes the rounding of
// `out` out of dq, is one more.
//
// Products, exponentials and fragment reads follow one another in a wave, as in the
// forward pass: 12 documents of up to 4001 tokens, 16 heads on 4 of 128: dq 346 us, dk
// and dv 346, their sums 39, the matrix units busy 54% and 52% of the first two; with
// the forward pass 887 us, in float16 (one launch more: dout and v once more: 18 us)
// 956. 8 sequences of 512, 8 heads of 64: 16 and 18 us, one round of blocks; a training
// pass 43 us, in float16 50. head_dim 72 to 120 costs nearly what 128 does.
#include <algorithm>

#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kGradWaves = 4;
constexpr int kHeld = 32 * kGradWaves;  // keys (queries) a block holds
// Keys a tile of the first pass, queries a tile of the second. Registers hold the
// scores of 32 at a time of head_dim 128.
constexpr int kStep(int dp) { return dp <= 64 ? 64 : 32; }

// float16: the largest squared norms of dout's and v's rows, in pieces of kNormRows rows of a
// sequence and head: [n_heads + n_kv][slots] as the bits of non-negative floats, whose order
// is that of integers. Piece p of sequence b is in slot b + first / kNormRows + p, first its
// first row, which leaves room for every sequence's, and each has one writer: nothing is
// cleared before, and a long sequence's pieces are many blocks'.
constexpr int kNormRows = 128, kNormThreads = 256;
int64_t norm_slots(int64_t n_q, int64_t n_k, int n_seqs) {
  return std::max(n_q, n_k) / kNormRows + n_seqs;
}
__device__ __forceinline__ int norms_at(const PromptArgs &a, int head, int seq, const Span &s) {
  return head * a.norm_slots + seq + s.first / kNormRows;
}
// The product of the largest norms of dout, of n query heads from `head` on, and of v; by
// whole waves.
__device__ __forceinline__ float most_norms(const PromptArgs &a, int seq, const Span &sq,
                                            const Span &sk, int head, int n, int hk) {
  const uint32_t *dout = a.norms + norms_at(a, head, seq, sq);
  const uint32_t *v = a.norms + norms_at(a, a.n_heads + hk, seq, sk);
  const int pieces = tiles_of(sq.count, kNormRows), douts = pieces * n;
  const int vs = tiles_of(sk.count, kNormRows), most = douts > vs ? douts : vs;
  uint32_t x = 0, y = 0;
  if (douts == 1 && vs == 1) {  // by scalars (1000 sequences of 20: 331 us, 320 so)
    x = dout[0];
    y = v[0];
  } else {
    for (int i = lane_id(); i < most; i += OPA_WAVE) {
      const int h = n == 1 || i >= douts ? 0 : i / pieces;
      if (i < douts) x = max(x, dout[h * a.norm_slots + i - h * pieces]);
      if (i < vs) y = max(y, v[i]);
    }
    x = wave_max(x);
    y = wave_max(y);
  }
  return sqrtf(__uint_as_float(x)) * sqrtf(__uint_as_float(y));
}

// Weights and their gradients are rounded to 16 bits for the products. For
// float16 both are scaled by powers of two first: the weights by 2^kWeight, and
// ds by 2^e with |ds| <= 2 |dout_i| |v_j|, so that its largest stays below
// 2^15 and small ones keep their bits. The largest are those of one sequence, of
// the n query heads from `head` on and key head hk: what is large, or not finite,
// in one sequence says nothing of another, and dq's of one head nothing of the next.
template <class E>
struct Scales {
  static constexpr float kWeight = 0.f;
  static __device__ __forceinline__ float ds(const PromptArgs &, int, const Span &, const Span &,
                                             int, int, int) {
    return 1.f;
  }
};
template <>
struct Scales<F16> {
  static constexpr float kWeight = 10.f;
  static __device__ __forceinline__ float ds(const PromptArgs &a, int seq, const Span &sq,
                                             const Span &sk, int head, int n, int hk) {
    const float most = most_norms(a, seq, sq, sk, head, n, hk);
    if (!(most > 0.f) || !(most < 1e30f)) return 1.f;
    int e;
    frexpf(most, &e);  // most < 2^e
    return ldexpf(1.f, clamp_to(14 - e, -100, 100));
  }
};

// A block takes a piece of one head: blockIdx.y is a query head, and past those a key
// head. 4 lanes a row. 8 heads of 64: 8 sequences of 512 4.1 us, one of 4000 beside three
// of 20 4.2 (16 heads on 4 of 128: 7.6); 12 documents of up to 4001 of those 18 to 21, 77 MB
// at 4 TB/s. Pieces of 512 rows by 1024 threads find 1000 sequences of 20 in 142 us and not
// 53, by 256 threads those of 512 in 6.6.
__global__ __launch_bounds__(kNormThreads) void k_attn_norms(PromptArgs a) {
  __shared__ float most[kNormThreads / OPA_WAVE];
  const int sub = threadIdx.x & 3;
  const bool q = (int)blockIdx.y < a.n_heads;
  const int head = q ? blockIdx.y : blockIdx.y - a.n_heads;
  const int n = q ? a.n_q : a.n_k;
  const Rows x = q ? a.dout : a.v;
  const int32_t *cu = q ? a.cu_q : a.cu_k;
  Span s, same;
  int part, seq;
  if (!find_tile(cu, n, cu, n, a.n_seqs, kNormRows, blockIdx.x, s, same, part, &seq)) return;
  const int past = s.count < (part + 1) * kNormRows ? s.count : (part + 1) * kNormRows;
  float top = 0.f;
  for (int t = part * kNormRows + (threadIdx.x >> 2); t < past; t += kNormThreads / 4) {
    const uint16_t *px = x.p + (int64_t)(s.first + t) * x.ts + (int64_t)head * x.hs;
    s16x8 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = (s16x8)(0);
      if (sub * 8 + 32 * j < a.head_dim)
        u[j] = *reinterpret_cast<const s16x8 *>(px + sub * 8 + 32 * j);
    }
    float norm = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float f = F16::widen((uint16_t)u[i / 8][i % 8]);
      norm = fmaf(f, f, norm);
    }
    norm += __shfl_xor(norm, 1);
    norm += __shfl_xor(norm, 2);
    top = fmaxf(top, norm);
  }
  top = __uint_as_float(wave_max(__float_as_uint(top)));
  if (lane_id() == 0) most[wave_id()] = top;
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int w = 1; w < kNormThreads / OPA_WAVE; ++w) top = fmaxf(top, most[w]);
  a.norms[norms_at(a, blockIdx.y, seq, s) + part] = __float_as_uint(top);
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
// W: through a window with sinks, with heads and keys as in the forward pass: 12
// documents of up to 4001 tokens, 16 heads on 4 of 128, window 512, 4 sinks, float16: 168
// us, dk and dv 175 and the sinks' sums 10 (without a window 360, 353 and 40).
template <class E, int DP, int G, bool W>
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
  const int hs = W ? a.head_shift : 0, heads = a.group >> hs;
  const int head = hk * a.group + (id % heads << hs) + (wave & ((1 << hs) - 1));
  const int rows = kHeld >> hs, from = (wave >> hs) * 32;  // the block's, the wave's first
  if (blockIdx.x == 0) {
    check_spans(a.cu_q, a.n_seqs, a.n_q, a.diag, G * kGradWaves * OPA_WAVE);
    check_spans(a.cu_k, a.n_seqs, a.n_k, a.diag, G * kGradWaves * OPA_WAVE);
  }
  Span sq, sk;
  int part, seq;
  if constexpr (W) {
    if (!find_tile(a.cu_q, a.n_q, a.cu_k, a.n_k, a.n_seqs, RowsLog2{7 - hs}, id / heads, sq, sk,
                   part, &seq))
      return;
  } else {
    if (!find_tile(a.cu_q, a.n_q, a.cu_k, a.n_k, a.n_seqs, kHeld, id / heads, sq, sk, part, &seq))
      return;
  }
  const int q0 = W ? (tiles_of(sq.count, RowsLog2{7 - hs}) - 1 - part) * rows
                   : ((sq.count + kHeld - 1) / kHeld - 1 - part) * kHeld;
  const int lead = sk.count - sq.count;
  const int qrow = q0 + from + r;
  const bool live = qrow < sq.count;
  const int last = (q0 + rows < sq.count ? q0 + rows : sq.count) - 1;
  const int front = W ? window_front(a.sinks) : 0;
  const int skip = W ? window_skip(q0 + lead, a.window, front) : 0;
  const int there = sk.count - skip;  // keys, without those skipped
  const int keys = a.causal ? clamp_to(last + lead + 1, 0, sk.count) - skip : sk.count;
  const int tiles = (keys + kStepK - 1) / kStepK;
  const int whole = a.causal ? clamp_to(q0 + from + lead + 1, 0, sk.count) - skip : sk.count;
  const int seen =
      live ? (a.causal ? clamp_to(qrow + lead + 1, 0, sk.count) - skip : sk.count) : 0;
  // where the window of the wave's last query begins
  const int latest = W ? q0 + from + 31 + lead + 1 - a.window - skip : 0;
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
  const float up = Scales<E>::ds(a, seq, sq, sk, head, 1, hk);
  const float fw = exp2_fast(-Scales<E>::kWeight), upw = up * fw;
  const int nat0 = nat_place<DP>(), tr0 = tr_place<DP>();
  f32x16 dq[DB], kp[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dq[d] = kp[d] = (f32x16)(0.f);

  const auto load = [&](uint16_t *k, uint16_t *v, int k0) __attribute__((always_inline)) {
    if constexpr (W) {
      window_tile_load<DP, kStepK, kGradWaves>(k, k0p, a.k.ts, k0, there - k0, front, skip,
                                               a.head_dim, wave);
      window_tile_load<DP, kStepK, kGradWaves>(v, v0p, a.v.ts, k0, there - k0, front, skip,
                                               a.head_dim, wave);
    } else {
      tile_load<DP, kStepK, kGradWaves>(k, k0p + k0 * a.k.ts, a.k.ts, there - k0, a.head_dim,
                                       wave);
      tile_load<DP, kStepK, kGradWaves>(v, v0p + k0 * a.v.ts, a.v.ts, there - k0, a.head_dim,
                                       wave);
    }
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
      // both: of a hidden key either may be past float32
      if constexpr (W) {
        hide_keys(k0 + 32 * kb, whole, fresh(seen), latest, a.window, a.sinks,
                  [&](int e) __attribute__((always_inline)) { x[e] = y[e] = 0.f; });
      } else if (cut) {
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
  uint16_t *const room = wave / kFit == 0 ? tk0[0]
                         : wave / kFit == 1 ? tk1[0]
                         : wave / kFit == 2 ? tv0[0]
                                            : tv1[0];
  store_rows<E, DP>(room + wave % kFit * 32 * DP, dq, 1.f,
                    a.dq.p + (int64_t)(sq.first + q0 + from) * a.dq.ts + (int64_t)head * a.dq.hs,
                    a.dq.ts, sq.count - q0 - from, a.head_dim);
}

// 32 pairs (lse, D) from p to LDS, to + at, past `left` of them zero; by a whole wave.
__device__ __forceinline__ void row_load(float *to, int at, const float *p, int left) {
  const int n = left < 0 ? 0 : left > 32 ? 32 : left;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float *>(reinterpret_cast<const float *>(
          uniform(reinterpret_cast<const uint16_t *>(p)))),
      (short)0, uniform(n * 8), 0x00027000);
  // (`at` once it is LDS: of a constant place past an array's first this compiler makes
  // a comparison that it cannot encode)
  __attribute__((address_space(3))) float *const lds =
      (__attribute__((address_space(3))) float *)to;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      rsrc, (__attribute__((address_space(3))) void *)(lds + at), 4, lane_id() * 4, 0, 0, 0);
}

// Tiles of queries that key tile `part` of a sequence meets: the first, and how many.
template <int DP, bool W>
__device__ __forceinline__ Span tile_queries(const PromptArgs &a, const Span &sq, const Span &sk,
                                             int part) {
  const int lead = sk.count - sq.count;
  const int begin = a.causal ? clamp_to(part * kHeld - lead, 0, sq.count) : 0;
  int past = sq.count;  // the last query that sees one, and one more
  if (W && part * kHeld >= a.sinks) {
    const int last = (part * kHeld + kHeld < sk.count ? part * kHeld + kHeld : sk.count) - 1;
    past = clamp_to(last - lead + a.window, begin, sq.count);
  }
  const int first = begin / kStep(DP), end = (past + kStep(DP) - 1) / kStep(DP);
  return {first, end - first};
}
// Blocks that share the tile: as many as bring each to a.split_steps steps of 32
// queries or fewer, at most a.splits.
template <int DP, bool W>
__device__ __forceinline__ int tile_splits(const PromptArgs &a, const Span &sq, const Span &sk,
                                           int part) {
  const int steps = tile_queries<DP, W>(a, sq, sk, part).count * a.group * (kStep(DP) / 32);
  return clamp_to((steps + a.split_steps - 1) / a.split_steps, 1, a.splits);
}

// Through a window the sinks' key tiles meet every query. Of a sequence whose first tile
// has the steps for more blocks than other tiles have, such tiles are shared by blocks of
// their own, `blocks` each: slots, counted through the sequences, their tiles, and a
// tile's blocks. tiles 0: none are.
struct Sinks {
  int tiles, blocks;
};
template <int DP>
__device__ __forceinline__ Sinks sinks_of(const PromptArgs &a, const Span &sq, const Span &sk) {
  if (a.sink_tiles == 0) return {0, 0};
  const int steps = tile_queries<DP, true>(a, sq, sk, 0).count * a.group * (kStep(DP) / 32);
  int blocks = (steps + (1 << a.sink_shift) - 1) >> a.sink_shift;
  if (blocks <= a.splits) return {0, 0};
  if (blocks > a.sink_most) blocks = a.sink_most;
  const int tiles = tiles_of(sk.count, kHeld);
  return {tiles < a.sink_tiles ? tiles : a.sink_tiles, blocks};
}
// Of the sequences' slots, or of their shared tiles, the one numbered `at`: its sequence and
// tile, and the tile's first slot; false past the last. By whole waves.
template <int DP, bool kSlots>
__device__ __forceinline__ bool find_sink(const PromptArgs &a, int at, Span &sk, Span &sq,
                                          int &seq, int &part, int &slot, int &blocks) {
  const int lane = lane_id();
  int before = 0;  // slots of the sequences so far
  for (int base = 0; base < a.n_seqs && before < a.sink_slots; base += OPA_WAVE) {
    const int b = base + lane < a.n_seqs ? base + lane : a.n_seqs - 1;
    const Span k = span_of(a.cu_k, b, a.n_k), q = span_of(a.cu_q, b, a.n_q);
    const Sinks x = base + lane < a.n_seqs ? sinks_of<DP>(a, q, k) : Sinks{0, 0};
    const int slots = x.tiles * x.blocks, past = wave_sums(slots);
    const int n = kSlots ? slots : x.tiles, inc = kSlots ? past : wave_sums(n);
    const uint64_t m = __ballot(inc > at);
    if (m) {
      const int w = __ffsll((unsigned long long)m) - 1;
      const auto from = [&](int v) { return __builtin_amdgcn_readlane(v, w); };
      sk = {from(k.first), from(k.count)};
      sq = {from(q.first), from(q.count)};
      seq = base + w;
      blocks = from(x.blocks);
      at -= from(inc - n);
      part = kSlots ? at / blocks : at;
      slot = before + from(past - slots) + part * blocks;
      return slot + blocks <= a.sink_slots;  // (offsets that overlap may ask for more)
    }
    at -= __builtin_amdgcn_readlane(inc, OPA_WAVE - 1);
    before += __builtin_amdgcn_readlane(past, OPA_WAVE - 1);
  }
  return false;
}

// A split's steps of a tile: a head's tiles of queries, then the next head's.
struct Steps {
  int first, past;
};
template <bool W>
__device__ __forceinline__ Steps split_steps(int all, int split, int splits) {
  if constexpr (W) {  // (one division for all of a tile's splits)
    const int each = all / splits, more = all - each * splits;
    const int first = split * each + (split < more ? split : more);
    return {first, first + each + (split < more)};
  }
  return {(int)((int64_t)all * split / splits), (int)((int64_t)all * (split + 1) / splits)};
}

// The queries that see a key of the 32 from key0 on, through a window.
struct Met {
  int first, past;
  __device__ __forceinline__ Met(const PromptArgs &a, const Span &sq, int lead, int key0)
      : first(clamp_to(key0 - lead, 0, sq.count)),
        past(key0 < a.sinks ? sq.count : key0 + 31 - lead + a.window) {}
};
// Whether a split has one: a wave without leaves no part.
template <int DP>
__device__ __forceinline__ bool split_meets(const Met &m, const Span &tiles, const Steps &s) {
  const int lo = m.first / kStep(DP) - tiles.first;
  const int hi = (m.past + kStep(DP) - 1) / kStep(DP) - tiles.first;
  for (int g = s.first / tiles.count; g * tiles.count < s.past; ++g) {
    const int from = g * tiles.count + (lo > 0 ? lo : 0);
    const int to = g * tiles.count + (hi < tiles.count ? hi : tiles.count);
    if ((from > s.first ? from : s.first) < (to < s.past ? to : s.past)) return true;
  }
  return false;
}

// Where a wave of one of a tile's blocks leaves its dk and dv, as its registers hold
// them: [parts][n_kv][waves][dk, dv][DP / 8][64 lanes] of four values, the parts
// [splits][tiles], none where splits is 1, and then the slots of the sinks' tiles.
template <int DP>
__device__ __forceinline__ f32x4 *part_at(const PromptArgs &a, int64_t at, int hk, int wave) {
  at = (at * a.n_kv + hk) * kGradWaves + wave;
  return reinterpret_cast<f32x4 *>(a.part) + at * (2 * DP / 8 * OPA_WAVE) + lane_id();
}
__device__ __forceinline__ int64_t tile_part(const PromptArgs &a, int split, int tile) {
  return split * (a.n_k / kHeld + (int64_t)a.n_seqs) + tile;
}
__device__ __forceinline__ int64_t sink_part(const PromptArgs &a, int slot) {
  return (a.splits > 1 ? tile_part(a, a.splits, 0) : 0) + slot;
}

// dk and dv of 32 keys a wave: S = Q K^T with the wave's keys as columns, so
// that a lane holds one key; P and dS then are the B operands of
// dv^T = dout^T P and dk^T = q^T dS.
template <class E, int DP, bool W>
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
  Span sq, sk;
  int part, seq, split;
  // W: past the blocks of every tile those of the sinks' tiles
  const int64_t past_tiles = W ? id - tile_part(a, a.splits, 0) : -1;
  int splits;
  int64_t place;  // of this block's part
  if (past_tiles >= 0) {
    int slot;
    if (!find_sink<DP, true>(a, (int)past_tiles, sk, sq, seq, part, slot, splits)) return;
    split = (int)past_tiles - slot;
    place = sink_part(a, (int)past_tiles);
  } else {
    split = id % a.splits;
    const int tile = id / a.splits;
    if (!find_tile(a.cu_k, a.n_k, a.cu_q, a.n_q, a.n_seqs, kHeld, tile, sk, sq, part, &seq))
      return;
    if (W && part < sinks_of<DP>(a, sq, sk).tiles) return;
    splits = tile_splits<DP, W>(a, sq, sk, part);
    place = tile_part(a, split, tile);
  }
  const int lead = sk.count - sq.count;
  const int key0 = part * kHeld + wave * 32, key = key0 + r;
  const bool live = key < sk.count;
  // the first query that sees every key of this wave, and the first that sees
  // this lane's
  const int whole = key0 + 32 > sk.count ? sq.count
                                         : a.causal ? clamp_to(key0 + 31 - lead, 0, sq.count) : 0;
  // (W: the query whose own key it is, or what no query is)
  const int from = W      ? (live ? key - lead : 1 << 30)
                   : live ? (a.causal ? clamp_to(key - lead, 0, sq.count) : 0)
                          : sq.count;
  // W: the first query that has left one of this wave's keys behind
  const int plain = key0 > a.sinks ? key0 : a.sinks;  // the wave's first key that is no sink
  const int left_from = W && plain < key0 + 32 ? plain - lead + a.window : sq.count;
  const Met mine(a, sq, lead, key0);
  const Span met = tile_queries<DP, W>(a, sq, sk, part);
  const int t0 = met.first, per = met.count;
  const int all = per * a.group;
  if (split >= splits) return;
  const Steps part_steps = split_steps<W>(all, split, splits);
  const int first = part_steps.first, steps = part_steps.past;
  const float up = Scales<E>::ds(a, seq, sq, sk, hk * a.group, a.group, hk);
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
        row_load(rows, 64 * b, a.rows + ((int64_t)head * a.n_q + tok + 32 * b) * 2, left - 32 * b);
  };
  const auto step = [&](const uint16_t *q, const uint16_t *dout, const float *rows, int t)
                        __attribute__((always_inline)) {
    const int q0 = (t0 + t % per) * kStepQ;
    if (W && (q0 >= mine.past || q0 + kStepQ <= mine.first || key0 >= sk.count)) return;
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
      if constexpr (W) {  // as hide_keys, of the queries
        const int at = q0 + 32 * qb;
        if (at < whole || at + 32 > left_from) {
          const int past = at + 4 * h - fresh(from);
          const uint32_t span = key0 + r < a.sinks ? INT_MAX : a.window;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if ((uint32_t)(past + 8 * (e >> 2) + (e & 3)) >= span) x[e] = y[e] = 0.f;
        }
      } else if (q0 < whole) {
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
    if (W && !split_meets<DP>(mine, met, part_steps)) return;
    f32x4 *p = part_at<DP>(a, place, hk, wave);
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
  uint16_t *const room = (wave / kFit == 0 ? tq0 : wave / kFit == 1 ? tq1
                                                 : wave / kFit == 2 ? td0
                                                                    : td1) +
                         wave % kFit * 32 * DP;
  const int64_t tok = sk.first + key0;
  store_rows<E, DP>(room, dk, fk, a.dk.p + tok * a.dk.ts + (int64_t)hk * a.dk.hs, a.dk.ts,
                    sk.count - key0, a.head_dim);
  store_rows<E, DP>(room, dv, fv, a.dv.p + tok * a.dv.ts + (int64_t)hk * a.dv.hs, a.dv.ts,
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
  int part, seq;
  if (!find_tile(a.cu_k, a.n_k, a.cu_q, a.n_q, a.n_seqs, kHeld, tile, sk, sq, part, &seq)) return;
  const int splits = tile_splits<DP, false>(a, sq, sk, part);
  const int key0 = part * kHeld + wave * 32;
  if (splits == 1 || key0 >= sk.count) return;
  f32x16 sum[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) sum[d] = (f32x16)(0.f);
  for (int k = 0; k < splits; ++k) {
    const f32x4 *p =
        part_at<DP>(a, tile_part(a, k, tile), hk, wave) + which * 4 * DB * OPA_WAVE;
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

// The same through a window: the sinks' tiles first, of which there are few and of many
// parts, then, where tiles are split, all the others. A wave takes 32 columns of dk or dv
// of 32 keys, with several parts' loads on their way: 12 documents' sinks 10 us (25 by
// whole rows, one part after another), 4 of up to 2000, window 2000, 19 us and not 24, one
// of 521, 8 heads on 1 of 64, 10 and not 13; where all of many tiles are split whole rows
// are read faster (12 documents, window 8192, 40 us and not 49).
template <class E, int DP>
__global__ __launch_bounds__(2 * kGradWaves * OPA_WAVE) void k_window_sum(PromptArgs a) {
  constexpr int DB = DP / 32;
  const int lane = lane_id(), r = lane & 31, h = lane >> 5;
  const int all = uniform(wave_id()), wave = all / 2, which = all % 2;
  int id = blockIdx.x;
  const int hk = id % a.n_kv;
  id /= a.n_kv;
  const int d = id % DB;
  int tile = id / DB, seq, part, splits;
  Span sq, sk;
  int64_t place, step = 1;  // of the tile's first part, and to its next
  if (tile < a.sink_sums) {
    int slot;
    if (!find_sink<DP, false>(a, tile, sk, sq, seq, part, slot, splits)) return;
    place = sink_part(a, slot);
  } else {
    tile -= a.sink_sums;
    if (!find_tile(a.cu_k, a.n_k, a.cu_q, a.n_q, a.n_seqs, kHeld, tile, sk, sq, part, &seq))
      return;
    if (part < sinks_of<DP>(a, sq, sk).tiles) return;
    splits = tile_splits<DP, true>(a, sq, sk, part);
    place = tile_part(a, 0, tile);
    step = tile_part(a, 1, 0);
  }
  const int key0 = part * kHeld + wave * 32;
  if (splits == 1 || key0 >= sk.count) return;
  const Met mine(a, sq, sk.count - sq.count, key0);
  const Span met = tile_queries<DP, true>(a, sq, sk, part);
  f32x4 sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = (f32x4)(0.f);
  constexpr int kAhead = 4;
  for (int k0 = 0; k0 < splits; k0 += kAhead) {
    f32x4 v[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool there =
          k0 + k < splits &&
          split_meets<DP>(mine, met, split_steps<true>(met.count * a.group, k0 + k, splits));
      const f32x4 *p =
          part_at<DP>(a, place + (k0 + k) * step, hk, wave) + (which * 4 * DB + 4 * d) * OPA_WAVE;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k][i] = there ? p[i * OPA_WAVE] : (f32x4)(0.f);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += v[k][i];
  }
  const Rows &o = which ? a.dv : a.dk;
  uint16_t *row = o.p + (int64_t)(sk.first + key0 + r) * o.ts + (int64_t)hk * o.hs;
  if (key0 + r >= sk.count) return;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int col = 32 * d + 8 * g + 4 * h;
    if (col < a.head_dim)
      *reinterpret_cast<u32x2 *>(row + col) =
          u32x2{E::pack(sum[g][0], sum[g][1]), E::pack(sum[g][2], sum[g][3])};
  }
}

template <class E, int DP, bool W>
static void launch(const PromptArgs &a, hipStream_t s) {
  const int hs = W ? a.head_shift : 0;
  const int64_t kt = (int64_t)a.n_k / kHeld + a.n_seqs;
  const int64_t qt = ((int64_t)a.n_q / (kHeld >> hs) + a.n_seqs) * (a.n_heads >> hs);
  const dim3 block(kGradWaves * OPA_WAVE);
  const dim3 rows((uint32_t)qt);
  const bool many = a.n_k >= (int64_t)kManyKeys * a.n_seqs &&
                    (!W || (int64_t)a.window + a.sinks >= kManyKeys);
  if (a.n_q > 0 && qt <= kFewBlocks && many)
    hipLaunchKernelGGL((k_attn_dq<E, DP, 2, W>), rows, dim3(2 * kGradWaves * OPA_WAVE), 0, s, a);
  else if (a.n_q > 0)
    hipLaunchKernelGGL((k_attn_dq<E, DP, 1, W>), rows, block, 0, s, a);
  if (a.n_k == 0) return;
  const int64_t parts = kt * a.splits + a.sink_slots;
  hipLaunchKernelGGL((k_attn_dkv<E, DP, W>), dim3((uint32_t)(parts * a.n_kv)), block, 0, s, a);
  const dim3 twice(2 * kGradWaves * OPA_WAVE);
  if constexpr (W) {
    const int64_t sums = ((a.splits > 1 ? kt : 0) + a.sink_sums) * (DP / 32) * a.n_kv;
    if (sums > 0)
      hipLaunchKernelGGL((k_window_sum<E, DP>), dim3((uint32_t)sums), twice, 0, s, a);
  } else if (a.splits > 1) {
    hipLaunchKernelGGL((k_dkv_sum<E, DP>), dim3((uint32_t)(kt * a.n_kv)), twice, 0, s, a);
  }
}

template <class E>
static void grad(const PromptArgs &a, hipStream_t s) {
  if (a.norms && (a.n_q > 0 || a.n_k > 0))
    hipLaunchKernelGGL(k_attn_norms, dim3(a.norm_slots, a.n_heads + a.n_kv), dim3(kNormThreads), 0,
                       s, a);
  if (a.window)
    a.head_dim <= 64 ? launch<E, 64, true>(a, s) : launch<E, 128, true>(a, s);
  else
    a.head_dim <= 64 ? launch<E, 64, false>(a, s) : launch<E, 128, false>(a, s);
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

static int most_splits(int64_t n) { return n < 1 ? 1 : n > 16 ? 16 : (int)n; }
static GradSplits causal_splits(int64_t n_q, int64_t n_k, int n_seqs, int group, int n_kv) {
  const int64_t blocks = (n_k / kHeld + n_seqs) * n_kv;
  GradSplits x{1, kSplitSteps, 0, 0, 0, 0, 0};
  const int64_t steps = n_q * group / 32 / n_seqs;
  if (blocks <= kFewTiles && steps >= kSplitSteps) x.steps = kFewSteps;
  const int64_t n = (2048 + blocks - 1) / blocks;
  x.most = most_splits(n < steps / x.steps ? n : steps / x.steps);
  return x;
}

// Through a window shorter than the sequences a key tile meets as many queries as any
// other, and partial sums cost more than they gain where the tiles fill the chip: they
// are split only to come to kRound blocks, by the longest sequence that there may be (a
// short one's tiles are split by their steps). A window as long as the mean sequence
// leaves the first tiles the most, as the causal mask does. 12 documents of up to 4001,
// 16 heads on 4 of 128, 608 blocks: through 1024 tokens dk and dv 278 us unsplit, 302 by
// the causal rule, sums included; through 2048 449 and 370, through 4096 706 and 408; one
// of 16000: through 4096 986 and 1018, through all 3315 and 2070.
//
// The sinks' tiles meet every query: where that is more than a block is to have, they are
// shared by blocks of 2^sink_shift steps, kMostSinks more than other tiles have at most, and
// of all key heads about kSinkBlocks at most, which begin last. Their room goes by the
// steps that there are, as the slots are counted through the sequences that have them: of
// 32 steps it is about half of the queries' own. dk and dv with the sums: 12 documents,
// window 512, 4 sinks, 190 us by 16 steps, 191 by 32, 214 by 64; 6 documents of 16 key heads
// 84, 101 and 144; with 300 sinks 12 documents 270, 245 and 263. Where tiles are few, by 8
// and by 32 steps: one of 4000 74 and 86 us, 3 of up to 609, one key head, 22 and 33.
constexpr int kRound = 512, kMostSinks = 31, kSinkBlocks = 2048, kSinkShift = 5, kFewShift = 3;
constexpr int64_t kManyBlocks = 1 << 16;  // past these more blocks say nothing (and one launch
                                          // takes as many)
static GradSplits window_splits(int64_t n_q, int64_t n_k, int n_seqs, int group, int n_kv,
                                int window, int sinks) {
  const int64_t blocks = (n_k / kHeld + n_seqs) * n_kv;
  GradSplits x{1, kSplitSteps, 0, 0, 0, 0, 0};
  const int64_t met = n_q < (int64_t)window + kHeld ? n_q : (int64_t)window + kHeld;
  const int64_t steps = (met * group + 31) / 32;
  x.most = most_splits(kRound / blocks < steps / kFewSteps ? kRound / blocks : steps / kFewSteps);
  const int64_t each = (steps + x.most - 1) / x.most;
  if (x.most > 1 || each > kSplitSteps) x.steps = (int)(each < kFewSteps ? kFewSteps : each);
  if (window >= n_q / n_seqs) {  // the mean length
    const GradSplits y = causal_splits(n_q, n_k, n_seqs, group, n_kv);
    if (y.most > x.most) return y;  // (the sinks' tiles are then like the first ones)
  }
  if (!sinks || blocks >= kManyBlocks) return x;
  const int64_t tiles = ((sinks < n_k ? sinks : n_k) + kHeld - 1) / kHeld;  // of a sequence
  int shift = blocks <= kFewTiles ? kFewShift : kSinkShift;
  // A sequence of n queries has (n + kMostEnd) group / 32 steps at most; to share its tiles
  // it has more than 2^shift, so that not every sequence of a batch can
  constexpr int64_t kMostEnd = 63;
  int64_t least = ((int64_t)32 << shift) / group - kMostEnd;
  if (least < 1) least = 1;
  const int64_t seqs = n_q / least < n_seqs ? n_q / least : n_seqs;
  const int64_t all = tiles * ((n_q + kMostEnd * seqs) * group / 32 + 1);  // steps, of them
  while (all >> shift > kSinkBlocks / n_kv) ++shift;
  if (shift > 30) return x;  // (no tile has as many steps)
  // of S = ceil(steps / 2^shift) blocks, more than one: less than 2 steps / 2^shift, and
  // than steps / 2^shift + 1
  const int64_t held = std::min(seqs * tiles, n_k / kHeld + seqs);
  const int64_t slots = std::min(std::min(2 * all >> shift, (all >> shift) + held),
                                 held * (x.most + kMostSinks));
  const int64_t most = ((n_q + kMostEnd) * group / 32 + (1 << shift)) >> shift;  // of a tile
  if (most <= x.most || slots <= x.most) return x;
  x.sink_tiles = (int)tiles;
  x.sink_shift = shift;
  x.sink_most = x.most + kMostSinks;
  x.sink_slots = (int)slots;
  x.sink_sums = (int)std::min(held, slots / (x.most + 1));
  return x;
}

int64_t grad_parts(const GradSplits &x, int64_t n_k, int n_seqs) {
  return (x.most > 1 ? x.most * (n_k / kHeld + n_seqs) : 0) + x.sink_slots;
}

GradSplits grad_splits(int64_t n_q, int64_t n_k, int n_seqs, int n_heads, int n_kv, int window,
                       int sinks) {
  if (n_seqs == 0 || n_k == 0) return {1, kSplitSteps, 0, 0, 0, 0, 0};
  const int group = n_heads / n_kv;
  return window ? window_splits(n_q, n_k, n_seqs, group, n_kv, window, sinks)
                : causal_splits(n_q, n_k, n_seqs, group, n_kv);
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
