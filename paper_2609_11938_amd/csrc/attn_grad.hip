// Gradient of attention over whole prompts (opattr_attn_prompt_grad).
//
// Three launches. k_attn_delta: D_i = dout_i . out_i, and for float16 the
// largest norms of dout's and v's rows. k_attn_dkv: a wave holds 32 keys of one
// key head, and dk and dv of them, and passes over the queries that see them of
// every query head of the group. k_attn_dq: a wave holds 32 queries and passes
// over their keys. Each recomputes the weights from lse; every sum has one
// owner and one order, so runs repeat bit for bit.
#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kGradWaves = 4;
constexpr int kHeld = 32 * kGradWaves;  // keys (queries) a block holds
constexpr int kStepQ = 32;              // queries a tile of the dk/dv pass
constexpr int kStepK = 64;              // keys a tile of the dq pass

// Weights and their gradients are rounded to 16 bits for the products. For
// float16 both are scaled by powers of two first: the weights by 2^kWeight, and
// ds by 2^e with |ds| <= 2 |dout_i| |v_j|, so that its largest stays below
// 2^15 and small ones keep their bits.
template <class E>
struct Scales {
  static constexpr float kWeight = 0.f;
  static __device__ __forceinline__ float ds(const uint32_t *, int) { return 1.f; }
};
template <>
struct Scales<F16> {
  static constexpr float kWeight = 10.f;
  static __device__ __forceinline__ float ds(const uint32_t *norms, int hk) {
    const float most = sqrtf(__uint_as_float(norms[2 * hk])) *
                       sqrtf(__uint_as_float(norms[2 * hk + 1]));
    if (!(most > 0.f) || !(most < 1e30f)) return 1.f;
    int e;
    frexpf(most, &e);  // most < 2^e
    return ldexpf(1.f, clamp_to(14 - e, -100, 100));
  }
};

// D_i, 4 lanes a row, and the largest squared norms of dout's and v's rows (the
// bits of non-negative floats order as integers, so the maximum is the same in
// any order). A block takes kDeltaRows rows of one head: blockIdx.y is a query
// head, and past those a key head whose values are only measured.
constexpr int kDeltaRows = 512;
template <class E>
__global__ __launch_bounds__(256) void k_attn_delta(PromptArgs a) {
  __shared__ float most[4];
  const int sub = threadIdx.x & 3;
  const bool q = (int)blockIdx.y < a.n_heads;
  const int head = q ? blockIdx.y : blockIdx.y - a.n_heads;
  const int n = q ? a.n_q : a.n_k;
  const Rows x = q ? a.dout : a.v;
  float top = 0.f;
  for (int64_t t = (int64_t)blockIdx.x * kDeltaRows + (threadIdx.x >> 2);
       t < n && t < ((int64_t)blockIdx.x + 1) * kDeltaRows; t += 64) {
    const uint16_t *px = x.p + t * x.ts + (int64_t)head * x.hs;
    const uint16_t *py = q ? a.out.p + t * a.out.ts + (int64_t)head * a.out.hs : px;
    float dot = 0.f, norm = 0.f;
    for (int c = sub * 8; c < a.head_dim; c += 32) {
      const s16x8 u = *reinterpret_cast<const s16x8 *>(px + c);
      const s16x8 w = *reinterpret_cast<const s16x8 *>(py + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = E::widen((uint16_t)u[i]);
        dot = fmaf(f, E::widen((uint16_t)w[i]), dot);
        norm = fmaf(f, f, norm);
      }
    }
    dot += __shfl_xor(dot, 1);
    dot += __shfl_xor(dot, 2);
    norm += __shfl_xor(norm, 1);
    norm += __shfl_xor(norm, 2);
    if (q && sub == 0) a.delta[(int64_t)head * a.n_q + t] = dot;
    top = fmaxf(top, norm);
  }
  if (!a.norms) return;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane_id() == 0) most[wave_id()] = top;
  __syncthreads();
  if (threadIdx.x == 0)
    atomicMax(&a.norms[2 * (q ? head / a.group : head) + !q],
              __float_as_uint(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]))));
}

__global__ void k_attn_zero(uint32_t *p, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0;
}

// dk and dv of 32 keys a wave: S = Q K^T with the wave's keys as columns, so
// that a lane holds one key; P and dS then are the B operands of
// dv^T = dout^T P and dk^T = q^T dS.
template <class E, int DP>
__global__ __launch_bounds__(kGradWaves * OPA_WAVE, 2) void k_attn_dkv(PromptArgs a) {
  constexpr int KS = DP / 16, DB = DP / 32;
  __shared__ __align__(16) uint16_t tq[2][kStepQ * DP], td[2][kStepQ * DP];
  __shared__ __align__(16) float tl[2][kStepQ], tD[2][kStepQ];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 31, h = lane >> 5;
  const int hk = blockIdx.x % a.n_kv;
  int seq, part;
  if (blockIdx.x == 0) {
    check_spans(a.cu_q, a.n_seqs, a.n_q, a.diag);
    check_spans(a.cu_k, a.n_seqs, a.n_k, a.diag);
  }
  if (!find_tile(a.cu_k, a.n_seqs, a.n_k, kHeld, blockIdx.x / a.n_kv, seq, part)) return;
  Span sq = span_of(a.cu_q, seq, a.n_q), sk = span_of(a.cu_k, seq, a.n_k);
  sq = {uniform(sq.first), uniform(sq.count)};
  sk = {uniform(sk.first), uniform(sk.count)};
  const int lead = sk.count - sq.count;
  const int key0 = part * kHeld + wave * 32, key = key0 + r;
  const bool live = key < sk.count;
  // the first query that sees a key of the block, and the first that sees this
  // lane's
  const int begin = a.causal ? clamp_to(part * kHeld - lead, 0, sq.count) : 0;
  const int from = live ? (a.causal ? clamp_to(key - lead, 0, sq.count) : 0) : sq.count;
  const int t0 = begin / kStepQ, t1 = (sq.count + kStepQ - 1) / kStepQ;
  const int per = t1 - t0, steps = per > 0 ? per * a.group : 0;
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
  const float up = Scales<E>::ds(a.norms, hk);
  const float fv = exp2_fast(-Scales<E>::kWeight), upw = up * fv;
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = dv[d] = (f32x16)(0.f);

  const auto load = [&](int step, int b) {
    const int head = hk * a.group + step / per, q0 = (t0 + step % per) * kStepQ;
    const int64_t tok = sq.first + q0;
    tile_load<DP, kStepQ, kGradWaves>(tq[b], a.q.p + tok * a.q.ts + (int64_t)head * a.q.hs,
                                      a.q.ts, sq.count - q0, a.head_dim, wave);
    tile_load<DP, kStepQ, kGradWaves>(td[b],
                                      a.dout.p + tok * a.dout.ts + (int64_t)head * a.dout.hs,
                                      a.dout.ts, sq.count - q0, a.head_dim, wave);
    // a query that is not there, or sees nothing, has weights 0: exp2(x - inf)
    if (threadIdx.x < 2 * kStepQ) {
      const int i = threadIdx.x & (kStepQ - 1), q = q0 + i;
      const int64_t at = (int64_t)head * a.n_q + tok + i;
      if (threadIdx.x < kStepQ) {
        float s = q < sq.count ? a.lse[at] * kLog2e - Scales<E>::kWeight : INFINITY;
        tl[b][i] = s == -INFINITY ? INFINITY : s;
      } else {
        tD[b][i] = q < sq.count ? a.delta[at] : 0.f;
      }
    }
  };
  if (steps > 0) load(0, 0);
  for (int t = 0; t < steps; ++t) {
    wait_loads();
    block_sync();
    const int b = t & 1, q0 = (t0 + t % per) * kStepQ;
    if (t + 1 < steps) load(t + 1, b ^ 1);
    f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      x = E::mfma(nat_frag<DP>(tq[b], r, 2 * s + h), kf[s], x);
      y = E::mfma(nat_frag<DP>(td[b], r, 2 * s + h), vf[s], y);
    }
    s16x8 pf[2], sf[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 wp, ws;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int q = 16 * s + 8 * g + 4 * h;
        const f32x4 L = *reinterpret_cast<const f32x4 *>(&tl[b][q]);
        const f32x4 D = *reinterpret_cast<const f32x4 *>(&tD[b][q]);
        float p[4], ds[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 8 * s + 4 * g + i;
          p[i] = exp2_fast(fmaf(x[e], c, -L[i]));
          ds[i] = p[i] * (y[e] - D[i]) * upw;
          if (q0 + q + i < from) p[i] = ds[i] = 0.f;
        }
        wp[2 * g] = E::pack(p[0], p[1]);
        wp[2 * g + 1] = E::pack(p[2], p[3]);
        ws[2 * g] = E::pack(ds[0], ds[1]);
        ws[2 * g + 1] = E::pack(ds[2], ds[3]);
      }
      pf[s] = __builtin_bit_cast(s16x8, wp);
      sf[s] = __builtin_bit_cast(s16x8, ws);
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        dv[d] = E::mfma(tr_frag<DP>(td[b], 16 * s, d), pf[s], dv[d]);
        dk[d] = E::mfma(tr_frag<DP>(tq[b], 16 * s, d), sf[s], dk[d]);
      }
  }
  if (!live) return;
  const float fk = a.scale / up;
  uint16_t *kp = a.dk.p + (int64_t)(sk.first + key) * a.dk.ts + (int64_t)hk * a.dk.hs;
  uint16_t *vp = a.dv.p + (int64_t)(sk.first + key) * a.dv.ts + (int64_t)hk * a.dv.hs;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * d + 8 * g + 4 * h;
      if (col >= a.head_dim) continue;
      const u32x2 w = {E::pack(dk[d][4 * g] * fk, dk[d][4 * g + 1] * fk),
                       E::pack(dk[d][4 * g + 2] * fk, dk[d][4 * g + 3] * fk)};
      const u32x2 u = {E::pack(dv[d][4 * g] * fv, dv[d][4 * g + 1] * fv),
                       E::pack(dv[d][4 * g + 2] * fv, dv[d][4 * g + 3] * fv)};
      *reinterpret_cast<u32x2 *>(kp + col) = w;
      *reinterpret_cast<u32x2 *>(vp + col) = u;
    }
}

// dq of 32 queries a wave: S^T = K Q^T with the wave's queries as columns;
// dS^T then is the B operand of dq^T = K^T dS^T.
template <class E, int DP>
__global__ __launch_bounds__(kGradWaves * OPA_WAVE, 2) void k_attn_dq(PromptArgs a) {
  constexpr int KS = DP / 16, DB = DP / 32;
  __shared__ __align__(16) uint16_t tk[2][kStepK * DP], tv[2][kStepK * DP];
  const int lane = lane_id(), wave = uniform(wave_id());
  const int r = lane & 31, h = lane >> 5;
  int id = blockIdx.x;
  const int hk = id % a.n_kv;
  id /= a.n_kv;
  const int head = hk * a.group + id % a.group;
  int seq, part;
  if (!find_tile(a.cu_q, a.n_seqs, a.n_q, kHeld, id / a.group, seq, part)) return;
  Span sq = span_of(a.cu_q, seq, a.n_q), sk = span_of(a.cu_k, seq, a.n_k);
  sq = {uniform(sq.first), uniform(sq.count)};
  sk = {uniform(sk.first), uniform(sk.count)};
  const int q0 = ((sq.count + kHeld - 1) / kHeld - 1 - part) * kHeld;
  const int lead = sk.count - sq.count;
  const int qrow = q0 + wave * 32 + r;
  const bool live = qrow < sq.count;
  const int last = (q0 + kHeld < sq.count ? q0 + kHeld : sq.count) - 1;
  const int keys = a.causal ? clamp_to(last + lead + 1, 0, sk.count) : sk.count;
  const int tiles = (keys + kStepK - 1) / kStepK;
  const int seen = live ? (a.causal ? clamp_to(qrow + lead + 1, 0, sk.count) : sk.count) : 0;
  s16x8 qf[KS], df[KS];
  float L = INFINITY, D = 0.f;
  {
    const int64_t tok = sq.first + (live ? qrow : 0);
    const uint16_t *qp = a.q.p + tok * a.q.ts + (int64_t)head * a.q.hs;
    const uint16_t *dp = a.dout.p + tok * a.dout.ts + (int64_t)head * a.dout.hs;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = (s16x8)(0);
      df[s] = (s16x8)(0);
      if (live && 16 * s + 8 * h < a.head_dim) {
        qf[s] = *reinterpret_cast<const s16x8 *>(qp + 16 * s + 8 * h);
        df[s] = *reinterpret_cast<const s16x8 *>(dp + 16 * s + 8 * h);
      }
    }
    if (live) {
      const int64_t at = (int64_t)head * a.n_q + tok;
      L = a.lse[at] * kLog2e;
      if (L == -INFINITY) L = INFINITY;
      D = a.delta[at];
    }
  }
  const uint16_t *kp = a.k.p + (int64_t)sk.first * a.k.ts + (int64_t)hk * a.k.hs;
  const uint16_t *vp = a.v.p + (int64_t)sk.first * a.v.ts + (int64_t)hk * a.v.hs;
  const float c = a.scale * kLog2e;
  const float up = Scales<E>::ds(a.norms, hk);
  f32x16 dq[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dq[d] = (f32x16)(0.f);
  if (tiles > 0) {
    tile_load<DP, kStepK, kGradWaves>(tk[0], kp, a.k.ts, sk.count, a.head_dim, wave);
    tile_load<DP, kStepK, kGradWaves>(tv[0], vp, a.v.ts, sk.count, a.head_dim, wave);
  }
  for (int t = 0; t < tiles; ++t) {
    wait_loads();
    block_sync();
    const int k0 = t * kStepK, b = t & 1;
    if (t + 1 < tiles) {
      tile_load<DP, kStepK, kGradWaves>(tk[b ^ 1], kp + (int64_t)(k0 + kStepK) * a.k.ts, a.k.ts,
                                        sk.count - k0 - kStepK, a.head_dim, wave);
      tile_load<DP, kStepK, kGradWaves>(tv[b ^ 1], vp + (int64_t)(k0 + kStepK) * a.v.ts, a.v.ts,
                                        sk.count - k0 - kStepK, a.head_dim, wave);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 x = (f32x16)(0.f), y = (f32x16)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        x = E::mfma(nat_frag<DP>(tk[b], 32 * kb + r, 2 * s + h), qf[s], x);
        y = E::mfma(nat_frag<DP>(tv[b], 32 * kb + r, 2 * s + h), df[s], y);
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float ds[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int e = 8 * s + 2 * i + j;
            const int key = k0 + 32 * kb + 8 * (e >> 2) + 4 * h + (e & 3);
            ds[j] = exp2_fast(fmaf(x[e], c, -L)) * (y[e] - D) * up;
            if (key >= seen) ds[j] = 0.f;
          }
          w[i] = E::pack(ds[0], ds[1]);
        }
        const s16x8 sf = __builtin_bit_cast(s16x8, w);
#pragma unroll
        for (int d = 0; d < DB; ++d)
          dq[d] = E::mfma(tr_frag<DP>(tk[b], 32 * kb + 16 * s, d), sf, dq[d]);
      }
    }
  }
  if (!live) return;
  const float f = a.scale / up;
  uint16_t *op = a.dq.p + (int64_t)(sq.first + qrow) * a.dq.ts + (int64_t)head * a.dq.hs;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * d + 8 * g + 4 * h;
      const u32x2 w = {E::pack(dq[d][4 * g] * f, dq[d][4 * g + 1] * f),
                       E::pack(dq[d][4 * g + 2] * f, dq[d][4 * g + 3] * f)};
      if (col < a.head_dim) *reinterpret_cast<u32x2 *>(op + col) = w;
    }
}

template <class E, int DP>
static void launch(const PromptArgs &a, hipStream_t s) {
  const int64_t kt = (int64_t)a.n_k / kHeld + a.n_seqs, qt = (int64_t)a.n_q / kHeld + a.n_seqs;
  const dim3 block(kGradWaves * OPA_WAVE);
  if (a.n_k > 0)
    hipLaunchKernelGGL((k_attn_dkv<E, DP>), dim3((uint32_t)(kt * a.n_kv)), block, 0, s, a);
  if (a.n_q > 0)
    hipLaunchKernelGGL((k_attn_dq<E, DP>), dim3((uint32_t)(qt * a.n_heads)), block, 0, s, a);
}

template <class E>
static void grad(const PromptArgs &a, hipStream_t s) {
  if (a.norms)
    hipLaunchKernelGGL(k_attn_zero, dim3((2 * a.n_kv + 63) / 64), dim3(64), 0, s, a.norms,
                       2 * a.n_kv);
  const int most = a.norms && a.n_k > a.n_q ? a.n_k : a.n_q;
  const dim3 grid((most + kDeltaRows - 1) / kDeltaRows, a.n_heads + (a.norms ? a.n_kv : 0));
  if (most > 0) hipLaunchKernelGGL((k_attn_delta<E>), grid, dim3(256), 0, s, a);
  if (a.head_dim <= 64)
    launch<E, 64>(a, s);
  else
    launch<E, 128>(a, s);
}

void run_prompt_grad(const PromptArgs &a, int dtype, hipStream_t s) {
  if (a.n_seqs == 0) return;
  if (dtype == OPATTR_BF16)
    grad<BF16>(a, s);
  else
    grad<F16>(a, s);
}

}  // namespace opa
