// Device parts shared by the attention kernels (gfx950, wave64): 16-bit
// element types and their matrix instructions, tiles in LDS, packed sequences.
//
// Matrix instruction used throughout: 32x32x16, D = A B + C. Lane l holds, with
// r = l % 32 and h = l / 32,
//   A[r][8h .. 8h+7], B[8h .. 8h+7][r], and D[8g + 4h + i][r] as element 4g + i.
// The order of the 16 contracted values is free as long as A and B agree, so a
// product's result feeds the next one without moving between lanes: of D's
// elements, 8 s .. 8 s + 7 (s = 0, 1) are rows 16 s + 4h + {0..3} and
// 16 s + 8 + 4h + {0..3} of column r, and B takes them as its eight values when
// A is loaded in that order (tr_frag).
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/opattr_attn.h"
#include "common.h"

namespace opa {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct BF16 {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  // Weights are exp2(x + kShift). float16 loses bits below 2^-14. bfloat16 values go
  // to float32's ends: weights of at most 2^(8 - 16) keep their sum in range while
  // |v| times the keys is below 2^136, and values of 2^-124 still have their bits
  // (with -24: of 2^-116).
  static constexpr float kShift = -16.f;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a),
                                                   __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a),
                                                   __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  // both rounded to nearest even
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const f32x2 f = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2));
  }
  static __device__ __forceinline__ float widen(uint16_t x) {
    return __uint_as_float((uint32_t)x << 16);
  }
};

struct F16 {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static constexpr float kShift = 6.f;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a),
                                                  __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a),
                                                  __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const f32x2 f = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2));
  }
  static __device__ __forceinline__ float widen(uint16_t x) {
    return (float)__builtin_bit_cast(_Float16, x);
  }
};

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) {
  return x < lo ? lo : x > hi ? hi : x;
}
// The same value in every lane, kept in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const uint16_t *uniform(const uint16_t *p) {
  const uint64_t x = (uint64_t)p;
  return (const uint16_t *)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 |
                            (uint32_t)uniform((int)x));
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The logarithm to base 2 of a weights' sum, without kShift (an exact product first:
// no bits are lost to a difference).
template <class E>
__device__ __forceinline__ float log2_sum(float l) {
  return log2f(l * exp2_fast(-E::kShift));
}

// Maximum and sum over a lane and its partner in the other half of the wave.
__device__ __forceinline__ float half_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// --------------------------------------------------------------------------
// Tiles in LDS: rows of DP 16-bit values (DP 64 or 128: head_dim rounded up,
// the rest zero), in 16-byte chunks. Chunk c of a row lies at place c ^
// swz(row), so that the reads below meet each bank once a cycle: along a
// column of chunks (nat_frag: 16 rows, one chunk) and across 4 rows by 4
// chunks (tr_frag).
// --------------------------------------------------------------------------
template <int DP>
__device__ __forceinline__ int swz(int row) {
  return DP == 128 ? ((row & 3) << 2) | ((row >> 2) & 3)
                   : ((row & 2) << 1) | ((row >> 2) & 3);
}

// Fragments. A lane's place in a tile is one offset (bytes), and the places it
// reads differ from it in bits that the swizzle leaves to an exclusive or:
//   nat_frag  row r of 32, values 16 s + 8 h .. + 7
//   tr_frag   column 32 db + l % 32 of rows 4h + {0..3} and 8 + 4h + {0..3}; the
//             transposing read gives lane i of 16 lanes the column i of four
//             rows, whose four 8-byte pieces lanes 4 r .. 4 r + 3 name
// `row0` is the first row, a multiple of 32 (nat_frag) or 16 (tr_frag).
template <int DP>
__device__ __forceinline__ int nat_place() {
  const int r = lane_id() & 31, h = lane_id() >> 5;
  return r * DP * 2 + ((h ^ swz<DP>(r)) << 4);
}
template <int DP>
__device__ __forceinline__ int tr_place() {
  const int l = lane_id(), i = l & 15;
  const int row = ((l >> 5) << 2) + (i >> 2), col = (l & 16) + ((i & 3) << 2);
  return row * DP * 2 + (((col >> 3) ^ swz<DP>(row)) << 4) + ((col & 4) << 1);
}
// Not a constant of a loop any more: the places above are cheaper to make again
// than to hold.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <int DP>
__device__ __forceinline__ s16x8 nat_frag(const uint16_t *tile, int place, int row0, int s) {
  return *reinterpret_cast<const s16x8 *>(reinterpret_cast<const char *>(tile) +
                                          row0 * DP * 2 + (place ^ (s << 5)));
}
template <int DP>
__device__ __forceinline__ s16x8 tr_frag(const uint16_t *tile, int place, int row0, int db) {
  typedef s16x4 __attribute__((address_space(3))) * lds4;
  const char *p = reinterpret_cast<const char *>(tile) + row0 * DP * 2;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + (place ^ (db << 6))));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds4)(p + 8 * DP * 2 + (place ^ (db << 6) ^ 32)));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ROWS rows from `src` (uniform; row stride `ts` elements, `left` rows exist,
// head_dim values each) into `tile`, by the NW waves of the block, straight to
// LDS. Rows and values that do not exist become zero: the buffer's range ends
// after `left` rows, and a chunk past head_dim asks past any range. The data is
// there after wait_loads() of every wave and a barrier. The compiler waits by
// itself before a read that may meet a load in flight, so that tiles used in
// turn have to be arrays of their own, each named where it is used.
template <int DP, int ROWS, int NW>
__device__ __forceinline__ void tile_load(uint16_t *tile, const uint16_t *src, int64_t ts,
                                          int left, int head_dim, int wave) {
  constexpr int C = DP / 8;  // chunks a row
  constexpr int N = ROWS * C / (NW * OPA_WAVE);
  static_assert(N * NW * OPA_WAVE == ROWS * C, "whole loads");
  const int n = left < 0 ? 0 : left > ROWS ? ROWS : left;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t *>(uniform(src)), (short)0, uniform((int)(n * ts * 2)), 0x00027000);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int first = (i * NW + wave) * OPA_WAVE;
    const int id = first + lane_id();
    const int row = id / C;
    const int chunk = (id % C) ^ swz<DP>(row);
    const uint32_t off = chunk * 8 < head_dim ? (uint32_t)(row * (int)ts * 2 + chunk * 16)
                                              : 0xfffffff0u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void *)(tile + first * 8), 16, (int)off, 0, 0,
        0);
  }
}

// 32 rows that a wave holds as columns (row l % 32 in lane l, values 32 d + 8 g +
// 4 h .. + 3 as elements 4 g .. of acc[d]), scaled and rounded, to rows of `out`,
// `left` of which exist: through the wave's own 32 * DP values of LDS, so that
// whole rows are written together (from the registers, 16 bytes of 32 rows a store:
// 16 prompts of 1024 tokens, head_dim 128: 111 us that way, 104 this).
template <class E, int DP>
__device__ __forceinline__ void store_rows(uint16_t *lds, const f32x16 (&acc)[DP / 32], float f,
                                           uint16_t *out, int64_t ts, int left, int head_dim) {
  constexpr int C = DP / 8;
  const int l = lane_id(), r = l & 31, h = l >> 5;
  char *const at = reinterpret_cast<char *>(lds);
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<u32x2 *>(at + r * DP * 2 + (((4 * d + g) ^ swz<DP>(r)) << 4) + h * 8) =
          u32x2{E::pack(acc[d][4 * g] * f, acc[d][4 * g + 1] * f),
                E::pack(acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f)};
#pragma unroll
  for (int i = 0; i < 32 * C / OPA_WAVE; ++i) {
    const int id = i * OPA_WAVE + l, row = id / C, c = id % C;
    const u32x4 v =
        *reinterpret_cast<const u32x4 *>(at + row * DP * 2 + ((c ^ swz<DP>(row)) << 4));
    if (row < left && c * 8 < head_dim)
      *reinterpret_cast<u32x4 *>(out + row * ts + c * 8) = v;
  }
}

// The wave's loads have arrived (also those straight to LDS). As the builtin, so
// that the compiler knows it too and does not wait again.
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  asm volatile("" ::: "memory");
}

// Barrier of the block after which every wave's LDS accesses before it are done.
__device__ __forceinline__ void block_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Tiles 0 .. n-1 through two buffers in turn, the next one's loads in flight
// while one is worked on. load(i, t) starts the loads of tile t into buffer i
// (tiles past the last too: they give zeros), step(i, t) works on it. No branch
// leaves the loop between steps: that would cost copies of the accumulators.
// Ends with no load in flight. (A third buffer changed nothing: 12 packed
// documents' gradient, 1 sequence of 512 a head.)
template <class Load, class Step>
__device__ __forceinline__ void run_tiles(int n, const Load &load, const Step &step) {
  const std::integral_constant<int, 0> b0;
  const std::integral_constant<int, 1> b1;
  if (n <= 0) return;
  load(b0, 0);
  int t = 0;
  for (; t + 1 < n; t += 2) {
    wait_loads();
    block_sync();
    load(b1, t + 1);
    step(b0, t);
    wait_loads();
    block_sync();
    load(b0, t + 2);
    step(b1, t + 1);
  }
  wait_loads();
  if (t < n) {
    block_sync();
    step(b0, t);
  }
}

// --------------------------------------------------------------------------
// Packed sequences
// --------------------------------------------------------------------------

// Sequence b's first row and its count of rows, clamped to [0, n].
struct Span {
  int first, count;
};
__device__ __forceinline__ Span span_of(const int32_t *cu, int b, int n) {
  const int s = clamp_to(cu[b], 0, n);
  const int e = clamp_to(cu[b + 1], s, n);
  return {s, e - s};
}

// Inclusive sum over the wave, in data-parallel-primitive moves: by shifts inside
// rows of 16 lanes, then the last lane of a row to the next, and of 32 to the others.
__device__ __forceinline__ int wave_sums(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

// The largest over the wave, uniform: the same moves.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  const auto moved = [&](auto how, auto rows) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(how)::value,
                                                 decltype(rows)::value, 0xf, false);
  };
  using std::integral_constant;
  const integral_constant<int, 0xf> all;
  x = max(x, moved(integral_constant<int, 0x111>(), all));
  x = max(x, moved(integral_constant<int, 0x112>(), all));
  x = max(x, moved(integral_constant<int, 0x114>(), all));
  x = max(x, moved(integral_constant<int, 0x118>(), all));
  x = max(x, moved(integral_constant<int, 0x142>(), integral_constant<int, 0xa>()));
  x = max(x, moved(integral_constant<int, 0x143>(), integral_constant<int, 0xc>()));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, OPA_WAVE - 1);
}

// Tile `tile` of the tiles of `rows` rows that the sequences of `cu` have: which
// of the sequence's tiles it is, the sequence's spans in both offset arrays, and
// which sequence; false past the last. By whole waves; the result is uniform. Each lane loads a
// sequence's four offsets at once: what follows waits for one load.
__device__ __forceinline__ int tiles_of(int count, int rows) { return (count + rows - 1) / rows; }
struct RowsLog2 {
  int n;  // 2^n rows
};
__device__ __forceinline__ int tiles_of(int count, RowsLog2 rows) {
  return (count + (1 << rows.n) - 1) >> rows.n;
}
template <class R>
__device__ __forceinline__ bool find_tile(const int32_t *cu, int n, const int32_t *other,
                                          int n_other, int n_seqs, R rows, int tile, Span &mine,
                                          Span &its, int &part, int *seq = nullptr) {
  const int lane = lane_id();
  for (int base = 0; base < n_seqs; base += OPA_WAVE) {
    const int b = base + lane < n_seqs ? base + lane : n_seqs - 1;
    const Span x = span_of(cu, b, n), y = span_of(other, b, n_other);
    const int tiles = base + lane < n_seqs ? tiles_of(x.count, rows) : 0;
    const int inc = wave_sums(tiles);
    const uint64_t m = __ballot(inc > tile);
    if (m) {
      const int w = __ffsll((unsigned long long)m) - 1;
      const auto from = [&](int v) { return __builtin_amdgcn_readlane(v, w); };
      mine = {from(x.first), from(x.count)};
      its = {from(y.first), from(y.count)};
      part = tile - from(inc - tiles);
      if (seq) *seq = base + w;
      return true;
    }
    tile -= __builtin_amdgcn_readlane(inc, OPA_WAVE - 1);
  }
  return false;
}

// Through a window with sinks a block of queries counts its keys without those that
// lie between the first `front` (the sinks, and up to a multiple of 8) and its first
// query's window: key j is place j, or past the front place j - window_skip. place: how
// many keys stand before its first query's.
__device__ __forceinline__ int window_front(int sinks) { return (sinks + 7) & ~7; }
__device__ __forceinline__ int window_skip(int place, int window, int front) {
  const int first = place + 1 - window;
  return first > front ? first - front : 0;
}
// tile_load of the places from k0 on; `left` places exist from there. A load's rows are
// 8 or fewer, all of the front or none.
template <int DP, int ROWS, int NW>
__device__ __forceinline__ void window_tile_load(uint16_t *tile, const uint16_t *src, int64_t ts,
                                                 int k0, int left, int front, int skip,
                                                 int head_dim, int wave) {
  if (skip == 0 || k0 >= front) {
    tile_load<DP, ROWS, NW>(tile, src + (int64_t)(k0 + skip) * ts, ts, left, head_dim, wave);
    return;
  }
  constexpr int C = DP / 8, N = ROWS * C / (NW * OPA_WAVE), R = OPA_WAVE / C;
  static_assert(R <= 8 && 8 % R == 0, "a load's rows");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int first = (i * NW + wave) * OPA_WAVE, row0 = first / C;
    const int rows = clamp_to(left - row0, 0, R);
    const int key = k0 + row0 < front ? k0 + row0 : k0 + row0 + skip;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(uniform(src + (int64_t)key * ts)), (short)0,
        uniform((int)(rows * ts * 2)), 0x00027000);
    const int row = lane_id() / C, chunk = (lane_id() % C) ^ swz<DP>(row0 + row);
    const uint32_t off = chunk * 8 < head_dim ? (uint32_t)(row * (int)ts * 2 + chunk * 16)
                                              : 0xfffffff0u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void *)(tile + first * 8), 16, (int)off, 0, 0,
        0);
  }
}

// Where a query of the wave does not see all of 32 keys that begin at place c0, hide(e)
// for each of this lane's elements e that it does not see: it sees those of the window
// that ends before place `seen`, and the sinks before that. All queries see the places
// below `whole`, and those from `latest` on.
template <class Hide>
__device__ __forceinline__ void hide_keys(int c0, int whole, int seen, int latest, int window,
                                          int sinks, const Hide &hide) {
  if (c0 + 32 <= whole && (c0 >= latest || c0 + 32 <= sinks)) return;
  // how far the lane's first element is past the window's begin: one comparison of
  // numbers without a sign for both ends
  const int past = c0 + ((lane_id() >> 5) << 2) - seen + window;
  const int kept = c0 < sinks ? (sinks < seen ? sinks : seen) - seen + window : INT_MIN;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int at = past + 8 * (e >> 2) + (e & 3);
    if ((uint32_t)at >= (uint32_t)window && at >= kept) hide(e);
  }
}

// Errors found in the data, into the record's flags, status and bad_records.
__device__ inline void report(opattr_diag *diag, uint32_t flag, int bad) {
  if (!diag || bad <= 0) return;
  atomicOr(&diag->flags, flag);
  if (flag & OPATTR_F_DATA) {
    atomicAdd((unsigned long long *)&diag->bad_records, (unsigned long long)bad);
    atomicExch(&diag->status, OPATTR_ERR_DATA);
  } else {
    const int32_t was = diag->status;
    if (was != OPATTR_ERR_DATA && was != OPATTR_ERR_ORDER)
      atomicCAS(&diag->status, was, OPATTR_ERR_LIMIT);
  }
}

// Offsets outside [0, n] or decreasing, by one block of `threads`. (Asking the launch for
// them makes a kernel's arguments 256 bytes longer: 0.2 us of a launch of 6.4.)
__device__ inline void check_spans(const int32_t *cu, int n_seqs, int n, opattr_diag *diag,
                                   int threads) {
  if (!diag) return;
  int bad = 0;
  for (int b = threadIdx.x; b < n_seqs; b += threads)
    bad += cu[b] < 0 || cu[b + 1] > n || cu[b + 1] < cu[b];
  if (bad) report(diag, OPATTR_F_DATA, bad);
}

}  // namespace opa
