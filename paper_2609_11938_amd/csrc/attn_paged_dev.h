// Shares of the sequences' tokens, for the attention of one new token a sequence
// over a paged cache (16 bits and 8).
#pragma once
#include <limits.h>

#include "attn_dev.h"
#include "attn_impl.h"

namespace opa {

constexpr int kPagedWaves = 4;
constexpr int kTile = 32;        // tokens a wave takes at a time
constexpr int kMinShare = 256;   // tokens of the smallest share
// Blocks that the shares come to: few enough that a block's start is a small part of it,
// enough that the last ones leave no chiplet idle for long. Over 8 bits a share of as many
// tokens is done sooner: 96 sequences of up to 9001 tokens, 8 key heads of 128, 65 us in
// 2048 blocks, 68 us in 1024 and 67 us in 4096, whose join takes 7 us and not 5.
constexpr int kBlocks = 1024, kScaledBlocks = 2048;

// Tokens of sequence b, as many as its table can name; of these, as many as its
// query sees: the first and the last ones, through a window with sinks.
__device__ __forceinline__ int paged_tokens(const PagedArgs &a, int b) {
  return b < a.n_seqs ? clamp_to(a.lens[b], 0, a.slots) : 0;
}
__device__ __forceinline__ int paged_len(const PagedArgs &a, int b) {
  const int n = paged_tokens(a, b);
  return n < a.most ? n : a.most;
}

__device__ __forceinline__ int shares_of(int len, int c) { return len > c ? (len + c - 1) / c : 1; }

// Over the cache of 8 bits a query's tokens are counted through by runs of 16, which
// lie on one page each where pages have as many: the sinks' last and the window's first
// may hold tokens that are not seen. Token j is place j, or past the sinks' runs place
// j - skip; places [hide, shown) are not seen.
struct Seen {
  int front, skip, hide, shown;
};
__device__ __forceinline__ Seen seen_of(const ScaledArgs &a, int tokens) {
  Seen s{(a.sinks + 15) & ~15, 0, 0, 0};
  const int first = tokens - a.window;
  if (first <= a.sinks) return s;
  if (first > s.front) s.skip = (first & ~15) - s.front;
  s.hide = a.sinks;
  s.shown = first - s.skip;
  return s;
}
__device__ __forceinline__ int paged_len(const ScaledArgs &a, int b) {
  const int n = paged_tokens(a, b);
  return n - seen_of(a, n).skip;
}

// Sequences one to a lane; past 64, loops of as many.
struct Share {
  int size;   // tokens of every share but a sequence's last
  int seq, part, len;
  int first;  // the sequence's first share, as the shares are counted
};

__host__ __device__ constexpr int blocks_of(const PagedArgs &) { return kBlocks; }
__host__ __device__ constexpr int blocks_of(const ScaledArgs &) { return kScaledBlocks; }

// Tokens of a share, from every sequence's length: as many as make blocks_of shares
// of the work of all key heads. mine: this lane's sequence's length.
template <class Args>
__device__ __forceinline__ int share_size(const Args &a, int mine) {
  if (a.most <= kMinShare) return kMinShare;
  int64_t sum = mine;
  for (int b = OPA_WAVE + lane_id(); b < a.n_seqs; b += OPA_WAVE) sum += paged_len(a, b);
  if (__all(sum < 1 << 25)) {
    sum = __builtin_amdgcn_readlane(wave_sums((int)sum), OPA_WAVE - 1);
  } else {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
  }
  const int64_t each = (sum * a.n_kv + blocks_of(a) - 1) / blocks_of(a);
  const int64_t c = (each + kTile * kPagedWaves - 1) / (kTile * kPagedWaves) *
                    (kTile * kPagedWaves);
  return uniform((int)(c < kMinShare ? kMinShare : c < 1 << 30 ? c : 1 << 30));
}

// Share `item` of all the sequences' shares; false past the last. By whole waves.
template <class Args>
__device__ __forceinline__ bool find_share(const Args &a, int item, Share &s) {
  const int lane = lane_id();
  const int mine = paged_len(a, lane);
  s.size = share_size(a, mine);
  int done = 0;
  for (int base = 0; base < a.n_seqs; base += OPA_WAVE) {
    const int b = base + lane;
    const int len = base ? paged_len(a, b) : mine;
    const int n = b < a.n_seqs ? shares_of(len, s.size) : 0;
    const int inc = wave_sums(n);
    const uint64_t m = __ballot(done + inc > item);
    if (m) {
      const int w = __ffsll((unsigned long long)m) - 1;
      s.seq = base + w;
      s.first = done + __builtin_amdgcn_readlane(inc - n, w);
      s.part = item - s.first;
      s.len = __builtin_amdgcn_readlane(len, w);
      return true;
    }
    done += __builtin_amdgcn_readlane(inc, OPA_WAVE - 1);
  }
  return false;
}

// What the join wants to know of a sequence: its first share, and how many.
__device__ __forceinline__ void note_shares(const PagedArgs &a, const Share &s) {
  if (a.shares && s.part == 0 && threadIdx.x == 0)
    *reinterpret_cast<int2 *>(a.shares + 2 * s.seq) = int2{s.first, shares_of(s.len, s.size)};
}

// Shares at most: sum of ceil(len / c) with c >= kMinShare and c >= sum / (blocks
// / n_kv).
inline int64_t most_items(int n_seqs, int n_kv, int most, int blocks) {
  const int64_t a = (int64_t)blocks / n_kv + 1 + n_seqs;
  const int64_t b = (int64_t)n_seqs * (most > kMinShare ? (most + kMinShare - 1) / kMinShare : 1);
  return a < b ? a : b;
}

}  // namespace opa
