// What the kernels of attention over the cache in 8 bits share: codes as operands, the softmax level's constants, a sequence's counts.
#pragma once

#include "block.h"

namespace innerq {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// log2 of the weight that the largest score has when it raises the level, and of the largest weight before the level is raised (fp16 ends at 2^15.999).
constexpr float kTop = 10.0f, kRaise = 15.9f;
constexpr float kFar = 0x1p19f;                          // levels beyond: neighbours in fp32 are 2^-4 apart and more
constexpr float kFarShare = 0x1p-16f;                    // of its own size, by which a level is raised the sooner

// By which power of two a tensor's codes are multiplied.  E4M3: its bits in fp32; integers: see int_codes.
template <bool E4M3>
__device__ __forceinline__ constexpr uint32_t codes_times(int x) { return E4M3 ? (uint32_t)(x + 127) << 23 : int_codes(x); }
// Eight codes as fp16, times that: exact down to multiples of 2^-24 (integers to 2^-24, E4M3, whose codes reach 2^-9, to 2^-15), rounded to them below.
template <bool E4M3>
__device__ __forceinline__ half8_t expand(uint32_t a, uint32_t b, uint32_t by) {
  half2_t h[4];
  if constexpr (E4M3) {
    const float f = __uint_as_float(by);
    h[0] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, f, false));
    h[1] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, f, true));
    h[2] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, f, false));
    h[3] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, f, true));
  } else {
    const half2_t both = __builtin_bit_cast(half2_t, by), f = {both.x, both.x}, bias = {both.y, both.y};
    const uint32_t top = int_codes_top(by);
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    h[0] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(top, a, 0x04010400u)), f, bias);
    h[1] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(top, a, 0x04030402u)), f, bias);
    h[2] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(top, b, 0x04010400u)), f, bias);
    h[3] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(top, b, 0x04030402u)), f, bias);
  }
  return half8_t{h[0].x, h[0].y, h[1].x, h[1].y, h[2].x, h[2].y, h[3].x, h[3].y};
}

struct BlockSeq { int n, t, packed; };
__device__ __forceinline__ BlockSeq block_seq(const BlockAttnArgs& a, int b) {
  const int cap = (int)a.s.capacity;
  BlockSeq s = {a.s.n_tokens, a.s.t_new, 0};
  if (a.s.n_dev) {
    s.n = a.s.n_dev[b];
    s.n = s.n < 0 ? 0 : s.n > cap ? cap : s.n;
    if (a.s.t_dev) s.t = a.s.t_dev[b];
    s.t = s.t < 0 ? 0 : s.t > a.s.t_new ? a.s.t_new : s.t;
  }
  s.packed = (int)block_packed(s.n, a.s.block);
  return s;
}

__device__ __forceinline__ float lane_of(float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); }
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x, i); }
// The magnitude that raises a level: beyond kFar the sooner, so that a weight stays in fp16 whatever the rounding of the sum.
__device__ __forceinline__ float threshold(float m) { return __builtin_fmaf(-kFarShare, __builtin_fabsf(m), m) + kRaise; }

// Scales.  That of a block of keys is a factor of its scores.  That of a block of values is a summand of the exponent, so that a weight carries it:
//   w = 2^(s + log2 S - level),  O = sum w code,  l = sum w / S  (of the same rounded weights).
// A token whose S is far below that of a stronger one would meet fp16's smallest step, 2^-24, the sooner, though it counts in full in l.  So the scale of a block
// is taken as S = 2^k S_v, from half of the largest one so far up to all of it, with codes times 2^-k; and that of new and open rows, which is 1, as a power of
// two not below half of the largest, with values divided by it.  Weights are then off by 2^-25 at a level of 2^10 below the largest one, and by one
// factor of two for the scales: 2^-34 of the largest.  (Scales as they are down to 1/16 of the largest, and 1 for new rows: 2^-30, and 2^-25.)
// Of the codes' products fp16 holds multiples of 2^-24, so that every S is taken 2^-kLift times and codes 2^kLift times as large: what is rounded is off by 2^-25
// at 2^-5 of the largest scale and less, 2^-36 of the largest value; and new rows are divided by more than 1 only beside values above 2^12.
constexpr int kLift = 5;                                 // (1152 2^5, which integers have taken away, is an fp16 number)
struct Scales { float by, add, inv; uint32_t values; };  // factor of the scores, log2 S, 1 / S, by what codes of values are multiplied

constexpr float kScoreScale = 0.08838834764831845f * 1.4426950408889634f;        // log2(e) / sqrt(d)

// Where 64 tiles of a sequence's kv head lie, and their scales: a tile a lane.
template <bool E4M3>
struct BlockUnits {
  long long at = 0;
  float by = 0.f, add = 0.f, inv = 0.f, largest = 0.f;
  uint32_t values = 0u;
  int base = -1;
  // Tile u (not below an earlier one) is among them from now on; tiles end before u1.
  __device__ __forceinline__ void look(const BlockStore& s, int b, int h, int u, int u1, int lane) {
    if (base >= 0 && u < base + 64) return;              // (uniform)
    base = u;
    at = block_tile(s, b, h, u + lane < u1 ? u + lane : u1 - 1);
    const long long sc = block_scale(s, at);
    by = s.k.scales[sc] * kScoreScale;
    const float vs = s.v.scales[sc];
    float most = vs;
#pragma unroll
    for (int i = 32; i > 0; i /= 2) most = fmaxf(most, __shfl_xor(most, i));
    largest = fmaxf(largest, most);
    const int e = largest > 0.f ? __builtin_amdgcn_frexp_expf(largest) : 1 + kLift, k = vs > 0.f ? e - __builtin_amdgcn_frexp_expf(vs) : 0;
    const float size = __builtin_amdgcn_ldexpf(vs > 0.f ? vs : 0.5f, (vs > 0.f ? k : e) - kLift);      // (no values but zeros: any)
    values = codes_times<E4M3>(kLift - k);
    add = __builtin_amdgcn_logf(size);
    inv = 1.0f / size;
  }
  __device__ __forceinline__ long long tile(int u) const {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(at >> 32), u - base) << 32) |
                       (unsigned)__builtin_amdgcn_readlane((int)at, u - base));
  }
  __device__ __forceinline__ Scales scales(int u) const {
    return {lane_of(by, u - base), lane_of(add, u - base), lane_of(inv, u - base), lane_of(values, u - base)};
  }
};

// log2 of the divisor of fp16 rows behind blocks whose largest scale is `largest` (0: none).  The level and the sum of a row are brought to its unit before such rows
// and back behind them, so that the rows' weights are what they would be with S = 1.
__device__ __forceinline__ int plain_shift(float largest) {
  const int e = __builtin_amdgcn_readfirstlane(largest > 0.f ? __builtin_amdgcn_frexp_expf(largest) : 0) - 1 - kLift;
  return e < 0 ? 0 : e;
}
constexpr Scales kPlainScales = {kScoreScale, 0.f, 1.f, 0u};
__device__ __forceinline__ uint32_t times(uint32_t pair, uint32_t by) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pair) * __builtin_bit_cast(half2_t, by));
}

// What a work-group does.
struct BlockWork { int b, h, row_block, split, n_splits; long long slot; };

// The same counts for all, or the same work-groups whatever the counts: sequence-heads that can be shared out evenly stay on one XCD (its L2 then brings
// every tile from memory once), those of a sequence, which are as long, on different ones; the last rows, which have the most keys, go first.
__device__ __forceinline__ BlockWork uniform_work(const BlockAttnArgs& a) {
  const unsigned heads = (unsigned)(a.s.batch * a.s.n_kv_heads), n = (unsigned)a.n_splits;
  const bool pinned = heads % 8u == 0u && a.row_blocks > 1;
  const unsigned at = pinned ? blockIdx.x / 8u : blockIdx.x, mine = pinned ? heads / 8u : heads;
  const unsigned rank = at / (mine * n), rest = at % (mine * n), bh = pinned ? rest / n * 8u + blockIdx.x % 8u : rest / n;
  BlockWork w;
  w.b = (int)(bh / (unsigned)a.s.n_kv_heads);
  w.h = (int)(bh % (unsigned)a.s.n_kv_heads);
  w.row_block = a.row_blocks - 1 - (int)rank;
  w.split = (int)(rest % n);
  w.n_splits = a.n_splits;
  w.slot = ((long long)bh * a.row_blocks + w.row_block) * a.n_splits + w.split;
  return w;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
  return x;
}
// A ragged batch: work-groups find their work from the counts of all sequences (four a lane; the arithmetic is the plan's), every wavefront
// the same: of the sequences with rows above `from` and up to `to`, those of work-group `group`.
template <int ROWS, int WAVES>
__device__ __forceinline__ bool find_work(const BlockAttnArgs& a, int from, int to, int group, BlockWork& w) {
  constexpr int N = kBlockListMost / 64;
  constexpr int ITEMS = block_list_items(BlockForm{ROWS, WAVES});
  const int lane = (int)threadIdx.x & 63;
  int units[N], tiles[N];                                // of the lane's sequences
  int most = 1;
  float work = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int b = N * lane + j;
    units[j] = tiles[j] = 0;
    if (b < a.s.batch) {
      const BlockSeq s = block_seq(a, b);
      const BlockShare share = block_share(s.n, s.t, a.k.p != nullptr, a.heads_per_kv, a.s.n_kv_heads, from, to, ROWS);
      units[j] = share.units;
      tiles[j] = share.tiles;
    }
    most = tiles[j] > most ? tiles[j] : most;
    work += (float)units[j] * (float)tiles[j];
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int x = __shfl_xor(most, i);
    most = x > most ? x : most;
    work += __shfl_xor(work, i);
  }
  most = __builtin_amdgcn_readfirstlane(most);
  int length = __builtin_amdgcn_readfirstlane(block_first_length(work, ITEMS));
  int mine, ranges;
  while (true) {
    mine = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) mine += units[j] * block_ranges(tiles[j], length);
    ranges = __builtin_amdgcn_readfirstlane(wave_sum(mine));
    if (block_length_fits(length, most, ranges, ITEMS)) break;
    length = __builtin_amdgcn_readfirstlane(block_next_length(length, ranges, ITEMS));
  }
  // this work-group's place in the line, and the sequence that it belongs to
  const bool by_head = block_by_head(a.s.n_kv_heads);
  const int place = block_turn(group, ranges, by_head), scale = by_head ? 8 : 1;
  if (place < 0) return false;                           // (uniform)
  if (by_head) mine /= 8;
  int before = mine;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int x = __shfl_up(before, i);
    if (lane >= i) before += x;
  }
  const unsigned long long reach = __builtin_amdgcn_ballot_w64(before > place);
  if (reach == 0) return false;                          // (uniform)
  const int owner = __builtin_ctzll(reach);
  int first = __builtin_amdgcn_readlane(before - mine, owner);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int u = __builtin_amdgcn_readlane(units[j], owner), splits = block_ranges(__builtin_amdgcn_readlane(tiles[j], owner), length), all = u * splits / scale;
    if (place >= first && place < first + all) {
      const int range = block_range(place - first, group, u, a.s.n_kv_heads, splits, by_head);
      const BlockPlace at = block_place(range, u, a.s.n_kv_heads, splits);
      w.b = N * owner + j;
      w.h = at.h;
      w.row_block = at.row_block;
      w.split = at.split;
      w.n_splits = splits;
      w.slot = first * scale + range;
      if (range == 0 && threadIdx.x == 0) {
        a.table[2 * w.b] = first * scale;
        a.table[2 * w.b + 1] = splits;
      }
      return true;
    }
    first += all;
  }
  return false;
}

}  // namespace innerq
