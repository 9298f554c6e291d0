// Writing the cache in 8 bits with block scales, and reading it back.
//
// Both are copies that change width: a value is read once and written once (2 + 1 bytes), and what bounds them is memory; for a single token it is
// the launch.  Writing 4 x 8 heads x 32k tokens, 806 MB: 143 us, 5.6 TB/s (a copy of as many bytes 163); reading them back 146, and 119 where the codes stay
// in the last-level cache; ragged prompts of 16 x 8 heads, 46 MB, 17; a token of 32 x 8 heads 7.5, the newest 257 tokens of 8 x 8 heads 5.2.
//
// A wavefront takes a block of one head by itself (32 x 128 values: 64 a lane, in registers), so the largest magnitude
// is a reduction over its lanes and no barrier stands in the way.  Keys: a lane has sixteen channels of a token, sixteen bytes of the
// store.  Values: a lane has two channels of eight tokens, the sixteen bytes that a lane of the attention kernel takes as one operand of
// either channel, so the transposition is made of whole registers.
#include "block.h"

namespace innerq {
namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = kHeadDim;

// Stores past the caches: what is written is not read again here, and lines that wait in the L2 for the rest of a line cost more than they bring
// (us, with and without: reading 4 x 8 heads x 32k tokens 119, 154; writing them 141, 151).
template <typename T>
__device__ __forceinline__ void store_past(T* p, T x) { __builtin_nontemporal_store(x, p); }

// What a sequence has and takes (ragged: from device memory).
struct Take { int n, t; };
__device__ __forceinline__ Take take_of(const BlockStore& s, int b) {
  Take x = {s.n_tokens, s.t_new};
  if (!s.n_dev) return x;
  const int cap = (int)s.capacity;
  x.n = s.n_dev[b];
  if (s.t_dev) x.t = s.t_dev[b];
  x.t = x.t < 0 ? 0 : x.t > s.t_new ? s.t_new : x.t;
  if (x.n < 0 || x.n > cap) return {0, 0};               // (a count that is none: nothing is written)
  x.t = x.t > cap - x.n ? cap - x.n : x.t;
  return x;
}

__device__ __forceinline__ uint32_t wave_most(uint32_t x) {
#pragma unroll
  for (int i = 32; i > 0; i /= 2) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, i);
    x = x > y ? x : y;
  }
  return x;
}
// Larger magnitude of fp16 pairs, as integers (which order as the magnitudes do).
__device__ __forceinline__ uint32_t most_of(uint32_t a, uint32_t b) {
  typedef unsigned short us2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b & 0x7fff7fffu)));
}

// The quotient rounded as a division rounds it, for every fp16 x and every scale of a block that can hold it: the product with the rounded reciprocal
// is off by a step or two, its exact remainder puts that right (all 5e8 pairs of either type: a test walks them).  Three instructions
// instead of ten, of which a block has 64 a lane.
struct Divisor { float scale, reciprocal; };
__device__ __forceinline__ float quotient(float x, const Divisor& d) {
  const float q = x * d.reciprocal;
  return __builtin_fmaf(-__builtin_fmaf(q, d.scale, -x), d.reciprocal, q);      // (with these signs zeros keep theirs)
}
// Two pairs of values as four codes.
template <bool E4M3>
__device__ __forceinline__ uint32_t encode(uint32_t x, uint32_t y, const Divisor& d) {
  const half2_t a = __builtin_bit_cast(half2_t, x), b = __builtin_bit_cast(half2_t, y);
  const float q[4] = {quotient((float)a.x, d), quotient((float)a.y, d), quotient((float)b.x, d), quotient((float)b.y, d)};
  if constexpr (E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
  } else {
    // (rounded to an integer in the low bits of 1.5 x 2^23 + q: half to even, as every fp32 sum)
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(q[i] + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
  }
}

// A block of 32 SUB tokens from token g0 on (g0 a multiple of the block): token i comes from the open rows if it is cached, else from the
// new rows.
template <bool E4M3, int SUB>
__device__ __forceinline__ void pack_block(const BlockStore& s, const BlockTensor& x, const RowView& fresh, bool keys, int b, int h, int n, int g0, int lane) {
  const __half* open = x.open + ((long long)b * s.n_kv_heads + h) * (32 * SUB) * D;
  const __half* rows = fresh.p + b * fresh.batch + h * fresh.head;
  auto row = [&](int i) { return g0 + i < n ? open + i * D : rows + (g0 + i - n) * fresh.token; };
  const long long tile = block_tile(s, b, h, g0 / kBlockTile);
  uint32_t w[SUB][32];
  uint32_t most = 0u;
  if (keys) {
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half* src = row(32 * u + 8 * i + (lane >> 3)) + 16 * (lane & 7);
        const u32x4 p = *reinterpret_cast<const u32x4*>(src), q = *reinterpret_cast<const u32x4*>(src + 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[u][8 * i + e] = p[e];
          w[u][8 * i + 4 + e] = q[e];
        }
      }
  } else {
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int i = 0; i < 32; ++i) w[u][i] = *reinterpret_cast<const uint32_t*>(row(32 * u + i) + 2 * lane);
  }
#pragma unroll
  for (int u = 0; u < SUB; ++u)
#pragma unroll
    for (int i = 0; i < 32; ++i) most = most_of(most, w[u][i]);
  const uint32_t top = wave_most((most & 0xffffu) > (most >> 16) ? most & 0xffffu : most >> 16);
  const float largest = (float)__builtin_bit_cast(_Float16, (unsigned short)top);
  const float scale = largest / (E4M3 ? 448.f : 127.f);
  const Divisor by = {scale, scale == 0.f ? 0.f : 1.0f / scale};      // (a block of zeros: zeros)
  if (lane == 0) x.scales[block_scale(s, tile)] = scale;
#pragma unroll
  for (int u = 0; u < SUB; ++u) {
    uint8_t* dst = x.codes + (tile + u) * kBlockTileBytes;
    if (keys) {
      // lane's token 8 i + lane / 8 is 16 a + c, its channels are 32 g + 16 h
      const int part = lane & 7;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t* p = w[u] + 8 * i;
        const u32x4 o = {encode<E4M3>(p[0], p[1], by), encode<E4M3>(p[2], p[3], by), encode<E4M3>(p[4], p[5], by), encode<E4M3>(p[6], p[7], by)};
        const int token = 8 * i + (lane >> 3);
        store_past(reinterpret_cast<u32x4*>(dst + (token >> 4) * 2048 + (part & 1) * 1024 + (part >> 1) * 256 + (token & 15) * 16), o);
      }
    } else {
      // lane's channels 2 lane, 2 lane + 1 are 32 q + 2 c + m
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t* p = w[u] + 16 * i + 4 * g;
          const uint32_t lo[2] = {__builtin_amdgcn_perm(p[1], p[0], 0x05040100u), __builtin_amdgcn_perm(p[3], p[2], 0x05040100u)};
          const uint32_t hi[2] = {__builtin_amdgcn_perm(p[1], p[0], 0x07060302u), __builtin_amdgcn_perm(p[3], p[2], 0x07060302u)};
          o[i] = encode<E4M3>(lo[0], lo[1], by);
          o[2 + i] = encode<E4M3>(hi[0], hi[1], by);
        }
        store_past(reinterpret_cast<u32x4*>(dst + (lane >> 4) * 1024 + g * 256 + (lane & 15) * 16), o);
      }
    }
  }
}

// New tokens from `stays` on wait in the open rows.
__device__ __forceinline__ void keep_open(const BlockStore& s, const BlockTensor& x, const RowView& fresh, int b, int h, int n, int end, int stays, int lane) {
  __half* open = x.open + ((long long)b * s.n_kv_heads + h) * s.block * D;
  const __half* rows = fresh.p + b * fresh.batch + h * fresh.head;
  for (int token = (stays > n ? stays : n) + (lane >> 4); token < end; token += 4)
    *reinterpret_cast<u32x4*>(open + (token & (s.block - 1)) * D + 8 * (lane & 15)) =
        *reinterpret_cast<const u32x4*>(rows + (token - n) * fresh.token + 8 * (lane & 15));
}

// Unit j of a head: block j of those that the call reaches; the first one's wavefront, which reads the open rows, is also the one that writes them.
template <bool E4M3>
__device__ __forceinline__ void append_unit(const BlockAppendArgs& a, bool keys, int b, int h, int j, const Take& t, int lane) {
  const BlockStore& s = a.s;
  const BlockTensor& x = keys ? s.k : s.v;
  const RowView& fresh = keys ? a.k : a.v;
  const int mask = s.block - 1, end = t.n + t.t, stays = end & ~mask, g0 = (t.n & ~mask) + j * s.block;
  if (t.t == 0) return;
  if (g0 < stays) {
    if (s.block == 32) pack_block<E4M3, 1>(s, x, fresh, keys, b, h, t.n, g0, lane);
    else pack_block<E4M3, 2>(s, x, fresh, keys, b, h, t.n, g0, lane);
  }
  asm volatile("" ::: "memory");                         // (what was read of the open rows is read)
  if (j == 0) keep_open(s, x, fresh, b, h, t.n, end, stays, lane);
}

// A wavefront a unit; heads of one token next to each other, as a projection leaves them.
template <bool E4M3>
__global__ void __launch_bounds__(256) block_append_kernel(BlockAppendArgs a, unsigned units) {
  const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (unit >= units) return;
  const unsigned H = (unsigned)a.s.n_kv_heads, rest = unit / H;
  const int h = (int)(unit - rest * H), lane = (int)threadIdx.x & 63;
  const bool keys = (rest & 1) == 0;
  const int b = (int)((rest >> 1) / (unsigned)a.units), j = (int)(rest >> 1) - b * a.units;
  append_unit<E4M3>(a, keys, b, h, j, take_of(a.s, b), lane);
}

// Few rows of a ragged batch: a work-group a sequence, which then advances its count.  (Without the second launch a step takes 3.2 us in place of 4.2, but its 16
// wavefronts pack the 2 H tensors' heads in turns.  In one launch and in two, us, a step that packs nothing, one that does, and 32 rows: 1 sequence of 8 heads 3.2
// and 4.2, 6.2 and 5.9, 6.7 and 6.5; 1 of 16 3.6 and 4.2, 10.1 and 6.1, 10.9 and 6.9; 1 of 32 4.8 and 4.2, 19 and 6.1, 20 and 6.6; 64 of 32 the last two
// 20.6 and 10.5, 22 and 11; 256 of 8 3.9 and 4.7, 8.2 and 10.6, 13.0 and 13.3.  Every 32nd step packs; so in one where there is one turn, and of few rows also in two.)
template <bool E4M3>
__global__ void __launch_bounds__(1024) block_append_step_kernel(BlockAppendArgs a, int* counts) {
  const int b = (int)blockIdx.x, lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Take t = take_of(a.s, b);
  __syncthreads();                                       // (everybody has read the count)
  if (threadIdx.x == 0 && t.t > 0) counts[b] = t.n + t.t;
  for (int unit = wave; unit < a.units * 2 * a.s.n_kv_heads; unit += 16) {
    const int h = unit % a.s.n_kv_heads, rest = unit / a.s.n_kv_heads;
    append_unit<E4M3>(a, (rest & 1) == 0, b, h, rest >> 1, t, lane);
  }
}

__global__ void __launch_bounds__(256) block_counts_kernel(BlockStore s, int* counts) {
  const int b = (int)(blockIdx.x * 256 + threadIdx.x);
  if (b >= s.batch) return;
  const Take t = take_of(s, b);
  if (t.t > 0) counts[b] = t.n + t.t;
}

// ---- reading back

// Four codes times the scale, rounded to fp32 and then to fp16.
template <bool E4M3>
__device__ __forceinline__ void decode(uint32_t w, float scale, uint32_t (&out)[2]) {
  float x[4];
  if constexpr (E4M3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
  half2_t r[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y = x[i] * scale;
    asm("" : "+v"(y));                                   // (two roundings: merged with the conversion it would be one)
    r[i / 2][i % 2] = (_Float16)y;
  }
  out[0] = __builtin_bit_cast(uint32_t, r[0]);
  out[1] = __builtin_bit_cast(uint32_t, r[1]);
}

// A wavefront takes the tokens of one 32-token tile of a head that are asked for.
template <bool E4M3>
__global__ void __launch_bounds__(256) block_read_kernel(BlockReadArgs a, unsigned tiles, unsigned units) {
  const unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (unit >= units) return;
  const BlockStore& s = a.s;
  const unsigned H = (unsigned)s.n_kv_heads, rest = unit / H;
  const int h = (int)(unit - rest * H), lane = (int)threadIdx.x & 63;
  const bool keys = (rest & 1) == 0;
  const int b = (int)((rest >> 1) / tiles), j = (int)((rest >> 1) - b * tiles);
  __half* out = keys ? a.k : a.v;
  if (!out) return;
  int n = s.n_tokens;
  long long first = a.first;
  if (s.n_dev) {
    n = s.n_dev[b];
    n = n < 0 ? 0 : n > (int)s.capacity ? (int)s.capacity : n;
    if (a.first_dev) first = a.first_dev[b];
  }
  // tokens of the tile that are asked for and there
  const long long from = first < 0 ? 0 : first, to = first + s.t_new < n ? first + s.t_new : n;
  const long long tile0 = from / kBlockTile + j, t0 = tile0 * kBlockTile;
  if (t0 >= to) return;
  const int lo = (int)(from > t0 ? from - t0 : 0), hi = (int)(to - t0 < kBlockTile ? to - t0 : kBlockTile);
  const long long pitch = keys ? a.k_token : a.v_token;
  out += b * (keys ? a.k_batch : a.v_batch) + h * (keys ? a.k_head : a.v_head) + (t0 - first) * pitch;     // (of the tile's token 0)
  const BlockTensor& x = keys ? s.k : s.v;
  const int packed = n & ~(s.block - 1);
  if (t0 >= packed) {
    const __half* open = x.open + ((long long)b * H + h) * s.block * D + (t0 & (s.block - 1)) * D;
    for (int i = lo + (lane >> 4); i < hi; i += 4)
      *reinterpret_cast<u32x4*>(out + i * pitch + 8 * (lane & 15)) = *reinterpret_cast<const u32x4*>(open + i * D + 8 * (lane & 15));
    return;
  }
  const long long tile = block_tile(s, b, h, (int)tile0);
  const uint8_t* src = x.codes + tile * kBlockTileBytes;
  const float scale = x.scales[block_scale(s, tile)];
  if (keys) {
    // (eight channels a lane: a wavefront writes four whole rows at once)
    const int part = lane & 15, at = (part >> 1 & 1) * 1024 + (part >> 2) * 256 + (part & 1) * 8;
    u32x2 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int token = 4 * i + (lane >> 4);
      w[i] = *reinterpret_cast<const u32x2*>(src + (token >> 4) * 2048 + (token & 15) * 16 + at);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int token = 4 * i + (lane >> 4);
      uint32_t o[4];
      decode<E4M3>(w[i].x, scale, *reinterpret_cast<uint32_t(*)[2]>(o));
      decode<E4M3>(w[i].y, scale, *reinterpret_cast<uint32_t(*)[2]>(o + 2));
      if (token >= lo && token < hi) store_past(reinterpret_cast<u32x4*>(out + token * pitch + 8 * part), u32x4{o[0], o[1], o[2], o[3]});
    }
  } else {
    u32x4 w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) w[g] = *reinterpret_cast<const u32x4*>(src + (lane >> 4) * 1024 + g * 256 + (lane & 15) * 16);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t even[2], odd[2];
        decode<E4M3>(w[g][i], scale, even);
        decode<E4M3>(w[g][2 + i], scale, odd);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int token = 16 * i + 4 * g + e;
          const uint32_t pair = __builtin_amdgcn_perm(odd[e / 2], even[e / 2], e & 1 ? 0x07060302u : 0x05040100u);
          if (token >= lo && token < hi) store_past(reinterpret_cast<uint32_t*>(out + token * pitch + 2 * lane), pair);
        }
      }
  }
}

}  // namespace

// (up to a block of rows complete one block at most: a unit a head and tensor)
static bool append_in_one(const BlockStore& s) {
  return s.t_new <= s.block && (2 * s.n_kv_heads <= 16 || (2 * s.n_kv_heads <= 32 && 8 * s.t_new <= s.block));
}
hipError_t launch_block_append(const BlockAppendArgs& a, int* counts, bool e4m3, hipStream_t stream) {
  if (counts && append_in_one(a.s)) {
    if (e4m3) block_append_step_kernel<true><<<a.s.batch, 1024, 0, stream>>>(a, counts);
    else block_append_step_kernel<false><<<a.s.batch, 1024, 0, stream>>>(a, counts);
    return hipGetLastError();
  }
  const long long units = (long long)a.s.batch * a.s.n_kv_heads * 2 * a.units, groups = ceil_div(units, 4);
  if (units >= (1LL << 31)) return hipErrorInvalidValue;       // (4 KB of the store each: more than the card has)
  if (e4m3) block_append_kernel<true><<<(unsigned)groups, 256, 0, stream>>>(a, (unsigned)units);
  else block_append_kernel<false><<<(unsigned)groups, 256, 0, stream>>>(a, (unsigned)units);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && counts) {
    block_counts_kernel<<<(unsigned)ceil_div(a.s.batch, 256), 256, 0, stream>>>(a.s, counts);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_block_read(const BlockReadArgs& a, bool e4m3, hipStream_t stream) {
  // (a range that begins inside a tile reaches into one more)
  const int tiles = (int)((a.s.n_dev ? kBlockTile - 1 : a.first % kBlockTile) + a.s.t_new - 1) / kBlockTile + 1;
  const long long units = (long long)a.s.batch * a.s.n_kv_heads * 2 * tiles, groups = ceil_div(units, 4);
  if (units >= (1LL << 31)) return hipErrorInvalidValue;       // (8 KB of rows each: more than the card has)
  if (e4m3) block_read_kernel<true><<<(unsigned)groups, 256, 0, stream>>>(a, (unsigned)tiles, (unsigned)units);
  else block_read_kernel<false><<<(unsigned)groups, 256, 0, stream>>>(a, (unsigned)tiles, (unsigned)units);
  return hipGetLastError();
}

}  // namespace innerq
