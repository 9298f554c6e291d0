// Attention over the cache in 8 bits with block scales, up to 64 rows of a kv head: what a work-group does (attention_block.hip says how).
#pragma once

#include "block.h"
#include "block_math.h"

namespace innerq {
namespace block_few {

constexpr int D = kHeadDim;

__device__ __forceinline__ float row_most(float x) {     // over the four lanes of a query row
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Four channels of the output.
__device__ __forceinline__ void store_four(const BlockAttnArgs& a, long long at, float w, float x, float y, float z) {
  if (a.out_is_fp32) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = float4{w, x, y, z};
  } else {
    const half2_t lo = {(_Float16)w, (_Float16)x}, hi = {(_Float16)y, (_Float16)z};
    *reinterpret_cast<u32x2*>(static_cast<_Float16*>(a.out) + at) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

// A wavefront's 16 NR query rows (lane: row lane % 16 of each sixteen; channels 32 (lane / 16) + 8 s + ..): operands, outputs (two
// accumulators of 4: channels 32 q + 8 (lane / 16) + 2 i + m at o[2 q + m][i]), level, the lane's part of the sum.
template <int NR>
struct Rows {
  half8_t q[NR][4];
  float4_t o[NR][8];
  float m[NR], l[NR];
};

template <int NR>
constexpr int kPieces = NR == 4 ? 1 : 2;                 // fp16 pieces of a weight

__device__ __forceinline__ float largest_of(const float4_t (&s)[2]) {
  return fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
}
// Weights of the scores of a tile (level and sum move on).  s[r][a][i]: token 16 a + 4 (lane / 16) + i.
template <int NR>
__device__ __forceinline__ void weights(Rows<NR>& r, float4_t (&s)[NR][2], const Scales& u, half8_t (&p)[NR][kPieces<NR>]) {
  bool raise = false;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][a][i] = __builtin_fmaf(s[n][a][i], u.by, u.add);
        asm("" : "+v"(s[n][a][i]));                      // (rounded before the level is taken from it: far levels need that)
      }
    raise |= largest_of(s[n]) > threshold(r.m[n]);
  }
  if (__builtin_amdgcn_ballot_w64(raise)) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float top = row_most(largest_of(s[n]));
      const bool up = top > threshold(r.m[n]);
      const float level = up ? fmaxf(r.m[n], __builtin_fabsf(top) > kFar ? top : top - kTop) : r.m[n];
      const float f = up ? __builtin_amdgcn_exp2f(r.m[n] - level) : 1.f;         // (0 from the empty state)
      r.l[n] *= f;
#pragma unroll
      for (int x = 0; x < 8; ++x) r.o[n][x] *= f;
      r.m[n] = level;
    }
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const float level = r.m[n] == -INFINITY ? 0.f : r.m[n];                      // (a row that has met no token yet)
    float sum = 0.f;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = __builtin_amdgcn_exp2f(s[n][a][i] - level);
        p[n][0][4 * a + i] = (_Float16)w;
        if constexpr (kPieces<NR> == 2) p[n][1][4 * a + i] = (_Float16)(w - (float)p[n][0][4 * a + i]);
        sum += kPieces<NR> == 2 ? w : (float)p[n][0][4 * a + i];
      }
    r.l[n] = __builtin_fmaf(sum, u.inv, r.l[n]);
  }
}

// One tile's codes as they are loaded, and its scales.
struct Tile {
  u32x4 k[4], v[4];
  Scales scales;
};

template <int NR>
__device__ __forceinline__ void add_values(Rows<NR>& r, int x, const half8_t& v, const half8_t (&p)[NR][kPieces<NR>]) {
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int i = 0; i < kPieces<NR>; ++i) r.o[n][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[n][i], r.o[n][x], 0, 0, 0);
}
template <bool E4M3, int NR>
__device__ __forceinline__ void use_tile(Rows<NR>& r, const Tile& t) {
  float4_t s[NR][2];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
#pragma unroll
    for (int n = 0; n < NR; ++n) s[n][a] = float4_t{};
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      const u32x4 w = t.k[2 * a + st / 2];
      const half8_t k = st & 1 ? expand<E4M3>(w.z, w.w, codes_times<E4M3>(0)) : expand<E4M3>(w.x, w.y, codes_times<E4M3>(0));
#pragma unroll
      for (int n = 0; n < NR; ++n) s[n][a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, r.q[n][st], s[n][a], 0, 0, 0);
    }
  }
  half8_t p[NR][kPieces<NR>];
  weights<NR>(r, s, t.scales, p);
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      add_values<NR>(r, 2 * q + m, m ? expand<E4M3>(t.v[q].z, t.v[q].w, t.scales.values) : expand<E4M3>(t.v[q].x, t.v[q].y, t.scales.values), p);
}

// A sequence's fp16 tokens behind the packed ones, in order: the open ones, then the new ones.
struct Plain {
  const __half *ko, *vo, *kf, *vf;
  long long kp, vp;                    // from a new token to the next
  int open;
  __device__ __forceinline__ const __half* key(int i) const { return i < open ? ko + i * D : kf + (i - open) * kp; }
  __device__ __forceinline__ const __half* value(int i) const { return i < open ? vo + i * D : vf + (i - open) * vp; }
};

constexpr int W = 4;                                    // wavefronts of a work-group
template <int NR>
constexpr int kFloats = W * NR * (32 + 2) * 64;          // of LDS

// ws, slots: where partial results go, and how many it holds, each of slot_rows rows.
template <bool E4M3, int NR>
__device__ __forceinline__ void attend(const BlockAttnArgs& a, const BlockWork& work, float* lds, float* ws, long long slots, int slot_rows = 16 * NR) {
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int b = work.b, h = work.h;
  const long long bh = (long long)b * a.s.n_kv_heads + h;
  const BlockSeq s = block_seq(a, b);
  const int rows = s.t * a.heads_per_kv, row0 = work.row_block * 16 * NR;
  if (row0 >= rows) return;                              // (uniform)
  Rows<NR> r;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = row0 + 16 * n + c, i = row / a.heads_per_kv;
    const __half* src = a.q.p + b * a.q.batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.q.head + i * a.q.token + 32 * g;
#pragma unroll
    for (int st = 0; st < 4; ++st) r.q[n][st] = row < rows ? *reinterpret_cast<const half8_t*>(src + 8 * st) : half8_t{};
#pragma unroll
    for (int x = 0; x < 8; ++x) r.o[n][x] = float4_t{};
    r.m[n] = -INFINITY;
    r.l[n] = 0.f;
  }

  // this wavefront's share of the tiles: packed ones, then those of fp16 tokens
  const bool causal = a.k.p != nullptr;
  const int last_row = (row0 + 16 * NR < rows ? row0 + 16 * NR : rows) - 1;
  const int open = s.n - s.packed, plain = open + (causal ? last_row / a.heads_per_kv + 1 : 0);
  const int tiles1 = s.packed / kBlockTile, tiles = tiles1 + (plain + kBlockTile - 1) / kBlockTile;
  const int parts = work.n_splits * W, part = work.split * W + wave, share = tiles / parts, more = tiles % parts;
  const int t0 = part * share + (part < more ? part : more), t1 = t0 + share + (part < more ? 1 : 0);

  const int u1 = t1 < tiles1 ? t1 : tiles1;
  BlockUnits<E4M3> units;
  if (t0 < u1) {
    // (tiles are loaded two ahead; behind the last one: that one again)
    auto load = [&](int u, Tile& t) {
      u = u < u1 ? u : u1 - 1;
      units.look(a.s, b, h, u, u1, lane);
      const long long tile = units.tile(u) * kBlockTileBytes;
      const u32x4* kp = reinterpret_cast<const u32x4*>(a.s.k.codes + tile);
      const u32x4* vp = reinterpret_cast<const u32x4*>(a.s.v.codes + tile);
#pragma unroll
      for (int x = 0; x < 4; ++x) t.k[x] = __builtin_nontemporal_load(kp + 64 * x + lane);
#pragma unroll
      for (int x = 0; x < 4; ++x) t.v[x] = __builtin_nontemporal_load(vp + 64 * x + lane);
      t.scales = units.scales(u);
    };
    Tile x, y;
    load(t0, x);
    load(t0 + 1, y);
    for (int u = t0;;) {
      use_tile<E4M3, NR>(r, x);
      if (++u == u1) break;
      load(u + 1, x);
      use_tile<E4M3, NR>(r, y);
      if (++u == u1) break;
      load(u + 1, y);
    }
  }
  if (t1 > tiles1) {
    Plain p;
    const long long open_at = bh * a.s.block * D;
    p.ko = a.s.k.open + open_at;
    p.vo = a.s.v.open + open_at;
    p.kf = a.k.p + b * a.k.batch + h * a.k.head;
    p.vf = a.v.p + b * a.v.batch + h * a.v.head;
    p.kp = a.k.token;
    p.vp = a.v.token;
    p.open = open;
    const int shift = plain_shift(units.largest);
    const uint32_t by = half_power(-shift) * 0x10001u;
    auto shift_by = [&](int e) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        r.m[n] -= (float)e;
        r.l[n] = __builtin_amdgcn_ldexpf(r.l[n], e);
      }
    };
    if (shift) shift_by(shift);                          // (uniform)
    for (int u = t0 > tiles1 ? t0 : tiles1; u < t1; ++u) {
      const int i0 = (u - tiles1) * kBlockTile;
      auto token = [&](int i) { return i0 + i < plain ? i0 + i : plain - 1; };    // (behind the last one: that one again, masked)
      float4_t sc[NR][2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const __half* src = p.key(token(16 * x + c)) + 32 * g;
#pragma unroll
        for (int n = 0; n < NR; ++n) sc[n][x] = float4_t{};
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          const half8_t k = *reinterpret_cast<const half8_t*>(src + 8 * st);
#pragma unroll
          for (int n = 0; n < NR; ++n) sc[n][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, r.q[n][st], sc[n][x], 0, 0, 0);
        }
      }
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int row = row0 + 16 * n + c, limit = causal ? open + (row < rows ? row : rows - 1) / a.heads_per_kv : plain - 1;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i0 + 16 * x + 4 * g + i > limit) sc[n][x][i] = -INFINITY;
      }
      half8_t w[NR][kPieces<NR>];
      weights<NR>(r, sc, kPlainScales, w);
      const __half* vsrc[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) vsrc[j] = p.value(token(16 * (j >> 2) + 4 * g + (j & 3))) + 2 * c;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t x[8], e[4], o[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = times(*reinterpret_cast<const uint32_t*>(vsrc[j] + 32 * q), by);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          e[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
          o[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
        }
        add_values<NR>(r, 2 * q, __builtin_bit_cast(half8_t, u32x4{e[0], e[1], e[2], e[3]}), w);
        add_values<NR>(r, 2 * q + 1, __builtin_bit_cast(half8_t, u32x4{o[0], o[1], o[2], o[3]}), w);
      }
    }
    if (shift) shift_by(-shift);
  }

  // the wavefronts' results meet in LDS, each joins CH channels of a lane's eight in channels 32 q ..
  constexpr int CH = 32 / W;
  float* ml = lds + W * NR * 32 * 64;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) lds[((wave * NR + n) * 32 + 4 * x + i) * 64 + lane] = r.o[n][x][i];
    ml[((wave * NR + n) * 2) * 64 + lane] = r.m[n];
    ml[((wave * NR + n) * 2 + 1) * 64 + lane] = row_sum(r.l[n]);
  }
  __syncthreads();
  const int q = wave * CH / 8, from = wave * CH % 8;     // (channel 2 i + m of the eight is o[2 q + m][i])
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float top = -INFINITY, l = 0.f, o[CH];
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, ml[((w * NR + n) * 2) * 64 + lane]);
#pragma unroll
    for (int i = 0; i < CH; ++i) o[i] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float m = ml[((w * NR + n) * 2) * 64 + lane];
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      l = __builtin_fmaf(f, ml[((w * NR + n) * 2 + 1) * 64 + lane], l);
#pragma unroll
      for (int i = 0; i < CH; ++i) o[i] = __builtin_fmaf(f, lds[((w * NR + n) * 32 + 8 * q + 4 * (i & 1) + (from + i) / 2) * 64 + lane], o[i]);
    }
    const int row = row0 + 16 * n + c;
    if (row >= rows) continue;
    const int channel = 32 * q + 8 * g + from;
    if (work.n_splits > 1) {
      const long long slot_row = work.slot * slot_rows + 16 * n + c;
      float* dst = ws + slots * (slot_rows * 2) + slot_row * D + channel;
#pragma unroll
      for (int i = 0; i < CH; i += 4) *reinterpret_cast<float4*>(dst + i) = float4{o[i], o[i + 1], o[i + 2], o[i + 3]};
      if (wave == 0 && g == 0) *reinterpret_cast<float2*>(ws + slot_row * 2) = float2{top, l};
      continue;
    }
    const float f = l > 0.f ? 1.0f / l : 0.f;            // (no token: zero)
    const int i = row / a.heads_per_kv;
    const long long at = b * a.out_batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.out_head + i * a.out_token + channel;
#pragma unroll
    for (int e = 0; e < CH; e += 4) store_four(a, at + e, o[e] * f, o[e + 1] * f, o[e + 2] * f, o[e + 3] * f);
  }
}

}  // namespace block_few
}  // namespace innerq
