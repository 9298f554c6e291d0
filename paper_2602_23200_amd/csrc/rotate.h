// Rotary positions: the rotation of one token row's channels, shared by the launches that rotate.  Every translation unit that includes this is compiled with
// -ffp-contract=off: an output is fp16(fl(x1 c) -+ fl(x2 s)), each fp32 operation rounded by itself, so that rotating on the way
// into the cache, rotating beforehand and rotating in another program give the same bits.
#pragma once

#include "rows.h"

namespace innerq {
namespace {

// A row of 128 channels is eight units of two chunks of eight channels; unit u holds pairs 8 u .. 8 u + 7, or, from the rotated
// channels' end on, two chunks that pass through (rot_dim is a multiple of 16: no chunk is half rotated).
constexpr int kUnits = kHeadDim / 16;

struct UnitChunks { int a, b; };                         // first channels
__device__ __forceinline__ UnitChunks unit_chunks(const RotArgs& r, int u) {
  const bool halves = !r.interleaved && 8 * u < r.pairs;
  return {halves ? 8 * u : 16 * u, halves ? 8 * u + r.pairs : 16 * u + 8};
}

// Cosines and sines of a unit's eight pairs for one token.
struct Turn { float c[8], s[8]; };

__device__ __forceinline__ long long clamped_position(const RotArgs& r, int p) {
  return p < 0 ? 0 : p > r.last_position ? r.last_position : p;
}

// bt: index of the token in the positions of one axis; place: its position where there are none.
__device__ __forceinline__ void load_turn(Turn& x, const RotArgs& r, long long bt, int place, int u) {
  if (8 * u >= r.pairs) return;
  const uint32_t low = (uint32_t)(r.axis_low >> (8 * u)) & 0xffu, high = (uint32_t)(r.axis_high >> (8 * u)) & 0xffu;
  if (!r.positions || ((low == 0u || low == 0xffu) && (high == 0u || high == 0xffu))) {
    // (one axis for all eight: the tables' rows in wide loads)
    const int axis = (low ? 1 : 0) + (high ? 2 : 0);
    const long long at = clamped_position(r, r.positions ? r.positions[axis * r.axis_stride + bt] : place) * r.pairs + 8 * u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 c = *reinterpret_cast<const float4*>(r.cos + at + 4 * i), s = *reinterpret_cast<const float4*>(r.sin + at + 4 * i);
      x.c[4 * i] = c.x; x.c[4 * i + 1] = c.y; x.c[4 * i + 2] = c.z; x.c[4 * i + 3] = c.w;
      x.s[4 * i] = s.x; x.s[4 * i + 1] = s.y; x.s[4 * i + 2] = s.z; x.s[4 * i + 3] = s.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int axis = (int)(low >> i & 1u) + 2 * (int)(high >> i & 1u);
    const long long at = clamped_position(r, r.positions[axis * r.axis_stride + bt]) * r.pairs + 8 * u + i;
    x.c[i] = r.cos[at];
    x.s[i] = r.sin[at];
  }
}

// (the empty asm keeps the fp32 rounding of the sum apart from the conversion: one mixed-precision instruction would round once)
__device__ __forceinline__ __half turned_half(float x, float y) {
  float z = x + y;
  asm("" : "+v"(z));
  return __float2half_rn(z);
}

__device__ __forceinline__ void turn_unit(const Turn& t, const RotArgs& r, int u, uint4& a, uint4& b) {
  if (8 * u >= r.pairs) return;
  __half* x = reinterpret_cast<__half*>(&a);
  __half* y = reinterpret_cast<__half*>(&b);
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __half* p = i < 4 ? x + 2 * i : y + 2 * (i - 4);
      const float p0 = __half2float(p[0]), p1 = __half2float(p[1]);
      p[0] = turned_half(p0 * t.c[i], -(p1 * t.s[i]));
      p[1] = turned_half(p1 * t.c[i], p0 * t.s[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = __half2float(x[i]), p1 = __half2float(y[i]);
      x[i] = turned_half(p0 * t.c[i], -(p1 * t.s[i]));
      y[i] = turned_half(p1 * t.c[i], p0 * t.s[i]);
    }
  }
}

}  // namespace
}  // namespace innerq
