// What the kernels of attention over the cache in 8 bits share: codes as operands, the softmax level's constants, a sequence's counts.
#pragma once

#include "block.h"

namespace innerq {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// log2 of the weight that the largest score has when it raises the level, and of the largest weight before the level is raised.
constexpr float kTop = 9.0f, kRaise = 15.0f;
constexpr float kFar = 0x1p19f;                          // levels beyond: neighbours in fp32 are 2^-4 apart and more
constexpr float kFarShare = 0x1p-16f;                    // of its own size, by which a level is raised the sooner

// Eight codes as fp16, times a power of two.
template <bool E4M3>
__device__ __forceinline__ half8_t expand_by(uint32_t a, uint32_t b, float by) {
  half2_t h[4];
  if constexpr (E4M3) {
    h[0] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, false));
    h[1] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, true));
    h[2] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, false));
    h[3] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, true));
  } else {
    // (1024 + 128 + code under the exponent of 1024; exact for every power of two up to 1)
    const half2_t f = {(_Float16)by, (_Float16)by}, bias = f * (_Float16)-1152.f;
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    h[0] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)), f, bias);
    h[1] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)), f, bias);
    h[2] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)), f, bias);
    h[3] = __builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)), f, bias);
  }
  return half8_t{h[0].x, h[0].y, h[1].x, h[1].y, h[2].x, h[2].y, h[3].x, h[3].y};
}
template <bool E4M3>
__device__ __forceinline__ half8_t expand(uint32_t a, uint32_t b) { return expand_by<E4M3>(a, b, 1.f); }

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

}  // namespace innerq
