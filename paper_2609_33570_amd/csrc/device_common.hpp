// Device helpers shared by the gfx950 kernels (wave64, CDNA4).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hilore {

constexpr int kWave = 64;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// bf16 halves of a packed word -> fp32 (exact).
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two fp32 -> packed bf16 pair, round to nearest even (v_cvt_pk_bf16_f32;
// checked bit for bit against the software rule over every finite fp32).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// The 8 bf16 values of w as fp32 (exact).
__device__ __forceinline__ void unpack_bf16x8(u32x4 w, float v[8]) {
  v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x);
  v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
  v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z);
  v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}

__device__ __forceinline__ u32x4 pack_bf16x8(const float v[8]) {
  return u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
               pack_bf16(v[6], v[7])};
}

// 8 codes of an L unit as the bf16 values that decompress writes, in fp32
// (SCALED: times their block scale s and rounded; else exact values of the cast).
template <bool INT8, bool SCALED>
__device__ __forceinline__ void decode_codes8(u32x2 c, float s, float v[8]) {
  float q[8];
  if constexpr (INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[i] = (float)(int)__builtin_amdgcn_sbfe(c.x, 8 * i, 8);
      q[4 + i] = (float)(int)__builtin_amdgcn_sbfe(c.y, 8 * i, 8);
    }
  } else {
    f32x2 d;
    d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false); q[0] = d.x; q[1] = d.y;
    d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);  q[2] = d.x; q[3] = d.y;
    d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false); q[4] = d.x; q[5] = d.y;
    d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);  q[6] = d.x; q[7] = d.y;
  }
  if constexpr (SCALED) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t h = pack_bf16(q[i] * s, q[i + 1] * s);
      v[i] = bf16_lo(h);
      v[i + 1] = bf16_hi(h);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q[i];
  }
}

// Cross-lane operations inside a wave.  DPP controls (gfx9 encoding).
enum : int {
  kDppQuadXor1 = 0xB1,      // quad_perm [1,0,3,2]
  kDppQuadXor2 = 0x4E,      // quad_perm [2,3,0,1]
  kDppRowHalfMirror = 0x141,
  kDppRowMirror = 0x140,
};

// v and its DPP neighbour combined by an unsigned max: the DPP move folds
// into v_max_u32_dpp (lanes without a source read 0, the identity).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}

// Unsigned max over aligned groups of L lanes (L = 4, 8, 16 or 32); every
// lane of the group receives the group maximum.  After the quad steps each
// quad holds its max; the half-row mirror pairs quads 0<->1 and 2<->3, the
// row mirror pairs the two halves of a 16-lane row, and a swizzle pairs the
// two rows of 32.
template <int L>
__device__ __forceinline__ uint32_t group_max_u32(uint32_t v) {
  static_assert(L == 4 || L == 8 || L == 16 || L == 32, "group size");
  v = dpp_max_u32<kDppQuadXor1>(v);
  v = dpp_max_u32<kDppQuadXor2>(v);
  if constexpr (L >= 8) v = dpp_max_u32<kDppRowHalfMirror>(v);
  if constexpr (L >= 16) v = dpp_max_u32<kDppRowMirror>(v);
  if constexpr (L >= 32) v = max(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401F));
  return v;
}

// Largest magnitude of the 8 bf16 values of w, as bf16 bits in the low half
// (non-negative bf16 patterns order like their values; NaN is out of
// contract).
__device__ __forceinline__ uint32_t absmax_bf16x8(u32x4 w) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 a = __builtin_bit_cast(u16x2, w.x & 0x7FFF7FFFu);
  const u16x2 b = __builtin_bit_cast(u16x2, w.y & 0x7FFF7FFFu);
  const u16x2 c = __builtin_bit_cast(u16x2, w.z & 0x7FFF7FFFu);
  const u16x2 d = __builtin_bit_cast(u16x2, w.w & 0x7FFF7FFFu);
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(a, b),
                                            __builtin_elementwise_max(c, d));
  return max((uint32_t)m.x, (uint32_t)m.y);
}

// Sum over the whole wave as a butterfly (xor 1, 2, 4, ..., 32).  Addition
// is commutative, so every lane ends with the same value: the pairwise tree
// (first half) + (second half), recursively, over the 64 lanes.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

// The value that a DPP control brings to the lane (the controls above have a source for
// every lane).
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Largest unsigned value over aligned groups of 32 (L = 32) or all 64 lanes, all of them
// receiving it, without LDS instructions: DPP within rows of 16, then the rows swapped in
// pairs, then the halves.
template <int L>
__device__ __forceinline__ uint32_t lanes_max_u32(uint32_t v) {
  static_assert(L == 32 || L == 64, "group size");
  v = group_max_u32<16>(v);
  auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(p[0], p[1]);
  if constexpr (L == 64) {
    p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(p[0], p[1]);
  }
  return v;
}

// wave_sum's tree, and so its bits, without LDS instructions.
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp_f32<kDppQuadXor1>(v);
  v += dpp_f32<kDppQuadXor2>(v);
  v += dpp_f32<kDppRowHalfMirror>(v);
  v += dpp_f32<kDppRowMirror>(v);
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Rounding of a token's values to int8: the factor 127 / amax and the scale amax / 127.
// Below 2^-64 both are 0; an infinite or NaN amax gives factor 0 and scale NaN.
__device__ __forceinline__ float token_scale(float amax, float &scale) {
  if (amax < 0x1p-64f) {
    scale = 0.0f;
    return 0.0f;
  }
  if (!(amax < __builtin_inff())) {
    scale = __builtin_nanf("");
    return 0.0f;
  }
  scale = amax / 127.0f;
  return 127.0f / amax;
}

// 8 codes RNE(v * r), clamped to [-127, 127]; 0 where r is 0 (v may be anything then).
__device__ __forceinline__ u32x2 token_codes8(const float v[8], float r) {
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = __builtin_amdgcn_fmed3f(rintf(v[i] * r), -127.0f, 127.0f);
    c[i] = r == 0.0f ? 0u : (uint32_t)(int)q & 0xFFu;
  }
  return u32x2{c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24};
}

}  // namespace hilore
