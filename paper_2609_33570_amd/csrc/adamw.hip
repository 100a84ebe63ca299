// AdamW over many tensors and the global norm of their gradients, on gfx950.
//
// Step, g = clip * grad:
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr wd) - lr (m / c1) / (sqrt(v / c2) + eps),  c = 1 - beta^step
// States in 32 bits are m and v.  States in 8 bits are E4M3FN codes of m and of
// r = sqrt(v) (half of v's range in binades, so that 18 binades of a block's r
// survive) in blocks of 256 with fp32 scale amax / 448.
//
// Rounding of an 8-bit state is random and unbiased: with beta2 = 0.999 a step
// changes v by a thousandth of itself, a sixtieth of half a code's spacing, and
// rounding to nearest would keep the old code forever.  The scaled magnitude times
// 2^-120 has the exponent field of an E4M3FN (subnormals included), so the code
// is (bits + 20 random bits) >> 20; the hash gives the upper 16 of them.
//
// Bound by HBM: per element 28 B with everything in fp32 (p, m, v read and
// written, g read), 10 B with bf16 parameters and gradients and 8-bit states.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 256;
constexpr int kLaneElems = 4;                       // consecutive elements of a lane
constexpr int kBlock = kWave * kLaneElems;          // 256: one state block a wave
constexpr int kBlocksPerWave = (int)(kAdamwChunk / kThreads / kLaneElems);
static_assert(kBlock == kAdamwBlock, "a wave owns one state block at a time");

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Largest unsigned value of the wave (all lanes receive it).
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = group_max_u32<32>(v);
  return max(v, (uint32_t)__shfl_xor((int)v, 32, kWave));
}

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// Four consecutive elements at p + i, of which `n` exist; the others read as 0.
__device__ __forceinline__ void load4(const float *p, int64_t i, int n, float v[4]) {
  if (n >= 4) {
    const f32x4 w = *reinterpret_cast<const f32x4 *>(p + i);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = k < n ? p[i + k] : 0.0f;
  }
}

__device__ __forceinline__ void store4(float *p, int64_t i, int n, const float v[4]) {
  if (n >= 4) {
    *reinterpret_cast<f32x4 *>(p + i) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) p[i + k] = v[k];
  }
}

__device__ __forceinline__ void load4(const uint16_t *p, int64_t i, int n, float v[4]) {
  if (n >= 4) {
    const u32x2 w = *reinterpret_cast<const u32x2 *>(p + i);
    v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x);
    v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = k < n ? __uint_as_float((uint32_t)p[i + k] << 16) : 0.0f;
  }
}

__device__ __forceinline__ void store4_bf16(uint16_t *p, int64_t i, int n, uint32_t lo,
                                            uint32_t hi) {
  if (n >= 4) {
    *reinterpret_cast<u32x2 *>(p + i) = u32x2{lo, hi};
  } else {
    if (n > 0) p[i] = (uint16_t)lo;
    if (n > 1) p[i + 1] = (uint16_t)(lo >> 16);
    if (n > 2) p[i + 2] = (uint16_t)hi;
  }
}

__device__ __forceinline__ uint32_t load4_codes(const uint8_t *p, int64_t i, int n) {
  if (n >= 4) return *reinterpret_cast<const uint32_t *>(p + i);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) w |= (uint32_t)p[i + k] << (8 * k);
  return w;
}

__device__ __forceinline__ void store4_codes(uint8_t *p, int64_t i, int n, uint32_t w) {
  if (n >= 4) {
    *reinterpret_cast<uint32_t *>(p + i) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) p[i + k] = (uint8_t)(w >> (8 * k));
  }
}

__device__ __forceinline__ void decode4(uint32_t c, float s, float v[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  v[0] = a.x * s; v[1] = a.y * s; v[2] = b.x * s; v[3] = b.y * s;
}

// Codes of a block's values (this lane's 4) with 16 random bits each, and its scale.
template <bool KEEP>
__device__ __forceinline__ uint32_t encode4(const float x[4], const uint32_t bits[4], float &scale) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) top = max(top, __float_as_uint(fabsf(x[k])));
  const float amax = __uint_as_float(wave_max_u32(top));
  const bool none = amax < 0x1p-64f;
  scale = none ? 0.0f : amax * (1.0f / 448.0f);
  const float r = none ? 0.0f : 448.0f * (1.0f / amax);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = fabsf(x[k]) * r * 0x1p-120f;
    uint32_t c = min((__float_as_uint(a) + (bits[k] << 4)) >> 20, 0x7Eu);
    if constexpr (KEEP) c = x[k] > 0.0f && !none ? max(c, 1u) : c;
    else c |= (__float_as_uint(x[k]) >> 24) & 0x80u;
    w |= c << (8 * k);
  }
  return w;
}

struct Scalars {
  float beta1, one_beta1, beta2, one_beta2, eps, inv_sqrt_c2;
};

// One chunk of one tensor.  PARAM: 0 fp32, 1 fp32 with a bf16 copy, 2 bf16.
template <bool EIGHT, bool GRAD16, int PARAM>
__device__ __forceinline__ void step_chunk(const AdamwTensor &t, int64_t begin, float clip,
                                           const Scalars &s) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int b = 0; b < kBlocksPerWave; ++b) {
    const int64_t block = begin / kBlock + b * (kThreads / kWave) + wave;
    const int64_t i = block * kBlock + lane * kLaneElems;
    if (block * kBlock >= t.n) return;  // the whole wave
    const int64_t left = t.n - i;
    const int n = left >= 4 ? 4 : left > 0 ? (int)left : 0;
    float p[4], g[4], m[4], v[4], r[4];
    if constexpr (PARAM == 2) load4(t.p16, i, n, p);
    else load4(t.p, i, n, p);
    if constexpr (GRAD16) load4(static_cast<const uint16_t *>(t.grad), i, n, g);
    else load4(static_cast<const float *>(t.grad), i, n, g);
    if constexpr (EIGHT) {
      const uint32_t mc = load4_codes(static_cast<const uint8_t *>(t.m), i, n);
      const uint32_t vc = load4_codes(static_cast<const uint8_t *>(t.v), i, n);
      decode4(mc, t.m_scales[block], m);
      decode4(vc, t.v_scales[block], r);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = r[k] * r[k];
    } else {
      load4(static_cast<const float *>(t.m), i, n, m);
      load4(static_cast<const float *>(t.v), i, n, v);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float gk = g[k] * clip;
      m[k] = s.beta1 * m[k] + s.one_beta1 * gk;
      v[k] = s.beta2 * v[k] + s.one_beta2 * (gk * gk);
      r[k] = sqrtf(v[k]);
      // rcp is within 1 ulp; eps keeps its operand a normal number
      p[k] = p[k] * t.decay -
             (t.step_size * m[k]) * __builtin_amdgcn_rcpf(r[k] * s.inv_sqrt_c2 + s.eps);
    }
    if constexpr (EIGHT) {
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t w = mix32((uint32_t)(i + k) ^ t.key_state);
        lo[k] = w & 0xFFFFu;
        hi[k] = w >> 16;
      }
      float ms, vs;
      const uint32_t mc = encode4<false>(m, lo, ms);
      const uint32_t vc = encode4<true>(r, hi, vs);
      store4_codes(static_cast<uint8_t *>(t.m), i, n, mc);
      store4_codes(static_cast<uint8_t *>(t.v), i, n, vc);
      if (lane == 0) {
        t.m_scales[block] = ms;
        t.v_scales[block] = vs;
      }
    } else {
      store4(static_cast<float *>(t.m), i, n, m);
      store4(static_cast<float *>(t.v), i, n, v);
    }
    if constexpr (PARAM != 2) store4(t.p, i, n, p);
    if constexpr (PARAM == 1)
      store4_bf16(t.p16, i, n, pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]));
    if constexpr (PARAM == 2) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // NaN and infinity have no bits to round
        const uint32_t u = __float_as_uint(p[k]);
        const uint32_t q = mix32((uint32_t)(i + k) ^ t.key_param) & 0xFFFFu;
        w[k] = (u & 0x7F800000u) == 0x7F800000u ? u | ((u & 0xFFFFu) ? 0x10000u : 0u) : u + q;
      }
      store4_bf16(t.p16, i, n, (w[0] >> 16) | (w[1] & 0xFFFF0000u),
                  (w[2] >> 16) | (w[3] & 0xFFFF0000u));
    }
  }
}

// Tensor of workgroup `b`: the last one whose chunks begin at or before it.
__device__ __forceinline__ int tensor_of(const uint32_t *begin, int n, int64_t b) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (begin[mid] <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamwBatch a) {
  float clip = 1.0f;
  if (a.norm) {
    clip = a.norm[1];
    if (!(clip <= 1.0f)) return;  // NaN: the step is skipped
  }
  const int k = tensor_of(a.begin, a.n, blockIdx.x);
  const AdamwTensor &t = a.t[k];
  const int64_t begin = ((int64_t)blockIdx.x - a.begin[k]) * kAdamwChunk;
  const Scalars s = {a.beta1, a.one_beta1, a.beta2, a.one_beta2, a.eps, a.inv_sqrt_c2};
  const int param = t.p ? (t.p16 ? 1 : 0) : 2;
  const int kind = (t.m_scales ? 6 : 0) + (t.grad16 ? 3 : 0) + param;
  switch (kind) {
    case 0: return step_chunk<false, false, 0>(t, begin, clip, s);
    case 1: return step_chunk<false, false, 1>(t, begin, clip, s);
    case 2: return step_chunk<false, false, 2>(t, begin, clip, s);
    case 3: return step_chunk<false, true, 0>(t, begin, clip, s);
    case 4: return step_chunk<false, true, 1>(t, begin, clip, s);
    case 5: return step_chunk<false, true, 2>(t, begin, clip, s);
    case 6: return step_chunk<true, false, 0>(t, begin, clip, s);
    case 7: return step_chunk<true, false, 1>(t, begin, clip, s);
    case 8: return step_chunk<true, false, 2>(t, begin, clip, s);
    case 9: return step_chunk<true, true, 0>(t, begin, clip, s);
    case 10: return step_chunk<true, true, 1>(t, begin, clip, s);
    default: return step_chunk<true, true, 2>(t, begin, clip, s);
  }
}

// ------------------------------------------------------------------ norm --
// Sum of v over the workgroup in a fixed order; thread 0 receives it.
__device__ __forceinline__ double group_sum(double v, double *lds) {
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double sum = 0.0;
  for (int w = 0; w < (int)blockDim.x / kWave; ++w) sum += lds[w];
  return sum;
}

// Sum of squares of one chunk of one gradient, in fp64 (an fp32 square would
// overflow from 2^64 on and vanish below 2^-75).
__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const NormBatch a) {
  __shared__ double lds[kThreads / kWave];
  const int k = tensor_of(a.begin, a.n, blockIdx.x);
  const NormTensor &t = a.t[k];
  const int64_t begin = ((int64_t)blockIdx.x - a.begin[k]) * kNormChunk;
  double sum = 0.0;
#pragma unroll 4
  for (int j = 0; j < (int)(kNormChunk / kThreads / 4); ++j) {
    const int64_t i = begin + (j * kThreads + (int)threadIdx.x) * 4;
    const int64_t left = t.n - i;
    const int n = left >= 4 ? 4 : left > 0 ? (int)left : 0;
    float g[4];
    if (t.grad16) load4(static_cast<const uint16_t *>(t.grad), i, n, g);
    else load4(static_cast<const float *>(t.grad), i, n, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = fma((double)g[e], (double)g[e], sum);
  }
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

constexpr int kFoldThreads = 1024;

__global__ __launch_bounds__(kFoldThreads) void norm_fold_kernel(const double *part, int64_t n,
                                                                 float max_norm, float *norm) {
  __shared__ double lds[kFoldThreads / kWave];
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kFoldThreads) sum += part[i];
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) {
    // the sum rounded to 24 bits, then fp32 operations (a 53-bit root of 24 bits rounds
    // to the same fp32 as theirs; fp32's exponents would not hold every sum)
    const uint64_t u = __builtin_bit_cast(uint64_t, sum);
    const double sum24 =
        __builtin_bit_cast(double, (u + 0xFFFFFFFu + ((u >> 29) & 1u)) & ~uint64_t(0x1FFFFFFF));
    const float total = (float)sqrt(sum24);
    const float f = max_norm / (total + 1e-6f);
    norm[0] = total;
    norm[1] = !(total < __builtin_inff()) ? __builtin_nanf("") : f < 1.0f ? f : 1.0f;
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwBatch &a, hipStream_t s) {
  hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)a.begin[a.n]), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_norm_partial(const NormBatch &a, hipStream_t s) {
  hipLaunchKernelGGL(norm_partial_kernel, dim3((unsigned)a.begin[a.n]), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_norm_fold(const double *part, int64_t n, float max_norm, float *norm,
                            hipStream_t s) {
  hipLaunchKernelGGL(norm_fold_kernel, dim3(1), dim3(kFoldThreads), 0, s, part, n, max_norm, norm);
  return hipGetLastError();
}

// Key of the random bits of tensor `index` of a call.
uint32_t adamw_key(uint32_t seed, int index, uint32_t salt) {
  uint32_t x = seed + 0x9E3779B1u * (uint32_t)(index + 1) + salt;
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

}  // namespace hilore
