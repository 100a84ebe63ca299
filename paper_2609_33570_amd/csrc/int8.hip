// Linear layer with int8 weights (one scale per output channel) and its operand
// rounded to int8 with one scale per token, on gfx950 MFMA:
//   out[t][n] = (sum_k a[t][k] w[n][k]) * sa_t * sw_n + bias[n]
// The sums are exact in int32 (k <= 2^17), whatever the order.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ------------------------------------------------------- rounding of tokens --
constexpr int kQuantThreads = 256;

// 8 values of x * factor at col.
__device__ __forceinline__ void load_scaled8(const uint16_t *x, const float *factor, int64_t col,
                                             float v[8]) {
  unpack_bf16x8(*reinterpret_cast<const u32x4 *>(x + col), v);
  if (factor) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= factor[col + i];
  }
}

__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const QuantArgs a) {
  __shared__ uint32_t lds[kQuantThreads / kWave];
  for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
  const uint16_t *x = a.x + row * a.ldx;
  uint32_t top = 0;
  for (int64_t col = threadIdx.x * 8; col < a.k; col += kQuantThreads * 8) {
    float v[8];
    load_scaled8(x, a.factor, col, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(fabsf(v[i])));
  }
  top = group_max_u32<32>(top);
  top = max(top, (uint32_t)__shfl_xor((int)top, 32, kWave));
  __syncthreads();  // of the row before
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int w = 0; w < kQuantThreads / kWave; ++w) top = max(top, lds[w]);
  float scale;
  const float r = token_scale(__uint_as_float(top), scale);
  if (threadIdx.x == 0) a.scales[row] = scale;
  for (int64_t col = threadIdx.x * 8; col < a.k; col += kQuantThreads * 8) {
    float v[8];
    load_scaled8(x, a.factor, col, v);
    *reinterpret_cast<u32x2 *>(a.codes + row * a.k + col) = token_codes8(v, r);
  }
  }
}

// ------------------------------------------------------------------ product --
// One value of the output: the exact sum, scaled, with bias, added or written.
__device__ __forceinline__ void finish(const Int8Args &a, int64_t t, int64_t n, int sum) {
  float v = (float)sum * a.a_scales[t];
  if (a.w_scales) v *= a.w_scales[n];
  if (a.bias) v += __uint_as_float((uint32_t)a.bias[n] << 16);
  if (a.out_f32) {
    float *o = static_cast<float *>(a.out) + t * a.ldo + n;
    *o = a.accumulate ? *o + v : v;
  } else {
    uint16_t *o = static_cast<uint16_t *>(a.out) + t * a.ldo + n;
    if (a.accumulate) v += __uint_as_float((uint32_t)*o << 16);
    *o = (uint16_t)pack_bf16(v, 0.0f);
  }
}

// 64 x 64 outputs per workgroup, 32 x 32 per wave, operands straight from memory.
__global__ __launch_bounds__(256) void int8_kernel(const Int8Args a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t tiles_n = (uint32_t)((a.n + 63) / 64);
  const int64_t t0 = (int64_t)(blockIdx.x / tiles_n) * 64 + (wave >> 1) * 32;
  const int64_t n0 = (int64_t)(blockIdx.x % tiles_n) * 64 + (wave & 1) * 32;
  const int64_t ta = t0 + (lane & 31) < a.tokens ? t0 + (lane & 31) : a.tokens - 1;
  const int64_t nb = n0 + (lane & 31) < a.n ? n0 + (lane & 31) : a.n - 1;
  const int8_t *pa = a.a + ta * a.k, *pb = a.w + nb * a.k;
  i32x16 acc = {};
  for (int k = (lane >> 5) * 16; k < a.k + (lane >> 5) * 16; k += 32) {
    i32x4 x = {}, y = {};
    if (k < a.k) {
      x = *reinterpret_cast<const i32x4 *>(pa + k);
      y = *reinterpret_cast<const i32x4 *>(pb + k);
    }
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, y, acc, 0, 0, 0);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int64_t t = t0 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3), n = n0 + (lane & 31);
    if (t < a.tokens && n < a.n) finish(a, t, n, acc[r]);
  }
}

}  // namespace

hipError_t launch_quantize_tokens(const QuantArgs &a, hipStream_t s) {
  if (a.tokens == 0) return hipSuccess;
  const unsigned groups = (unsigned)(a.tokens < (1 << 20) ? a.tokens : 1 << 20);
  hipLaunchKernelGGL(quantize_kernel, dim3(groups), dim3(kQuantThreads), 0, s, a);
  return hipGetLastError();
}

size_t int8_part_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_int8(const Int8Args &a, hipStream_t s) {
  if (a.tokens == 0 || a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(int8_kernel, dim3((unsigned)(((a.n + 63) / 64) * ((a.tokens + 63) / 64))),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hilore
