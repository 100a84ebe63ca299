// Backward of the gated MLP activation on gfx950, with an L unit decoded in
// registers.  The evaluated models' MLP computes h = silu(g) * u from the gate
// and up projections g and u (silu(g) = g * sigmoid(g)); when g or u is an L
// unit, backward consumes its reconstruction (App. B.1 Eq. fp8-roundtrip):
//   du = dh * silu(g)
//   dg = dh * u * sigmoid(g) * (1 + g * (1 - sigmoid(g)))
// An L operand is xhat = bf16_RNE(value(code) * scale), bit for bit the value
// hilore_decompress writes, formed in registers and never stored; a bf16
// operand is read as is.  Arithmetic in fp32 (sigmoid from the hardware exp2
// and reciprocal), each output rounded once to bf16 (RNE).
//
// Elementwise and bound by HBM: per element 2 B of dh, 1 + 4/BLOCK B per L
// operand or 2 B per bf16 operand, 4 B of outputs.  A thread takes 8
// consecutive columns of one row (16-byte loads and stores, 8-byte code loads),
// all touched once, so loads and stores are non-temporal.  A workgroup is one
// wave covering 512 columns of a row (4.5 KiB at 9 B per element) and the grid
// is one pass of such short-lived workgroups, columns fastest, rows on the
// grid's second dimension: on 16384 x 18944 this ran ~17% faster than
// 256-thread workgroups over 2048 columns.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 64;
constexpr int kColsPerThread = 8;
constexpr int kRowGrid = 65535;

// The raw bits of 8 values of one operand at (row, col .. col+7): a bf16
// operand's 16 bytes, or an L operand's 8 code bytes and its block scale.
struct Raw {
  u32x4 w;
  u32x2 c;
  float s;
};

template <int CODE, int BLOCK, bool L>
__device__ __forceinline__ void load_operand(const uint16_t *x, const uint8_t *codes,
                                             const float *scales, int64_t ld, int64_t cols,
                                             int64_t row, int64_t col, Raw &r) {
  if constexpr (!L) {
    r.w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(x + row * ld + col));
  } else {
    r.c = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(codes + row * cols + col));
    if constexpr (CODE != kCodeCast) r.s = scales[row * (cols / BLOCK) + col / BLOCK];
  }
}

// The 8 values as fp32: an L operand decoded exactly as decompress does it.
template <int CODE, bool L>
__device__ __forceinline__ void decode_operand(const Raw &r, float v[8]) {
  if constexpr (!L) unpack_bf16x8(r.w, v);
  else decode_codes8<CODE == kCodeInt8, CODE != kCodeCast>(r.c, r.s, v);
}

template <int CODE, int BLOCK, bool GL, bool UL>
__global__ __launch_bounds__(kThreads) void swiglu_bwd_kernel(const SwigluArgs a) {
  const int64_t col = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kColsPerThread;
  if (col >= a.cols) return;
  constexpr float kLog2e = 1.44269504088896340736f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    Raw rg, ru;
    load_operand<CODE, BLOCK, GL>(a.g_x, a.g_codes, a.g_scales, a.g_ld, a.cols, row, col, rg);
    load_operand<CODE, BLOCK, UL>(a.u_x, a.u_codes, a.u_scales, a.u_ld, a.cols, row, col, ru);
    const u32x4 dw =
        __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.dh + row * a.cols + col));
    float g[8], u[8], d[8];
    decode_operand<CODE, GL>(rg, g);
    decode_operand<CODE, UL>(ru, u);
    unpack_bf16x8(dw, d);
    float og[8], ou[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // sigmoid(g) = 1 / (1 + 2^(-g log2 e)); exp2 overflows to inf for very
      // negative g, giving sigmoid 0 as it should
      const float e = __builtin_amdgcn_exp2f(-g[i] * kLog2e);
      const float sg = __builtin_amdgcn_rcpf(1.0f + e);
      ou[i] = d[i] * (g[i] * sg);
      og[i] = (d[i] * u[i]) * (sg * (1.0f + g[i] * (1.0f - sg)));
    }
    __builtin_nontemporal_store(pack_bf16x8(og),
                                reinterpret_cast<u32x4 *>(a.dg + row * a.cols + col));
    __builtin_nontemporal_store(pack_bf16x8(ou),
                                reinterpret_cast<u32x4 *>(a.du + row * a.cols + col));
  }
}

template <int CODE, int BLOCK, bool GL, bool UL>
void launch_one(const SwigluArgs &a, hipStream_t s) {
  const int64_t chunks = (a.cols / kColsPerThread + kThreads - 1) / kThreads;
  const int64_t rg = a.rows < kRowGrid ? a.rows : kRowGrid;
  hipLaunchKernelGGL((swiglu_bwd_kernel<CODE, BLOCK, GL, UL>), dim3((unsigned)chunks, (unsigned)rg),
                     dim3(kThreads), 0, s, a);
}

template <int CODE, int BLOCK>
void by_operands(const SwigluArgs &a, hipStream_t s) {
  const bool gl = a.g_codes != nullptr, ul = a.u_codes != nullptr;
  if (gl && ul) launch_one<CODE, BLOCK, true, true>(a, s);
  else if (gl) launch_one<CODE, BLOCK, true, false>(a, s);
  else launch_one<CODE, BLOCK, false, true>(a, s);
}

template <int CODE>
void by_block(const SwigluArgs &a, int block, hipStream_t s) {
  switch (block) {
    case 32: return by_operands<CODE, 32>(a, s);
    case 64: return by_operands<CODE, 64>(a, s);
    case 128: return by_operands<CODE, 128>(a, s);
    default: return by_operands<CODE, 256>(a, s);
  }
}

}  // namespace

hipError_t launch_swiglu_bwd(const SwigluArgs &a, int code, int block, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  if (a.g_codes == nullptr && a.u_codes == nullptr) launch_one<kCodeInt8, 256, false, false>(a, s);
  else if (code == kCodeCast) by_operands<kCodeCast, 256>(a, s);  // no blocks; BLOCK unused
  else if (code == kCodeInt8) by_block<kCodeInt8>(a, block, s);
  else by_block<kCodeE4M3>(a, block, s);
  return hipGetLastError();
}

}  // namespace hilore
