// RMS norms on leaving a block and entering the next, fused with the block's gate
// and residual scale, and their backward, on gfx950.  N(v) = v rsqrt(mean(v^2) + eps):
//   h = bf16(res + scale * gate * (N(y) * w_post)),   n = N(h) * w_pre
// n is the norm of h as stored, so it can be recomputed from a kept h.
//
// Bound by HBM: forward reads res and y and writes h and n, 8 B an element (7 with
// int8 codes for n); backward reads h, y, dn and dh and writes dres and dy, 12 B
// (an L unit's operand 1 + 4/block B).
//
// A workgroup owns a row at a time and keeps it in registers between the passes
// over it: every thread holds up to V pieces of 8 columns, `threads` pieces apart,
// so that each load is 16 bytes a lane and contiguous over the wave.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kMaxWaves = kMaxThreads / kWave;

enum Gate : int { kGateNone = 0, kGateChannel = 1, kGateToken = 2, kGateElement = 3 };

// N sums over the workgroup, in a fixed order; all threads receive them.  `lds` has
// a slot of its own for every use in a row, so one barrier is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*lds)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) lds[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = lds[0][k];
    for (int w = 1; w < waves; ++w) v[k] += lds[w][k];
  }
}

__device__ __forceinline__ u32x4 load16(const uint16_t *p) {
  return *reinterpret_cast<const u32x4 *>(p);
}

// The gate's 8 values at (row, col ..), 1 without a gate.
__device__ __forceinline__ void load_gate(const uint16_t *gate, int kind, int64_t row, int col,
                                          int cols, float g[8]) {
  if (kind == kGateChannel) {
    unpack_bf16x8(load16(gate + col), g);
  } else if (kind == kGateElement) {
    unpack_bf16x8(load16(gate + row * cols + col), g);
  } else {
    const float v = kind == kGateToken ? __uint_as_float((uint32_t)gate[row] << 16) : 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = v;
  }
}

template <int V>
__global__ __launch_bounds__(kMaxThreads) void block_norm_kernel(const BlockNormArgs a) {
  __shared__ float lds[2][kMaxWaves][1];
  __shared__ uint32_t lds_max[kMaxWaves];
  const int64_t row = blockIdx.x;
  const int threads = blockDim.x;
  float h[V][8];
  float sum[1];
  // y, its norm and its gate
  float r_post = 1.0f;
  if (a.y) {
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      unpack_bf16x8(load16(a.y + row * a.ld_y + col), h[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
    }
    if (a.w_post) {
      sum[0] = ss;
      group_sum<1>(sum, lds[0]);
      r_post = 1.0f / sqrtf(sum[0] * a.inv_cols + a.eps);
      if (a.rstd_post && threadIdx.x == 0) a.rstd_post[row] = r_post;
    }
  }
  // h, rounded as it is stored
  float ss = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * threads + (int)threadIdx.x) * 8;
    if (col >= a.cols) continue;
    u32x4 stored = load16(a.res + row * a.ld_res + col);
    if (a.y) {
      float res[8], g[8];
      unpack_bf16x8(stored, res);
      if (a.w_post) {
        float w[8];
        unpack_bf16x8(load16(a.w_post + col), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r_post * w[i];
      }
      load_gate(a.gate, a.gate_kind, row, col, a.cols, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) res[i] += a.scale * (h[v][i] * g[i]);
      stored = pack_bf16x8(res);
    }
    if (a.h) *reinterpret_cast<u32x4 *>(a.h + row * a.cols + col) = stored;
    unpack_bf16x8(stored, h[v]);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
  }
  if (!a.w_pre) return;
  sum[0] = ss;
  group_sum<1>(sum, lds[1]);
  const float r_pre = 1.0f / sqrtf(sum[0] * a.inv_cols + a.eps);
  if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[row] = r_pre;
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * threads + (int)threadIdx.x) * 8;
    if (col >= a.cols) continue;
    float w[8];
    unpack_bf16x8(load16(a.w_pre + col), w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[v][i] = h[v][i] * r_pre * w[i];
      top = max(top, __float_as_uint(fabsf(h[v][i])));
    }
    if (a.n) *reinterpret_cast<u32x4 *>(a.n + row * a.cols + col) = pack_bf16x8(h[v]);
  }
  if (!a.codes) return;
  top = group_max_u32<32>(top);
  top = max(top, (uint32_t)__shfl_xor((int)top, 32, kWave));
  const int waves = threads >> 6;
  if (waves > 1) {
    if ((threadIdx.x & 63) == 0) lds_max[threadIdx.x >> 6] = top;
    __syncthreads();
    top = lds_max[0];
    for (int w = 1; w < waves; ++w) top = max(top, lds_max[w]);
  }
  float scale;
  const float r = token_scale(__uint_as_float(top), scale);
  if (threadIdx.x == 0) a.code_scales[row] = scale;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * threads + (int)threadIdx.x) * 8;
    if (col >= a.cols) continue;
    *reinterpret_cast<u32x2 *>(a.codes + row * a.cols + col) = token_codes8(h[v], r);
  }
}

// --------------------------------------------------------------- backward --
// 8 values of a saved tensor.  CODE: -1 bf16, else the code of L units.
template <int CODE>
__device__ __forceinline__ void load_saved(const SavedRows &s, int64_t row, int col, int cols,
                                           int block_log2, float v[8]) {
  if (CODE >= 0 && s.codes) {
    const u32x2 c = *reinterpret_cast<const u32x2 *>(s.codes + row * cols + col);
    float f = 1.0f;
    if constexpr (CODE != kCodeCast)
      f = s.scales[row * (cols >> block_log2) + (col >> block_log2)];
    decode_codes8<CODE == kCodeInt8, CODE != kCodeCast>(c, f, v);
  } else {
    unpack_bf16x8(load16(s.x + row * s.ld + col), v);
  }
}

// SUMS: keep this workgroup's sums over its rows of dn * hh, dz * yh and a channel's
// dgate in registers and write them to the workspace at the end.
template <int V, int CODE, bool SUMS>
__global__ __launch_bounds__(kMaxThreads) void block_norm_bwd_kernel(const BlockNormBwdArgs a) {
  __shared__ float lds1[2][kMaxWaves][1], lds2[2][kMaxWaves][2];
  const int threads = blockDim.x;
  float s_pre[SUMS ? V : 1][8], s_post[SUMS ? V : 1][8], s_gate[SUMS ? V : 1][8];
  if constexpr (SUMS)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s_pre[v][i] = s_post[v][i] = s_gate[v][i] = 0.0f;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float d[V][8];
    // through the norm before the next block
    float r_pre = 0.0f, c1 = 0.0f;
    float hh[V][8];
    if (a.dn) {
      r_pre = a.rstd_pre[row];
      float sum[1] = {0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * threads + (int)threadIdx.x) * 8;
        if (col >= a.cols) continue;
        float w[8];
        load_saved<CODE>(a.h, row, col, a.cols, a.block_log2, hh[v]);
        unpack_bf16x8(load16(a.dn + row * a.ld_dn + col), d[v]);
        unpack_bf16x8(load16(a.w_pre + col), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          hh[v][i] *= r_pre;
          if constexpr (SUMS) s_pre[v][i] = fmaf(d[v][i], hh[v][i], s_pre[v][i]);
          d[v][i] *= w[i];
          sum[0] = fmaf(d[v][i], hh[v][i], sum[0]);
        }
      }
      group_sum<1>(sum, lds1[turn]);
      c1 = sum[0] * a.inv_cols;
    }
    // D, and the sums of y's norm and of a token's gate
    const bool need_y = a.y.x || a.y.codes;
    const float r_post = a.w_post ? a.rstd_post[row] : 1.0f;
    float sum[2] = {0.0f, 0.0f};
    float yh[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      float dh[8] = {};
      if (a.dh) unpack_bf16x8(load16(a.dh + row * a.cols + col), dh);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        d[v][i] = a.dn ? dh[i] + r_pre * (d[v][i] - hh[v][i] * c1) : dh[i];
      if (a.dres) *reinterpret_cast<u32x4 *>(a.dres + row * a.cols + col) = pack_bf16x8(d[v]);
      float w[8], g[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.0f;
      if (a.w_post) unpack_bf16x8(load16(a.w_post + col), w);
      load_gate(a.gate, a.gate_kind, row, col, a.cols, g);
      if (need_y) load_saved<CODE>(a.y, row, col, a.cols, a.block_log2, yh[v]);
      float dg[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[v][i] *= a.scale;
        if (need_y) {
          yh[v][i] *= r_post;
          dg[i] = d[v][i] * (yh[v][i] * w[i]);
          sum[1] += dg[i];
          if constexpr (SUMS) s_gate[v][i] += dg[i];
        }
        d[v][i] *= g[i];
        if (need_y) {
          if constexpr (SUMS) s_post[v][i] = fmaf(d[v][i], yh[v][i], s_post[v][i]);
          d[v][i] *= w[i];
          sum[0] = fmaf(d[v][i], yh[v][i], sum[0]);
        }
      }
      if (a.dgate && a.gate_kind == kGateElement)
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.dgate) + row * a.cols + col) =
            pack_bf16x8(dg);
    }
    const bool token = a.dgate && a.gate_kind == kGateToken;
    if (a.w_post || token) group_sum<2>(sum, lds2[turn]);
    if (token && threadIdx.x == 0) static_cast<float *>(a.dgate)[row] = sum[1];
    if (!a.dy) continue;
    const float c2 = sum[0] * a.inv_cols;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      if (a.w_post)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[v][i] = r_post * (d[v][i] - yh[v][i] * c2);
      *reinterpret_cast<u32x4 *>(a.dy + row * a.cols + col) = pack_bf16x8(d[v]);
    }
  }
  if constexpr (SUMS) {
    const int64_t plane = (int64_t)gridDim.x * a.cols;
    float *part = a.part + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      float *p = part + col;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (a.dw_pre) p[i] = s_pre[v][i];
        if (a.dw_post) p[plane + i] = s_post[v][i];
        if (a.dgate && a.gate_kind == kGateChannel) p[2 * plane + i] = s_gate[v][i];
      }
    }
  }
}

// One sum over the workgroups' rows, in workgroup order; 64 columns by 4 quarters
// of the workgroups.
__global__ __launch_bounds__(256) void block_norm_fold_kernel(const BlockNormBwdArgs a) {
  __shared__ float lds[4][64];
  float *out = blockIdx.y == 0 ? a.dw_pre : blockIdx.y == 1 ? a.dw_post
               : a.gate_kind == kGateChannel ? static_cast<float *>(a.dgate) : nullptr;
  if (!out) return;
  const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (col < a.cols) {
    const float *p = a.part + ((int64_t)blockIdx.y * a.groups) * a.cols + col;
    for (int g = quarter; g < a.groups; g += 4) sum += p[(int64_t)g * a.cols];
  }
  lds[quarter][lane] = sum;
  __syncthreads();
  if (quarter == 0 && col < a.cols) {
    sum = (lds[0][lane] + lds[1][lane]) + (lds[2][lane] + lds[3][lane]);
    out[col] = a.accumulate ? out[col] + sum : sum;
  }
}

// Threads of a row and pieces of 8 columns of a thread (1, 2 or 4).
void row_shape(int cols, int &threads, int &pieces) {
  const int need = (cols + 7) / 8;
  pieces = need <= kMaxThreads ? 1 : need <= 2 * kMaxThreads ? 2 : 4;
  threads = ((need + pieces - 1) / pieces + kWave - 1) / kWave * kWave;
}

template <int V, int CODE>
void launch_bwd(const BlockNormBwdArgs &a, int threads, hipStream_t s) {
  if (a.sums)
    hipLaunchKernelGGL((block_norm_bwd_kernel<V, CODE, true>), dim3(a.groups), dim3(threads), 0, s, a);
  else
    hipLaunchKernelGGL((block_norm_bwd_kernel<V, CODE, false>), dim3(a.groups), dim3(threads), 0, s, a);
}

template <int CODE>
void by_pieces(const BlockNormBwdArgs &a, hipStream_t s) {
  int threads, pieces;
  row_shape(a.cols, threads, pieces);
  if (pieces == 1) launch_bwd<1, CODE>(a, threads, s);
  else if (pieces == 2) launch_bwd<2, CODE>(a, threads, s);
  else launch_bwd<4, CODE>(a, threads, s);
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  int threads, pieces;
  row_shape(a.cols, threads, pieces);
  const dim3 grid((unsigned)a.rows), block(threads);
  if (pieces == 1) hipLaunchKernelGGL(block_norm_kernel<1>, grid, block, 0, s, a);
  else if (pieces == 2) hipLaunchKernelGGL(block_norm_kernel<2>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(block_norm_kernel<4>, grid, block, 0, s, a);
  return hipGetLastError();
}

// Workgroups of the backward kernel: with sums over rows each writes a row of them,
// so no more than fill the chip.
int block_norm_bwd_groups(int64_t rows, int64_t cols, int sums) {
  const int64_t most = sums ? 512 : int64_t(1) << 20;
  return (int)(rows < most ? rows : most);
}

hipError_t launch_block_norm_bwd(const BlockNormBwdArgs &a, hipStream_t s) {
  if (a.cols == 0) return hipSuccess;
  if (a.rows > 0) {
    const bool l = a.h.codes || a.y.codes;
    if (!l) by_pieces<-1>(a, s);
    else if (a.code == kCodeInt8) by_pieces<kCodeInt8>(a, s);
    else if (a.code == kCodeE4M3) by_pieces<kCodeE4M3>(a, s);
    else by_pieces<kCodeCast>(a, s);
  }
  if (a.sums)
    hipLaunchKernelGGL(block_norm_fold_kernel, dim3((a.cols + 63) / 64, 3), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hilore
