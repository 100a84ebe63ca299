// RMS norms on leaving a block and entering the next, fused with the block's gate
// and residual scale, and their backward, on gfx950.  N(v) = v rsqrt(mean(v^2) + eps):
//   h = bf16(res + scale * gate * (N(y) * w_post)),   n = N(h) * w_pre
// n is the norm of h as stored, so it can be recomputed from a kept h.
//
// Bound by HBM: forward reads res and y and writes h and n, 8 B an element (7 with
// int8 codes for n); backward reads h, y, dn and dh and writes dres and dy, 12 B
// (an L unit's operand 1 + 4/block B).
//
// A workgroup takes a row at a time in registers: every thread holds up to V pieces of 8
// columns, `threads` pieces apart, so that each load is 16 bytes a lane and contiguous over
// the wave.  Workgroups stay for many rows; up to 8192 columns they keep the weights in
// registers and load the next row before they work on this one, so that neither the loads'
// latency nor the barriers of the row sums leave the memory idle.  16384 x 3584, whole passes in
// a row: forward 101 us, 4.7 TB/s, the rate of a large copy; backward with all gradients, its fold
// included, 152 us, 4.6 TB/s (under a kernel trace 162 to 177 and 5).  Longer rows are loaded when their
// turn comes: 4096 x 14336 forward 126 us, 3.7 TB/s, backward 212 us, 3.3 TB/s.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kMaxWaves = kMaxThreads / kWave;
constexpr int kForwardWaves = 28;  // of a CU

typedef float f32x4 __attribute__((ext_vector_type(4)));

enum Gate : int { kGateNone = 0, kGateChannel = 1, kGateToken = 2, kGateElement = 3 };

// N sums over the threads of a row (blockDim.x of them; blockDim.y rows side by side), in a
// fixed order; all of them receive them.  One barrier: `lds` must not be the place of the sums
// before.
template <int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*lds)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lanes_sum(v[k]);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return;
  lds += __builtin_amdgcn_readfirstlane(threadIdx.y) * waves;
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

constexpr uint32_t kOnes = 0x3F803F80u;  // two bf16 ones

// Outputs go past the caches, which the next row's operands need (16384 x 896: 27.0 -> 21.9 us;
// not measured for a few rows, whose reader would find them there).
__device__ __forceinline__ void store16(uint16_t *p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
}

// A row-independent vector, ones where there is none: its pieces kept packed where HOLD, else
// loaded when asked.
template <int V, bool HOLD>
struct Vector {
  const uint16_t *p;
  u32x4 held[HOLD ? V : 1];
  __device__ __forceinline__ u32x4 load(int col) const {
    return p ? load16(p + col) : u32x4{kOnes, kOnes, kOnes, kOnes};
  }
  __device__ __forceinline__ void init(const uint16_t *ptr, int cols, int threads) {
    p = ptr;
    if constexpr (HOLD)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * threads + (int)threadIdx.x) * 8;
        held[v] = col < cols ? load(col) : u32x4{};
      }
  }
  __device__ __forceinline__ u32x4 raw(int v, int col) const { return HOLD ? held[v] : load(col); }
  __device__ __forceinline__ void get(int v, int col, float w[8]) const {
    unpack_bf16x8(raw(v, col), w);
  }
};

// The gate's 8 values at a piece: a channel's (ones without a gate) or an element's, packed,
// times a token's.
__device__ __forceinline__ void gate_values(u32x4 packed, float token, float g[8]) {
  unpack_bf16x8(packed, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] *= token;
}

__device__ __forceinline__ float token_gate(const uint16_t *gate, int kind, int64_t row) {
  return kind == kGateToken ? __uint_as_float((uint32_t)gate[row] << 16) : 1.0f;
}

// What the forward reads of one row.
template <int V>
struct ForwardRow {
  u32x4 res[V], y[V], gate[V];
  float token;
};

template <int V>
__device__ __forceinline__ void load_row(ForwardRow<V> &x, const BlockNormArgs &a, int64_t row) {
  const int threads = blockDim.x;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * threads + (int)threadIdx.x) * 8;
    if (col >= a.cols) continue;
    x.res[v] = load16(a.res + row * a.ld_res + col);
    if (a.y) x.y[v] = load16(a.y + row * a.ld_y + col);
    if (a.gate_kind == kGateElement) x.gate[v] = load16(a.gate + row * a.cols + col);
  }
  x.token = token_gate(a.gate, a.gate_kind, row);
}

template <int V, bool HOLD>
__global__ __launch_bounds__(kMaxThreads) void block_norm_kernel(const BlockNormArgs a) {
  __shared__ float lds[2][2][kMaxWaves][1];
  __shared__ uint32_t lds_max[2][kMaxWaves];
  const int threads = blockDim.x;
  Vector<V, HOLD> w_post, w_pre, gate;
  w_post.init(a.w_post, a.cols, threads);
  w_pre.init(a.w_pre, a.cols, threads);
  gate.init(a.gate_kind == kGateChannel ? a.gate : nullptr, a.cols, threads);
  ForwardRow<V> next;
  if constexpr (HOLD) load_row(next, a, blockIdx.x);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    if constexpr (!HOLD) load_row(next, a, row);
    const ForwardRow<V> x = next;
    if constexpr (HOLD)
      if (row + gridDim.x < a.rows) load_row(next, a, row + gridDim.x);
    float h[V][8];
    float sum[1];
    // y and its norm
    float r_post = 1.0f;
    if (a.y) {
      sum[0] = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * threads + (int)threadIdx.x) * 8;
        if (col >= a.cols) continue;
        unpack_bf16x8(x.y[v], h[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = fmaf(h[v][i], h[v][i], sum[0]);
      }
      if (a.w_post) {
        row_sum<1>(sum, lds[turn][0]);
        r_post = 1.0f / sqrtf(sum[0] * a.inv_cols + a.eps);
        if (a.rstd_post && threadIdx.x == 0) a.rstd_post[row] = r_post;
      }
    }
    // h, rounded as it is stored
    sum[0] = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      u32x4 stored = x.res[v];
      if (a.y) {
        float res[8], g[8];
        unpack_bf16x8(stored, res);
        if (a.w_post) {
          float w[8];
          w_post.get(v, col, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r_post * w[i];
        }
        gate_values(a.gate_kind == kGateElement ? x.gate[v] : gate.raw(v, col), x.token, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) res[i] += a.scale * (h[v][i] * g[i]);
        stored = pack_bf16x8(res);
      }
      if (a.h) store16(a.h + row * a.cols + col, stored);
      unpack_bf16x8(stored, h[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[0] = fmaf(h[v][i], h[v][i], sum[0]);
    }
    if (!a.w_pre) continue;
    row_sum<1>(sum, lds[turn][1]);
    const float r_pre = 1.0f / sqrtf(sum[0] * a.inv_cols + a.eps);
    if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[row] = r_pre;
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols) continue;
      float w[8];
      w_pre.get(v, col, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] = h[v][i] * r_pre * w[i];
        top = max(top, __float_as_uint(fabsf(h[v][i])));
      }
      if (a.n) store16(a.n + row * a.cols + col, pack_bf16x8(h[v]));
    }
    if (!a.codes) continue;
    top = lanes_max_u32<64>(top);
    const int waves = threads >> 6;
    if (waves > 1) {
      if ((threadIdx.x & 63) == 0) lds_max[turn][threadIdx.x >> 6] = top;
      __syncthreads();
      top = lds_max[turn][0];
      for (int w = 1; w < waves; ++w) top = max(top, lds_max[turn][w]);
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
}

// --------------------------------------------------------------- backward --
// 8 values of a saved tensor as they lie in memory.  CODE: -1 bf16, else the code of the L unit.
template <int CODE>
struct Saved8 {
  u32x2 codes;
  float scale;
};
template <>
struct Saved8<-1> {
  u32x4 w;
};

template <int CODE>
__device__ __forceinline__ void load_saved(Saved8<CODE> &x, const SavedRows &s, int64_t row,
                                           int col, int cols, int block_log2) {
  if constexpr (CODE >= 0) {
    x.codes = *reinterpret_cast<const u32x2 *>(s.codes + row * cols + col);
    if constexpr (CODE != kCodeCast)
      x.scale = s.scales[row * (cols >> block_log2) + (col >> block_log2)];
  } else {
    x.w = load16(s.x + row * s.ld + col);
  }
}

// As packed bf16, which holds a decoded value exactly.
template <int CODE>
__device__ __forceinline__ u32x4 packed(const Saved8<CODE> &x) {
  if constexpr (CODE >= 0) {
    float v[8];
    decode_codes8<CODE == kCodeInt8, CODE != kCodeCast>(x.codes, x.scale, v);
    return pack_bf16x8(v);
  } else {
    return x.w;
  }
}

// What the backward reads of one row.  H, Y: the codes of the saved tensors.
template <int V, int H, int Y>
struct BackwardRow {
  Saved8<H> h[V];
  Saved8<Y> y[V];
  u32x4 dn[V], dh[V];
  float r_pre, r_post, token;
};

// What is not there is zeros, so that the row's work has no branches.
template <int V, int H, int Y>
__device__ __forceinline__ void load_row(BackwardRow<V, H, Y> &x, const BlockNormBwdArgs &a, bool y,
                                         int64_t row) {
  const int threads = blockDim.x;
  const bool live = row < a.rows;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * threads + (int)threadIdx.x) * 8;
    x.dn[v] = x.dh[v] = u32x4{};
    x.h[v] = Saved8<H>{};
    x.y[v] = Saved8<Y>{};
    if (col >= a.cols || !live) continue;
    if (a.dn) {
      x.dn[v] = load16(a.dn + row * a.ld_dn + col);
      load_saved(x.h[v], a.h, row, col, a.cols, a.block_log2);
    }
    if (a.dh) x.dh[v] = load16(a.dh + row * a.cols + col);
    if (y) load_saved(x.y[v], a.y, row, col, a.cols, a.block_log2);
  }
  x.r_pre = a.dn && live ? a.rstd_pre[row] : 0.0f;
  x.r_post = a.w_post && live ? a.rstd_post[row] : 1.0f;
  x.token = live ? token_gate(a.gate, a.gate_kind, row) : 1.0f;
}

// Two neighbouring columns of a row: d = dh + r_pre t with t = dn w_pre.
struct Pair {
  f32x2 dn, t, hh, d, yh, w, g;
};

__device__ __forceinline__ f32x2 bf16_pair(uint32_t w) { return f32x2{bf16_lo(w), bf16_hi(w)}; }

// With t = dn w_pre, c = mean(t hh): D = dh + r_pre (t - hh c).  The sums that need D are
// linear in it, so they are taken with dh + r_pre t and with hh, and one reduction gives all:
//   sum(q D) = sum(q (dh + r_pre t)) - r_pre c sum(q hh),   q = z (a token's dgate) or
//   q = scale gate w_post yh (the norm of y).
// SUMS: this workgroup's sums over its rows of dn hh, dz yh and a channel's dgate are kept in
// registers and written to the workspace at the end.
// One piece a thread: at most 128 registers, so that two workgroups share a CU.
template <int V, int H, int Y, bool HOLD, bool SUMS>
__global__ __launch_bounds__(kMaxThreads, V == 1 ? 4 : 2) void block_norm_bwd_kernel(
    const BlockNormBwdArgs a) {
  __shared__ float lds[2][kMaxWaves][5];
  const int threads = blockDim.x;
  Vector<V, HOLD> w_post, w_pre, gate;
  w_post.init(a.w_post, a.cols, threads);
  w_pre.init(a.w_pre, a.cols, threads);
  gate.init(a.gate_kind == kGateChannel ? a.gate : nullptr, a.cols, threads);
  float s_pre[SUMS ? V : 1][8], s_post[SUMS ? V : 1][8], s_gate[SUMS ? V : 1][8];
  if constexpr (SUMS)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s_pre[v][i] = s_post[v][i] = s_gate[v][i] = 0.0f;
  const bool need_y = a.y.x || a.y.codes;
  const bool token = a.dgate && a.gate_kind == kGateToken;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const int side = __builtin_amdgcn_readfirstlane(threadIdx.y);  // a row's threads are whole waves
  int64_t row = (int64_t)blockIdx.x * blockDim.y + side;
  BackwardRow<V, H, Y> next;
  if constexpr (HOLD) load_row(next, a, need_y, row);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.rows;
       first += step, row += step, turn ^= 1) {
    if constexpr (!HOLD) load_row(next, a, need_y, row);
    // the row stays packed; its values are formed twice, before and after the row sums, rather
    // than kept (24 registers a piece)
    u32x4 h[V], y[V], dn[V], dh[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      h[v] = packed(next.h[v]);
      y[v] = packed(next.y[v]);
      dn[v] = next.dn[v];
      dh[v] = next.dh[v];
    }
    const float r_pre = next.r_pre, r_post = next.r_post, gate_token = next.token;
    if constexpr (HOLD) load_row(next, a, need_y, row + step);
    const bool live = row < a.rows;
    const auto gate_of = [&](int v, int col) {
      return a.gate_kind == kGateElement ? load16(a.gate + row * a.cols + col) : gate.raw(v, col);
    };
    const auto pair = [&](int v, int k, uint32_t wp, uint32_t wq, uint32_t g) {
      Pair p;
      p.dn = bf16_pair(dn[v][k]);
      p.t = p.dn * bf16_pair(wp);
      p.hh = bf16_pair(h[v][k]) * r_pre;
      p.d = f32x2{fmaf(r_pre, p.t.x, bf16_lo(dh[v][k])), fmaf(r_pre, p.t.y, bf16_hi(dh[v][k]))};
      p.yh = bf16_pair(y[v][k]) * r_post;
      p.w = bf16_pair(wq);
      p.g = bf16_pair(g) * gate_token;
      return p;
    };
    float sum[5] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f};  // t hh; of q = ..yh: q d, q hh; of z: z d, z hh
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols || !live) continue;
      const u32x4 wp = w_pre.raw(v, col), wq = w_post.raw(v, col), g = gate_of(v, col);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Pair p = pair(v, k, wp[k], wq[k], g[k]);
        if constexpr (SUMS) {
          s_pre[v][2 * k] = fmaf(p.dn.x, p.hh.x, s_pre[v][2 * k]);
          s_pre[v][2 * k + 1] = fmaf(p.dn.y, p.hh.y, s_pre[v][2 * k + 1]);
        }
        sum[0] = fmaf(p.t.y, p.hh.y, fmaf(p.t.x, p.hh.x, sum[0]));
        const f32x2 z = p.yh * p.w, q = z * p.g;
        sum[1] = fmaf(q.y, p.d.y, fmaf(q.x, p.d.x, sum[1]));
        sum[2] = fmaf(q.y, p.hh.y, fmaf(q.x, p.hh.x, sum[2]));
        if (token) {
          sum[3] = fmaf(z.y, p.d.y, fmaf(z.x, p.d.x, sum[3]));
          sum[4] = fmaf(z.y, p.hh.y, fmaf(z.x, p.hh.x, sum[4]));
        }
      }
    }
    if (token) {
      row_sum<5>(sum, lds[turn]);
    } else if (a.dn || a.w_post) {
      float three[3] = {sum[0], sum[1], sum[2]};
      row_sum<3>(three, reinterpret_cast<float(*)[3]>(lds[turn]));
      sum[0] = three[0];
      sum[1] = three[1];
      sum[2] = three[2];
    }
    const float rc = r_pre * (sum[0] * a.inv_cols);
    const float c2 = a.w_post ? a.scale * (sum[1] - rc * sum[2]) * a.inv_cols : 0.0f;
    if (token && threadIdx.x == 0 && live)
      static_cast<float *>(a.dgate)[row] = a.scale * (sum[3] - rc * sum[4]);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * threads + (int)threadIdx.x) * 8;
      if (col >= a.cols || !live) continue;
      // the compiler would keep the values of the first time
      if constexpr (HOLD) asm volatile("" : "+v"(h[v]), "+v"(dn[v]), "+v"(dh[v]), "+v"(y[v]));
      const u32x4 wp = w_pre.raw(v, col), wq = w_post.raw(v, col), g = gate_of(v, col);
      u32x4 dres, dgate, dy;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Pair p = pair(v, k, wp[k], wq[k], g[k]);
        f32x2 d = {fmaf(-rc, p.hh.x, p.d.x), fmaf(-rc, p.hh.y, p.d.y)};
        dres[k] = pack_bf16(d.x, d.y);
        d *= a.scale;
        const f32x2 dg = d * (p.yh * p.w);
        dgate[k] = pack_bf16(dg.x, dg.y);
        d *= p.g;
        if constexpr (SUMS) {
          s_gate[v][2 * k] += dg.x;
          s_gate[v][2 * k + 1] += dg.y;
          s_post[v][2 * k] = fmaf(d.x, p.yh.x, s_post[v][2 * k]);
          s_post[v][2 * k + 1] = fmaf(d.y, p.yh.y, s_post[v][2 * k + 1]);
        }
        d *= p.w;
        // not with c2 = 0: a y that is not finite would reach the gradient of a block without norm
        if (a.w_post) d = f32x2{fmaf(-c2, p.yh.x, d.x), fmaf(-c2, p.yh.y, d.y)};
        dy[k] = pack_bf16(r_post * d.x, r_post * d.y);
      }
      const int64_t at = row * a.cols + col;
      if (a.dres) store16(a.dres + at, dres);
      if (a.dgate && a.gate_kind == kGateElement) store16(static_cast<uint16_t *>(a.dgate) + at, dgate);
      if (a.dy) store16(a.dy + at, dy);
    }
  }
  if constexpr (SUMS) {
    // the rows side by side, added in their order; then one row of sums to the workspace
    __shared__ f32x4 rows[V == 1 ? kMaxThreads : 1][2];
    const auto put = [&](const float (&s)[SUMS ? V : 1][8], int64_t plane) {
      float *part = a.part + (plane * gridDim.x + blockIdx.x) * a.cols;
      if constexpr (V == 1) {
        const int at = side * threads + (int)threadIdx.x;
        __syncthreads();
        rows[at][0] = f32x4{s[0][0], s[0][1], s[0][2], s[0][3]};
        rows[at][1] = f32x4{s[0][4], s[0][5], s[0][6], s[0][7]};
        __syncthreads();
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * threads + (int)threadIdx.x) * 8;
        if (col >= a.cols || side != 0) continue;
        f32x4 lo = {s[v][0], s[v][1], s[v][2], s[v][3]}, hi = {s[v][4], s[v][5], s[v][6], s[v][7]};
        if constexpr (V == 1)
          for (int r = 1; r < (int)blockDim.y; ++r) {
            lo += rows[r * threads + threadIdx.x][0];
            hi += rows[r * threads + threadIdx.x][1];
          }
        f32x4 *o = reinterpret_cast<f32x4 *>(part + col);
        o[0] = lo;
        o[1] = hi;
      }
    };
    if (a.dw_pre) put(s_pre, 0);
    if (a.dw_post) put(s_post, 1);
    if (a.dgate && a.gate_kind == kGateChannel) put(s_gate, 2);
  }
}

// One sum over the workgroups' rows, in a fixed order: 64 columns a workgroup, its waves take
// every 16th workgroup's row each.
constexpr int kFoldWaves = 16;

__global__ __launch_bounds__(kFoldWaves *kWave) void block_norm_fold_kernel(
    const BlockNormBwdArgs a) {
  __shared__ float lds[kFoldWaves][kWave];
  float *out = blockIdx.y == 0 ? a.dw_pre : blockIdx.y == 1 ? a.dw_post
               : a.gate_kind == kGateChannel ? static_cast<float *>(a.dgate) : nullptr;
  if (!out) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * kWave + lane;
  float sum = 0.0f;
  if (col < a.cols) {
    const float *p = a.part + ((int64_t)blockIdx.y * a.groups) * a.cols + col;
#pragma unroll 8
    for (int g = wave; g < a.groups; g += kFoldWaves) sum += p[(int64_t)g * a.cols];
  }
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < a.cols) {
    for (int w = 1; w < kFoldWaves; ++w) sum += lds[w][lane];
    out[col] = a.accumulate ? out[col] + sum : sum;
  }
}

// Threads of a row and pieces of 8 columns of a thread (1, 2 or 4).
void row_shape(int64_t cols, int &threads, int &pieces) {
  const int need = (int)(cols + 7) / 8;
  pieces = need <= kMaxThreads ? 1 : need <= 2 * kMaxThreads ? 2 : 4;
  threads = ((need + pieces - 1) / pieces + kWave - 1) / kWave * kWave;
}

// Workgroups that fill the chip with `waves` waves to a CU, `side` rows each at a time.
int row_groups(int64_t rows, int threads, int side, int waves) {
  const int per_cu = waves * kWave / (threads * side);
  const int64_t most = (int64_t)256 * (per_cu > 1 ? per_cu : 1), need = (rows + side - 1) / side;
  return (int)(need < most ? need : most);
}

// Rows that a backward workgroup takes side by side: as many as 512 threads hold.
int side_rows(int threads) { return kMaxThreads / threads; }

template <int V, int H, int Y>
void launch_bwd(const BlockNormBwdArgs &a, int threads, hipStream_t s) {
  constexpr bool kHold = V <= 2;
  const dim3 block(threads, side_rows(threads));
  if (a.sums)
    hipLaunchKernelGGL((block_norm_bwd_kernel<V, H, Y, kHold, true>), dim3(a.groups), block, 0, s, a);
  else
    hipLaunchKernelGGL((block_norm_bwd_kernel<V, H, Y, kHold, false>), dim3(a.groups), block, 0, s, a);
}

template <int H, int Y>
void by_pieces(const BlockNormBwdArgs &a, hipStream_t s) {
  int threads, pieces;
  row_shape(a.cols, threads, pieces);
  if (pieces == 1) launch_bwd<1, H, Y>(a, threads, s);
  else if (pieces == 2) launch_bwd<2, H, Y>(a, threads, s);
  else launch_bwd<4, H, Y>(a, threads, s);
}

// A saved tensor that is not read counts as an L unit like the other.
template <int CODE>
void by_units(const BlockNormBwdArgs &a, hipStream_t s) {
  const bool h = a.h.codes || !a.h.x, y = a.y.codes || !a.y.x;
  if (h && y) by_pieces<CODE, CODE>(a, s);
  else if (h) by_pieces<CODE, -1>(a, s);
  else by_pieces<-1, CODE>(a, s);
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  int threads, pieces;
  row_shape(a.cols, threads, pieces);
  const dim3 grid(row_groups(a.rows, threads, 1, kForwardWaves)), block(threads);
  if (pieces == 1) hipLaunchKernelGGL((block_norm_kernel<1, true>), grid, block, 0, s, a);
  else if (pieces == 2) hipLaunchKernelGGL((block_norm_kernel<2, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((block_norm_kernel<4, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

// Workgroups of the backward kernel.  With sums over rows each writes a row of them and the fold
// reads it, 24 B a column at some 4 TB/s; a turn of a workgroup takes about 1.5 us and 1 us more
// every 2200 columns.  So turns / groups + groups * row is least at the root below (with
// four turns for each workgroup 10 x 16128 took 37 us, now 16; 97 x 10112 37 and 19, 123 x 288 13.6 and
// 8.1; 512 x 3584 18 and 15, and in 512 workgroups 25).
int block_norm_bwd_groups(int64_t rows, int64_t cols, int sums) {
  if (cols == 0 || rows == 0) return 0;
  int threads, pieces;
  row_shape(cols, threads, pieces);
  const int side = side_rows(threads);
  const int full = row_groups(rows, threads, side, pieces == 1 ? 2 * kMaxWaves : kMaxWaves);
  if (!sums) return full;
  const double turns = (double)rows / side * (1.5 + (double)cols / 2200), row = (double)cols * 24 / 4e6;
  const double best = __builtin_sqrt(turns / row);
  return best < full ? (best < 1.0 ? 1 : (int)best) : full;
}

hipError_t launch_block_norm_bwd(const BlockNormBwdArgs &a, hipStream_t s) {
  if (a.cols == 0 || (a.rows == 0 && !a.sums)) return hipSuccess;
  if (a.rows > 0) {
    const bool l = a.h.codes || a.y.codes;
    if (!l) by_pieces<-1, -1>(a, s);
    else if (a.code == kCodeInt8) by_units<kCodeInt8>(a, s);
    else if (a.code == kCodeE4M3) by_units<kCodeE4M3>(a, s);
    else by_units<kCodeCast>(a, s);
  }
  if (a.sums)
    hipLaunchKernelGGL(block_norm_fold_kernel, dim3((a.cols + kWave - 1) / kWave, 3),
                       dim3(kFoldWaves * kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace hilore
