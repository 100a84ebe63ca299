// Norm and rotation of the heads of queries and keys, and their backward, on gfx950.
//   n = x rsqrt(mean(x^2) + eps) w,  out = R(position) n
//   dn = R^T g,  t = dn w,  dx = r (t - x r mean(t x r)),  dw = sum dn x r
//
// Bound by HBM: forward 4 B an element, backward 6 (an L unit's operand 1 + 4/block instead of 2).
//
// A wave takes a token, several heads at a time: a head lies in a group of G lanes, 16 columns a
// lane in two pieces of 16 bytes, so that both columns of a rotated pair meet in one lane (a piece
// of each half, or two neighbouring pieces), and a head's sums need only its group.  The token's
// cosines and sines are formed once, an angle a lane, and read from LDS by every group.
//
// 16384 tokens of 28 + 4 heads of 128, whole passes: forward 49.6 us, 5.4 TB/s (outputs kept in the caches 56.9);
// backward with the weights' gradients 89 us, 4.5 TB/s (75 of kernel, 5 of fold under a trace), where vector
// instructions take 44.  64 tokens forward 5.2 us, one launch's latencies.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kWaves = 4;  // of a workgroup, a token each

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sum over aligned groups of G lanes, all of them receiving it.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (G >= 2) v += dpp_f32<kDppQuadXor1>(v);
  if constexpr (G >= 4) v += dpp_f32<kDppQuadXor2>(v);
  if constexpr (G >= 8) v += dpp_f32<kDppRowHalfMirror>(v);
  if constexpr (G >= 16) v += dpp_f32<kDppRowMirror>(v);
  if constexpr (G >= 32) {
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  return v;
}

// A lane's 16 columns of a head: first columns of its two pieces, and whether they are rotated.
struct Place {
  int a, b, freq;
  bool live, turned;
};

__device__ __forceinline__ Place place(const HeadsArgs &h, int p) {
  Place at;
  at.live = 16 * p < h.dim;
  at.turned = 16 * p < h.rotated;
  at.freq = 8 * p;
  const bool halves = at.turned && !h.pairs;
  at.a = halves ? 8 * p : 16 * p;
  at.b = halves ? h.rotated / 2 + 8 * p : 16 * p + 8;
  return at;
}

// rsqrt(mean + eps), within 1 ulp of fp32 where the result is rounded to bf16.  The instruction takes a subnormal
// operand for 0, which only an eps below the normal numbers lets through: the IEEE operations then.
__device__ __forceinline__ float inverse_root(const HeadsArgs &h, float ss) {
  const float v = ss * h.inv_dim + h.eps;
  return h.eps >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(v) : 1.0f / sqrtf(v);
}

// The token's cosines and sines times rope_scale, to the wave's part of LDS (freq: first_freq).  The angle in turns is a
// product of two fp64 pairs (position * inv_freq and 1 / 2 pi with what their rounding leaves), so that
// positions up to 2^53 turn as exactly as near ones: the fraction is rounded once, to 2^-25 of a turn.
// first_freq: inv_freq[lane], read once by every wave (0 past its end).
__device__ __forceinline__ float first_freq(const HeadsArgs &h) {
  const int lane = threadIdx.x & 63;
  return lane < h.rotated / 2 ? h.inv_freq[lane] : 0.0f;
}

__device__ __forceinline__ void angles(const HeadsArgs &h, int64_t position, float freq, float *cs, float *sn) {
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;  // 1 / 2 pi
  const int half = h.rotated / 2, lane = threadIdx.x & 63;
  for (int i = lane; i < half; i += kWave) {
    const double p = (double)position, f = (double)(i < kWave ? freq : h.inv_freq[i]);
    const double a = p * f, a_rest = fma(p, f, -a);
    const double turns = a * kTurn, rest = fma(a, kTurn, -turns) + fma(a, kTurnRest, a_rest * kTurn);
    float s, c;
    sincospif(2.0f * (float)((turns - rint(turns)) + rest), &s, &c);
    cs[i] = c * h.rope_scale;
    sn[i] = s * h.rope_scale;
  }
  // the wave alone reads what it wrote, and its LDS operations are done in their order: a wider fence
  // would wait for the heads on their way
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct Angles {
  float c[8], s[8];
};

__device__ __forceinline__ Angles lane_angles(const float *cs, const float *sn, const Place &at) {
  Angles g;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    g.c[i] = at.turned ? cs[at.freq + i] : 1.0f;
    g.s[i] = at.turned ? sn[at.freq + i] : 0.0f;
  }
  return g;
}

// Two columns turned by an angle; BACK: by its negative.
template <bool BACK>
__device__ __forceinline__ void turn(float &a, float &b, float c, float s) {
  if constexpr (BACK) s = -s;
  const float x = a;
  a = fmaf(a, c, -(b * s));
  b = fmaf(b, c, x * s);
}

// x[0..7] and x[8..15]: a lane's pieces.
template <bool BACK>
__device__ __forceinline__ void rotate(float x[16], const Angles &g, bool pairs) {
  if (pairs) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<BACK>(x[2 * i], x[2 * i + 1], g.c[i], g.s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<BACK>(x[i], x[8 + i], g.c[i], g.s[i]);
  }
}

__device__ __forceinline__ u32x4 load16(const uint16_t *p) { return *reinterpret_cast<const u32x4 *>(p); }
__device__ __forceinline__ void store16(uint16_t *p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
}

__device__ __forceinline__ void unpack16(u32x4 a, u32x4 b, float x[16]) {
  unpack_bf16x8(a, x);
  unpack_bf16x8(b, x + 8);
}

// Heads are numbered through, the queries' first.
struct Weights {
  u32x4 q[2], k[2];
};

__device__ __forceinline__ void load_weights(Weights &w, const HeadsArgs &h, const Place &at) {
#pragma unroll
  for (int i = 0; i < 2; ++i) w.q[i] = w.k[i] = u32x4{};
  if (at.live && h.q.w) {
    w.q[0] = load16(h.q.w + at.a);
    w.q[1] = load16(h.q.w + at.b);
  }
  if (at.live && h.k.w) {
    w.k[0] = load16(h.k.w + at.a);
    w.k[1] = load16(h.k.w + at.b);
  }
}

constexpr int kForwardSteps = 4;  // heads a group has in flight

template <int G>
__global__ __launch_bounds__(kWaves *kWave) void heads_kernel(const HeadsArgs h, int parts) {
  __shared__ float cs[kWaves][kHeadMaxDim / 2], sn[kWaves][kHeadMaxDim / 2];
  constexpr int kSide = kWave / G;  // heads of a wave side by side
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int heads = h.heads_q + h.heads_k;
  const int steps = (heads + kSide - 1) / kSide, per = (steps + parts - 1) / parts;
  const Place at = place(h, lane % G);
  Weights w;
  load_weights(w, h, at);
  const float freq = first_freq(h);
  const int64_t units = h.tokens * parts;
  for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
    const int64_t token = unit / parts;
    const int part = (int)(unit - token * parts);
    const int first = part * per, last = min(first + per, steps);
    const int64_t position = h.positions ? h.positions[token] : token;
    Angles ang;
    for (int step = first; step < last; step += kForwardSteps) {
      u32x4 xa[kForwardSteps], xb[kForwardSteps];
#pragma unroll
      for (int i = 0; i < kForwardSteps; ++i) {
        const int head = (step + i) * kSide + lane / G;
        xa[i] = xb[i] = u32x4{};
        if (step + i >= last || head >= heads || !at.live) continue;
        const bool key = head >= h.heads_q;
        const uint16_t *x = key ? h.k.in.x + token * h.k.in.ld + (int64_t)(head - h.heads_q) * h.dim
                                : h.q.in.x + token * h.q.in.ld + (int64_t)head * h.dim;
        xa[i] = load16(x + at.a);
        xb[i] = load16(x + at.b);
      }
      if (step == first) {  // while the first heads are on their way
        if (position >= 0) angles(h, position, freq, cs[wave], sn[wave]);
        ang = lane_angles(cs[wave], sn[wave], at);
      }
#pragma unroll
      for (int i = 0; i < kForwardSteps; ++i) {
        const int head = (step + i) * kSide + lane / G;
        if (step + i >= last) break;
        const bool key = head >= h.heads_q;
        float x[16];
        unpack16(xa[i], xb[i], x);
        float ss = 0.0f;
#pragma unroll
        for (int c = 0; c < 16; ++c) ss = fmaf(x[c], x[c], ss);
        ss = group_sum<G>(ss);
        if (key ? h.k.w != nullptr : h.q.w != nullptr) {
          const float r = inverse_root(h, ss);
          float wv[16];
          unpack16(key ? w.k[0] : w.q[0], key ? w.k[1] : w.q[1], wv);
#pragma unroll
          for (int c = 0; c < 16; ++c) x[c] = x[c] * r * wv[c];
        }
        if (at.turned) rotate<false>(x, ang, h.pairs);
        if (head >= heads || !at.live) continue;
        uint16_t *o = key ? h.k.out + token * h.k.token_stride + (int64_t)(head - h.heads_q) * h.k.head_stride
                          : h.q.out + token * h.q.token_stride + (int64_t)head * h.q.head_stride;
        const bool pad = position < 0;
        store16(o + at.a, pad ? u32x4{} : pack_bf16x8(x));
        store16(o + at.b, pad ? u32x4{} : pack_bf16x8(x + 8));
      }
    }
  }
}

// --------------------------------------------------------------- backward --
// 8 columns of a saved head as packed bf16.  CODE: -1 bf16, else the code of an L unit.
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
__device__ __forceinline__ void load_saved(Saved8<CODE> &x, const SavedRows &s, int64_t token,
                                           int64_t cols, int64_t col, int block_log2) {
  if constexpr (CODE >= 0) {
    x.codes = *reinterpret_cast<const u32x2 *>(s.codes + token * cols + col);
    if constexpr (CODE != kCodeCast) x.scale = s.scales[token * (cols >> block_log2) + (col >> block_log2)];
  } else {
    x.w = load16(s.x + token * s.ld + col);
  }
}

template <int CODE>
__device__ __forceinline__ void saved_values(const Saved8<CODE> &x, float v[8]) {
  if constexpr (CODE >= 0) decode_codes8<CODE == kCodeInt8, CODE != kCodeCast>(x.codes, x.scale, v);
  else unpack_bf16x8(x.w, v);
}

// One side's saved operand may be bf16 where the other's is an L unit: Q and K are its codes.
template <int Q, int K>
struct SavedHead {
  Saved8<Q> qa, qb;
  Saved8<K> ka, kb;
};

// Heads that a group has in flight while it works on as many.  One, with the next one's loads ahead: 160 registers
// with sums, three waves a SIMD, 87 us; two 193 registers, 89 us (held to 168, spilled: 122); angles and weights read
// from LDS instead of held, 128 registers and four waves, 91 us; two without loads ahead 115 us.
constexpr int kBackwardSteps = 1;

// What the backward reads of some of a token's heads.
template <int Q, int K>
struct BackwardHeads {
  u32x4 ga[kBackwardSteps], gb[kBackwardSteps];
  SavedHead<Q, K> saved[kBackwardSteps];
};

template <int G, int Q, int K>
__device__ __forceinline__ void load_heads(BackwardHeads<Q, K> &x, const HeadsArgs &h, const Place &at, int64_t token, int step, int last) {
  constexpr int kSide = kWave / G;
  const int lane = threadIdx.x & 63, heads = h.heads_q + h.heads_k;
#pragma unroll
  for (int i = 0; i < kBackwardSteps; ++i) {
    const int head = (step + i) * kSide + lane / G;
    x.ga[i] = x.gb[i] = u32x4{};
    x.saved[i] = SavedHead<Q, K>{};
    if (step + i >= last || head >= heads || !at.live) continue;
    const bool key = head >= h.heads_q;
    const int j = key ? head - h.heads_q : head;
    const uint16_t *g = key ? h.k.g + token * h.k.token_stride + j * h.k.head_stride
                            : h.q.g + token * h.q.token_stride + j * h.q.head_stride;
    x.ga[i] = load16(g + at.a);
    x.gb[i] = load16(g + at.b);
    const int64_t col = (int64_t)j * h.dim;
    if constexpr (Q == K) {  // the sides differ in their addresses alone
      if (!(key ? h.k.w : h.q.w)) continue;
      const int64_t cols = (int64_t)(key ? h.heads_k : h.heads_q) * h.dim;
      const SavedRows in = {key ? h.k.in.x : h.q.in.x, key ? h.k.in.codes : h.q.in.codes, key ? h.k.in.scales : h.q.in.scales,
                            key ? h.k.in.ld : h.q.in.ld};
      load_saved<Q>(x.saved[i].qa, in, token, cols, col + at.a, h.block_log2);
      load_saved<Q>(x.saved[i].qb, in, token, cols, col + at.b, h.block_log2);
    } else if (key) {
      if (!h.k.w) continue;
      const int64_t cols = (int64_t)h.heads_k * h.dim;
      load_saved<K>(x.saved[i].ka, h.k.in, token, cols, col + at.a, h.block_log2);
      load_saved<K>(x.saved[i].kb, h.k.in, token, cols, col + at.b, h.block_log2);
    } else if (h.q.w) {
      const int64_t cols = (int64_t)h.heads_q * h.dim;
      load_saved<Q>(x.saved[i].qa, h.q.in, token, cols, col + at.a, h.block_log2);
      load_saved<Q>(x.saved[i].qb, h.q.in, token, cols, col + at.b, h.block_log2);
    }
  }
}

template <int G, int Q, int K, bool SUMS>
__global__ __launch_bounds__(kWaves *kWave, SUMS ? (Q == K ? 3 : 2) : 4) void heads_bwd_kernel(const HeadsArgs h, int parts) {
  __shared__ float cs[kWaves][kHeadMaxDim / 2], sn[kWaves][kHeadMaxDim / 2];
  constexpr int kSide = kWave / G;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int heads = h.heads_q + h.heads_k;
  const int steps = (heads + kSide - 1) / kSide, per = (steps + parts - 1) / parts;
  const Place at = place(h, lane % G);
  Weights w;
  load_weights(w, h, at);
  const float freq = first_freq(h);
  float sq[SUMS ? 16 : 1], sk[SUMS ? 16 : 1];
  if constexpr (SUMS)
#pragma unroll
    for (int c = 0; c < 16; ++c) sq[c] = sk[c] = 0.0f;
  const int64_t units = h.tokens * parts, stride = (int64_t)gridDim.x * kWaves;
  int64_t unit = (int64_t)blockIdx.x * kWaves + wave;
  BackwardHeads<Q, K> next;
  int64_t position = 0;
  if (unit < units) {
    const int64_t token = unit / parts;
    const int first = (int)(unit - token * parts) * per;
    position = h.positions ? h.positions[token] : token;
    load_heads<G, Q, K>(next, h, at, token, first, min(first + per, steps));
  }
  for (; unit < units; unit += stride) {
    const int64_t token = unit / parts;
    const int first = (int)(unit - token * parts) * per, last = min(first + per, steps);
    const bool pad = position < 0;
    if (!pad) angles(h, position, freq, cs[wave], sn[wave]);
    const Angles ang = lane_angles(cs[wave], sn[wave], at);
    // the next unit's first heads are loaded behind this one's last ones
    const int64_t unit2 = unit + stride < units ? unit + stride : unit, token2 = unit2 / parts;
    const int first2 = (int)(unit2 - token2 * parts) * per;
    position = h.positions ? h.positions[token2] : token2;
    for (int step = first; step < last; step += kBackwardSteps) {
      const BackwardHeads<Q, K> now = next;
      const bool more = step + kBackwardSteps < last;
      load_heads<G, Q, K>(next, h, at, more ? token : token2, more ? step + kBackwardSteps : first2, more ? last : min(first2 + per, steps));
#pragma unroll
      for (int i = 0; i < kBackwardSteps; ++i) {
        if (step + i >= last) break;
        const int head0 = (step + i) * kSide, head = head0 + lane / G;
        const bool key = head >= h.heads_q;
        float g[16];
        unpack16(now.ga[i], now.gb[i], g);
        if (at.turned) rotate<true>(g, ang, h.pairs);
        const bool inside = head < heads && at.live && !pad;
        if (key ? h.k.w != nullptr : h.q.w != nullptr) {
          float x[16], t[16];
          if (Q == K || !key) {
            saved_values<Q>(now.saved[i].qa, x);
            saved_values<Q>(now.saved[i].qb, x + 8);
          } else {
            saved_values<K>(now.saved[i].ka, x);
            saved_values<K>(now.saved[i].kb, x + 8);
          }
          unpack16(key ? w.k[0] : w.q[0], key ? w.k[1] : w.q[1], t);
          float ss = 0.0f, sx = 0.0f;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            t[c] = g[c] * t[c];
            ss = fmaf(x[c], x[c], ss);
            sx = fmaf(t[c], x[c], sx);
          }
          // a head's lanes are all of one side, so all of them are here
          ss = group_sum<G>(ss);
          sx = group_sum<G>(sx);
          const float r = inverse_root(h, ss);
          const float along = r * (sx * h.inv_dim);
#pragma unroll
          for (int c = 0; c < 16; ++c) x[c] *= r;
          if constexpr (SUMS)
            if (inside) {
              if (key)
#pragma unroll
                for (int c = 0; c < 16; ++c) sk[c] = fmaf(g[c], x[c], sk[c]);
              else
#pragma unroll
                for (int c = 0; c < 16; ++c) sq[c] = fmaf(g[c], x[c], sq[c]);
            }
#pragma unroll
          for (int c = 0; c < 16; ++c) g[c] = r * fmaf(-along, x[c], t[c]);
        }
        if (head >= heads || !at.live) continue;
        uint16_t *out = key ? h.k.out : h.q.out;
        if (!out) continue;
        out += token * (key ? h.k.ld_out : h.q.ld_out) + (int64_t)(key ? head - h.heads_q : head) * h.dim;
        store16(out + at.a, pad ? u32x4{} : pack_bf16x8(g));
        store16(out + at.b, pad ? u32x4{} : pack_bf16x8(g + 8));
      }
    }
  }
  if constexpr (SUMS) {
    // the workgroup's sums: groups of lanes and waves added in their order
    __shared__ float rows[kWaves * kWave][17];
    const auto put = [&](const float (&s)[SUMS ? 16 : 1], int plane) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < 16; ++c) rows[threadIdx.x][c] = s[c];
      __syncthreads();
      // column by (lane of the group, register)
      for (int i = threadIdx.x; i < G * 16; i += kWaves * kWave) {
        const int p = i / 16, c = i % 16;
        if (16 * p >= h.dim) continue;
        float sum = 0.0f;
        for (int r = p; r < kWaves * kWave; r += G) sum += rows[r][c];
        const Place o = place(h, p);
        h.part[((int64_t)plane * gridDim.x + blockIdx.x) * h.dim + (c < 8 ? o.a + c : o.b + c - 8)] = sum;
      }
    };
    if (h.q.dw) put(sq, 0);
    if (h.k.dw) put(sk, 1);
  }
}

// One sum over the workgroups' rows, in a fixed order: 64 columns a workgroup, its waves take
// every 16th row each.  One gradient for both sides (one weight) is the sum over the queries' rows and the keys' behind
// them, by the queries' workgroups: two that add to the same place would lose a side.
constexpr int kFoldWaves = 16;

__global__ __launch_bounds__(kFoldWaves *kWave) void heads_fold_kernel(const HeadsArgs h) {
  __shared__ float lds[kFoldWaves][kWave];
  float *out = blockIdx.y == 0 ? h.q.dw : h.k.dw;
  const bool shared = h.q.dw == h.k.dw;
  if (!out || (shared && blockIdx.y != 0)) return;
  const int groups = shared ? 2 * h.groups : h.groups;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * kWave + lane;
  float sum = 0.0f;
  if (col < h.dim) {
    const float *p = h.part + ((int64_t)blockIdx.y * h.groups) * h.dim + col;
#pragma unroll 16
    for (int g = wave; g < groups; g += kFoldWaves) sum += p[(int64_t)g * h.dim];
  }
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && col < h.dim) {
    for (int w = 1; w < kFoldWaves; ++w) sum += lds[w][lane];
    out[col] = h.accumulate ? out[col] + sum : sum;
  }
}

int lanes_of(int dim) {
  int g = 1;
  while (16 * g < dim) g *= 2;
  return g;
}

// Waves that share a token's heads: more than one until 4096 waves are at work.  28 + 4 heads of 128, us with one
// wave a token and with several: 64 tokens 6.0 and 5.1, 512 6.3 and 5.0, 2048 7.1 and 6.6, 4096 11.0 (16 waves a
// token 15.0); backward 64 tokens 12.4 and 9.9, 512 14.9 and 12.0.  None of them is without a head: the backward loads
// the next unit's first heads behind a unit's last ones.
int parts_of(int64_t tokens, int heads, int dim) {
  const int side = kWave / lanes_of(dim);
  const int steps = (heads + side - 1) / side;
  int parts = 1;
  while (parts < steps && tokens * parts < 4096) parts *= 2;
  const int per = (steps + parts - 1) / parts;  // of a wave
  return (steps + per - 1) / per;
}

template <int G>
void forward(const HeadsArgs &h, hipStream_t s) {
  const int parts = parts_of(h.tokens, h.heads_q + h.heads_k, h.dim);
  const int64_t units = h.tokens * parts;
  const int64_t need = (units + kWaves - 1) / kWaves;
  // a launch's work-items are counted in 32 bits
  const unsigned grid = (unsigned)(need < (1 << 22) ? need : (1 << 22));
  hipLaunchKernelGGL((heads_kernel<G>), dim3(grid), dim3(kWaves * kWave), 0, s, h, parts);
}

template <int G, int Q, int K>
void backward(const HeadsArgs &h, hipStream_t s) {
  const int parts = parts_of(h.tokens, h.heads_q + h.heads_k, h.dim);
  const dim3 grid(h.groups), block(kWaves * kWave);
  if (h.q.dw || h.k.dw) hipLaunchKernelGGL((heads_bwd_kernel<G, Q, K, true>), grid, block, 0, s, h, parts);
  else hipLaunchKernelGGL((heads_bwd_kernel<G, Q, K, false>), grid, block, 0, s, h, parts);
}

// A side that is not read counts as an L unit like the other.
template <int G, int CODE>
void by_units(const HeadsArgs &h, hipStream_t s) {
  const bool q = h.q.in.codes || !h.q.in.x, k = h.k.in.codes || !h.k.in.x;
  if (q && k) backward<G, CODE, CODE>(h, s);
  else if (q) backward<G, CODE, -1>(h, s);
  else backward<G, -1, CODE>(h, s);
}

template <int G>
void by_code(const HeadsArgs &h, hipStream_t s) {
  if (!h.q.in.codes && !h.k.in.codes) backward<G, -1, -1>(h, s);
  else if (h.code == kCodeInt8) by_units<G, kCodeInt8>(h, s);
  else if (h.code == kCodeE4M3) by_units<G, kCodeE4M3>(h, s);
  else by_units<G, kCodeCast>(h, s);
}

}  // namespace

hipError_t launch_heads(const HeadsArgs &h, hipStream_t s) {
  if (h.tokens == 0 || h.heads_q + h.heads_k == 0) return hipSuccess;
  switch (lanes_of(h.dim)) {
    case 1: forward<1>(h, s); break;
    case 2: forward<2>(h, s); break;
    case 4: forward<4>(h, s); break;
    case 8: forward<8>(h, s); break;
    case 16: forward<16>(h, s); break;
    default: forward<32>(h, s); break;
  }
  return hipGetLastError();
}

// Workgroups of the backward: as many as stay on the chip (three or, without sums, four waves a SIMD).  11987 x 16
// heads of 64 without sums: 1024 14.9 us, 768 16.6, 2048 16.2, one to every four tokens 17.9.
int heads_bwd_groups(int64_t tokens, int heads, int dim, int sums) {
  if (tokens == 0 || heads == 0) return 0;
  const int64_t need = (tokens * parts_of(tokens, heads, dim) + kWaves - 1) / kWaves;
  const int most = sums ? 768 : 1024;
  return (int)(need < most ? need : most);
}

hipError_t launch_heads_bwd(const HeadsArgs &h, hipStream_t s) {
  if (h.groups == 0 && !h.q.dw && !h.k.dw) return hipSuccess;
  if (h.groups > 0) switch (lanes_of(h.dim)) {
      case 1: by_code<1>(h, s); break;
      case 2: by_code<2>(h, s); break;
      case 4: by_code<4>(h, s); break;
      case 8: by_code<8>(h, s); break;
      case 16: by_code<16>(h, s); break;
      default: by_code<32>(h, s); break;
    }
  if (h.q.dw || h.k.dw)
    hipLaunchKernelGGL(heads_fold_kernel, dim3((h.dim + kWave - 1) / kWave, 2), dim3(kFoldWaves * kWave), 0, s, h);
  return hipGetLastError();
}

}  // namespace hilore
