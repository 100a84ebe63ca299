// Log-probabilities of chosen tokens from logits, and their backward, on gfx950.
//   m = max z,  S = sum exp(scale (z - m)),  logp = scale (z_t - m) - log S,
//   entropy = log S - sum p scale (z - m)
//   dz_j = scale (dlogp (1[j = t] - p_j) - dentropy p_j (l_j + entropy)),  l = scale (z - m) - log S
//
// Bound by HBM: forward reads the logits once, backward reads them once more (but for rows
// without a gradient) and writes as much.
//
// Forward: one pass with the running maximum and sums of a softmax.  A row is cut into segments of
// kSegment pieces of 16 bytes; a wave reduces its part of a segment over its lanes and joins the
// segments in order, then the waves are joined in order.  Where there are few rows a workgroup takes one segment and a
// second kernel joins them in that same order, or a larger workgroup takes four segments at a time, so that a row gives
// the same bits however many rows the call has.
//
// Whole passes, bf16: 8192 x 131072 with entropy 322 to 332 us, 6.5 TB/s (loads kept in the caches 363), of which vector
// instructions take 290, 9.4 a logit; one such row 9 us, two launches; backward with 30 % of the rows without a gradient
// 600 us, 6.1 TB/s.  997 x 50021 f32 backward 67 us, 5.4 TB/s.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kBatch = 4;                              // pieces of a lane in flight
constexpr int kBatches = 2;                            // of a lane in a segment (8192 rows: 1 351 us, 2 331, 4 330; one row 8.7, 9.2, 9.0)
constexpr int kSegment = kThreads * kBatch * kBatches; // pieces

constexpr float kLowest = -3.402823466e38f;  // below every logit: exp2 of the way to it is 0
constexpr float kNoWay = -200.0f;            // exp2 of it is 0 in fp32, and its products are finite
constexpr float kLn2 = 0.6931471805599453f;

// Rows may begin at any element: 16-byte loads and stores of that alignment.
typedef u32x4 __attribute__((aligned(2))) u32x4_bf16;
typedef u32x4 __attribute__((aligned(4))) u32x4_f32;

// The row's address is the same in all lanes and a piece's place in it fits 32 bits (vocab < 2^28).
template <bool F32>
__device__ __forceinline__ u32x4 load_piece(const void *row, int piece) {
  const char *p = static_cast<const char *>(row) + (uint32_t)piece * 16u;
  if constexpr (F32) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_f32 *>(p));
  else return __builtin_nontemporal_load(reinterpret_cast<const u32x4_bf16 *>(p));
}

template <bool F32>
__device__ __forceinline__ float load_one(const void *row, int64_t i) {
  if constexpr (F32) return static_cast<const float *>(row)[i];
  else return __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
}

template <bool F32>
constexpr int kPiece = F32 ? 4 : 8;  // elements of a piece

template <bool F32>
__device__ __forceinline__ void values(u32x4 w, float v[kPiece<F32>]) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  } else {
    unpack_bf16x8(w, v);
  }
}

template <bool F32>
__device__ __forceinline__ u32x4 piece_of(float x) {
  const uint32_t w = F32 ? __float_as_uint(x) : pack_bf16(x, x);
  return u32x4{w, w, w, w};
}

// The piece with its element i taken out (-inf, which adds nothing).
template <bool F32>
__device__ __forceinline__ u32x4 without(u32x4 w, int i) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (F32) {
      if (i == k) w[k] = 0xFF800000u;
    } else {
      if (i == 2 * k) w[k] = (w[k] & 0xFFFF0000u) | 0xFF80u;
      if (i == 2 * k + 1) w[k] = (w[k] & 0xFFFFu) | 0xFF800000u;
    }
  }
  return w;
}

// Running state over a set of logits: their maximum m, s = sum 2^d and t = sum 2^d d with
// d = c (z - m), c = scale log2(e).
struct State {
  float m, s, t;
};

__device__ __forceinline__ State nothing() { return State{kLowest, 0.0f, 0.0f}; }

// The state seen from another maximum (not below its own).
__device__ __forceinline__ State seen(const State &x, float m, float c) {
  const float d = fmaxf(c * (x.m - m), kNoWay), f = __builtin_amdgcn_exp2f(d);
  return State{m, x.s * f, f * fmaf(x.s, d, x.t)};
}

__device__ __forceinline__ State join(const State &x, const State &y, float c) {
  const float m = fmaxf(x.m, y.m);
  const State a = seen(x, m, c), b = seen(y, m, c);
  return State{m, a.s + b.s, a.t + b.t};
}

__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, dpp_f32<kDppQuadXor1>(v));
  v = fmaxf(v, dpp_f32<kDppQuadXor2>(v));
  v = fmaxf(v, dpp_f32<kDppRowHalfMirror>(v));
  v = fmaxf(v, dpp_f32<kDppRowMirror>(v));
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// One batch of a lane.  NaN stays in the sums: only the maximum and the entropy's factor pass it by.  The way to
// the maximum is a difference before it is scaled: exact for near logits and finite for those of the type's
// lowest value (c z - c m in one step was 3 % faster, 8192 x 131072 in 320 us, but off by a step of c m).
template <bool F32, bool ENTROPY>
__device__ __forceinline__ void take(State &x, const u32x4 (&w)[kBatch], float c) {
  constexpr int E = kPiece<F32>;
  float v[kBatch][E];
  float m = x.m;
#pragma unroll
  for (int p = 0; p < kBatch; ++p) {
    values<F32>(w[p], v[p]);
#pragma unroll
    for (int i = 0; i < E; ++i) m = fmaxf(m, v[p][i]);
  }
  const State old = seen(x, m, c);
  float s = old.s, t = old.t;
#pragma unroll
  for (int p = 0; p < kBatch; ++p) {
    // a piece's terms in pairs: a lane's sum of a segment has 11 roundings instead of 64
    float e[E], u = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = c * (v[p][i] - m);
      e[i] = __builtin_amdgcn_exp2f(d);
      if constexpr (ENTROPY) u = i == 0 ? e[i] * fmaxf(d, kNoWay) : fmaf(e[i], fmaxf(d, kNoWay), u);
    }
#pragma unroll
    for (int n = E / 2; n > 0; n /= 2)
#pragma unroll
      for (int i = 0; i < n; ++i) e[i] += e[i + n];
    s += e[0];
    if constexpr (ENTROPY) t += u;
  }
  x = State{m, s, t};
}

// This wave's part of one segment of a row, the chosen token left out; `thread` of the kThreads that take it.
template <bool F32, bool ENTROPY>
__device__ __forceinline__ State segment_state(const void *row, int vocab, int segment, int target, float c, int thread) {
  constexpr int E = kPiece<F32>;
  const int pieces = vocab / E, chosen = target / E;
  const int begin = segment * kSegment, mine = begin + thread;
  State x = nothing();
  if (begin + kSegment <= pieces) {
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
      u32x4 w[kBatch];
#pragma unroll
      for (int p = 0; p < kBatch; ++p) w[p] = load_piece<F32>(row, mine + (b * kBatch + p) * kThreads);
#pragma unroll
      for (int p = 0; p < kBatch; ++p)
        if (mine + (b * kBatch + p) * kThreads == chosen) w[p] = without<F32>(w[p], target - chosen * E);
      take<F32, ENTROPY>(x, w, c);
    }
  } else {
#pragma unroll 1
    for (int b = 0; b < kBatches; ++b) {
      u32x4 w[kBatch];
#pragma unroll
      for (int p = 0; p < kBatch; ++p) {
        const int piece = mine + (b * kBatch + p) * kThreads;
        w[p] = piece_of<F32>(-__builtin_inff());
        if (piece < pieces) w[p] = load_piece<F32>(row, piece);
        if (piece == chosen) w[p] = without<F32>(w[p], target - chosen * E);
      }
      take<F32, ENTROPY>(x, w, c);
    }
  }
  if (begin + kSegment >= pieces) {  // the last segment: what is left behind the last whole piece
    const int i = pieces * E + thread;
    if (i < vocab && i != target) {
      const float z = load_one<F32>(row, i), m = fmaxf(x.m, z);
      x = seen(x, m, c);
      const float d = c * (z - m), e = __builtin_amdgcn_exp2f(d);
      x.s += e;
      x.t = fmaf(e, fmaxf(d, kNoWay), x.t);
    }
  }
  const State y = seen(x, lanes_max(x.m), c);
  return State{y.m, lanes_sum(y.s), ENTROPY ? lanes_sum(y.t) : 0.0f};
}

// A row's chosen token and its logit (-inf where there is none).
template <bool F32>
__device__ __forceinline__ float chosen_logit(const LogprobsArgs &a, int64_t row, int64_t target) {
  const void *z = static_cast<const char *>(a.logits) + row * a.ld * (F32 ? 4 : 2);
  return target >= 0 && target < a.vocab ? load_one<F32>(z, target) : -__builtin_inff();
}

// The row's outputs from the chosen token's logit and the state of all others.
__device__ __forceinline__ void finish(const LogprobsArgs &a, int64_t row, int64_t target, float zt, const State &others, float c) {
  float logp = 0.0f, entropy = 0.0f, m = 0.0f, log_sum = 0.0f;
  if (target >= 0) {
    m = fmaxf(others.m, zt);
    const State x = seen(others, m, c);
    const float way = zt - m, d = c * way, e = __builtin_amdgcn_exp2f(d), sum = x.s + e;
    // the others alone where the chosen token is the largest: exact however small they are
    log_sum = way == 0.0f ? log1pf(x.s) : logf(sum);
    logp = target < a.vocab ? a.scale * way - log_sum : __builtin_nanf("");
    entropy = log_sum - kLn2 * (fmaf(e, fmaxf(d, kNoWay), x.t) / sum);
    if (sum == 0.0f) m = -__builtin_inff();
  }
  if (a.logp) a.logp[row] = logp;
  if (a.entropy) a.entropy[row] = entropy;
  if (a.row_max) a.row_max[row] = m;
  if (a.log_sum) a.log_sum[row] = log_sum;
}

template <bool F32, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobsArgs a, int segments) {
  __shared__ State lds[2][kWaves];
  const float c = a.scale * 1.4426950408889634f;
  const int wave = threadIdx.x >> 6;
  int turn = 0;
  const int64_t units = a.split ? a.rows * segments : a.rows;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x, turn ^= 1) {
    const int64_t row = a.split ? unit / segments : unit;
    const int64_t target = a.targets[row];
    const void *z = static_cast<const char *>(a.logits) + row * a.ld * (F32 ? 4 : 2);
    const int place = target < a.vocab ? (int)target : (int)a.vocab;  // none is taken out past the end
    if (a.split) {
      if (target < 0) continue;
      const State x = segment_state<F32, ENTROPY>(z, (int)a.vocab, (int)(unit - row * segments), place, c, (int)threadIdx.x);
      if ((threadIdx.x & 63) == 0) {
        float *o = a.part + (unit * kWaves + wave) * 4;
        o[0] = x.m;
        o[1] = x.s;
        o[2] = x.t;
      }
      continue;
    }
    const float zt = chosen_logit<F32>(a, row, target);
    State x = nothing();
    if (target >= 0)
      for (int g = 0; g < segments; ++g) x = join(x, segment_state<F32, ENTROPY>(z, (int)a.vocab, g, place, c, (int)threadIdx.x), c);
    if ((threadIdx.x & 63) == 0) lds[turn][wave] = x;
    __syncthreads();
    if (threadIdx.x == 0) {
      x = lds[turn][0];
      for (int w = 1; w < kWaves; ++w) x = join(x, lds[turn][w], c);
      finish(a, row, target, zt, x, c);
    }
  }
}

// A row's state from those of its segments [segment][wave], `Get` of them: by four neighbouring lanes, one for each
// wave that summed, all receiving it.
template <class Get>
__device__ __forceinline__ State join_segments(int segments, float c, Get get) {
  State x = nothing();
#pragma unroll 4
  for (int g = 0; g < segments; ++g) x = join(x, get(g), c);
  const int first = threadIdx.x & 63 & ~(kWaves - 1);
  State all = {__shfl(x.m, first), __shfl(x.s, first), __shfl(x.t, first)};
  for (int w = 1; w < kWaves; ++w) all = join(all, State{__shfl(x.m, first + w), __shfl(x.s, first + w), __shfl(x.t, first + w)}, c);
  return all;
}

// Joins the segments of split rows, four lanes a row.
template <bool F32>
__global__ __launch_bounds__(kWave) void logprobs_join_kernel(const LogprobsArgs a, int segments) {
  const float c = a.scale * 1.4426950408889634f;
  const int64_t row = (int64_t)blockIdx.x * (kWave / kWaves) + threadIdx.x / kWaves;
  const int64_t mine = row < a.rows ? row : a.rows - 1;  // past the last row the last one again, not written
  const int wave = threadIdx.x % kWaves;
  // the segments of a row without a token hold anything, and are not used
  const float *p = a.part + (mine * segments * kWaves + wave) * 4;
  const int64_t target = a.targets[mine];
  const float zt = chosen_logit<F32>(a, mine, target);
  const State x = join_segments(segments, c, [&](int g) {
    const float *q = p + (int64_t)g * kWaves * 4;
    return State{q[0], q[1], q[2]};
  });
  if (wave == 0 && row < a.rows) finish(a, row, target, zt, x, c);
}

// A row by one workgroup, kSide segments side by side.
constexpr int kSide = 4, kMaxWide = 16;  // segments at a time, and of a row

template <bool F32, bool ENTROPY>
__global__ __launch_bounds__(kSide *kThreads) void logprobs_wide_kernel(const LogprobsArgs a, int segments) {
  __shared__ State lds[kMaxWide][kWaves];
  const float c = a.scale * 1.4426950408889634f;
  const int64_t row = blockIdx.x, target = a.targets[row];
  const void *z = static_cast<const char *>(a.logits) + row * a.ld * (F32 ? 4 : 2);
  const int place = target < a.vocab ? (int)target : (int)a.vocab;  // none is taken out past the end
  const float zt = chosen_logit<F32>(a, row, target);
  const int thread = threadIdx.x % kThreads, side = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  if (target >= 0)
    for (int g = side; g < segments; g += kSide) {
      const State x = segment_state<F32, ENTROPY>(z, (int)a.vocab, g, place, c, thread);
      if ((threadIdx.x & 63) == 0) lds[g][thread >> 6] = x;
    }
  __syncthreads();
  if (threadIdx.x >= kWaves) return;
  const State x = join_segments(target >= 0 ? segments : 0, c, [&](int g) { return lds[g][threadIdx.x]; });
  if (threadIdx.x == 0) finish(a, row, target, zt, x, c);
}

// --------------------------------------------------------------- backward --
// Threads of a workgroup by the logits' type, with kBwdPieces of 16 bytes each.  Short-lived one-wave workgroups
// keep reads and writes mixed: 8192 x 131072 bf16 in 595 us, with 128 threads 616, 256 629, with 8 pieces 624 (256
// threads 666), with 2 606.  997 x 50021 f32, whose rows begin anywhere, in 69, 67 and 67 us.
template <bool F32>
constexpr int kBwdThreads = F32 ? 256 : 64;
constexpr int kBwdPieces = 4;
template <bool F32>
constexpr int kBwdChunk = kBwdThreads<F32> * kBwdPieces;

template <bool F32>
__device__ __forceinline__ void store_piece(void *row, int piece, u32x4 w) {
  char *p = static_cast<char *>(row) + (uint32_t)piece * 16u;
  if constexpr (F32) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_f32 *>(p));
  else __builtin_nontemporal_store(w, reinterpret_cast<u32x4_bf16 *>(p));
}

// What a row's gradient is made of.
struct RowGradient {
  float m, log_sum, entropy, g, e;
  float c, log2_sum, scale;
};

template <bool ENTROPY>
__device__ __forceinline__ float gradient(const RowGradient &r, float z) {
  const float way = z - r.m;
  const float p = __builtin_amdgcn_exp2f(fmaf(way, r.c, -r.log2_sum));
  if constexpr (ENTROPY) {
    // -inf: p = 0 times something finite
    const float l = fmaxf(fmaf(way, r.scale, -r.log_sum), kNoWay);
    return -p * fmaf(r.e, l + r.entropy, r.g);
  }
  return -p * r.g;
}

// The chosen token's: 1 - p without cancellation.
template <bool ENTROPY>
__device__ __forceinline__ float chosen_gradient(const RowGradient &r, float z) {
  const float l = r.scale * (z - r.m) - r.log_sum;
  float d = -expm1f(l) * r.g;
  if constexpr (ENTROPY) d -= __builtin_amdgcn_exp2f(l * 1.4426950408889634f) * r.e * (fmaxf(l, kNoWay) + r.entropy);
  return d;
}

template <bool F32, bool ENTROPY>
__global__ __launch_bounds__(kBwdThreads<F32>) void logprobs_bwd_kernel(const LogprobsBwdArgs a, int chunks) {
  constexpr int E = kPiece<F32>;
  const int64_t units = a.rows * chunks;
  const int vocab = (int)a.vocab, pieces = vocab / E;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t row = unit / chunks;
    const int begin = (int)(unit - row * chunks) * kBwdChunk<F32>, mine = begin + (int)threadIdx.x;
    const void *z = static_cast<const char *>(a.logits) + row * a.ld * (F32 ? 4 : 2);
    void *out = static_cast<char *>(a.dlogits) + row * a.ld_out * (F32 ? 4 : 2);
    const int64_t target = a.targets[row];
    RowGradient r{};
    r.g = a.dlogp[row];
    if constexpr (ENTROPY) r.e = a.dentropy[row];
    const bool last = begin + kBwdChunk<F32> >= pieces;
    const int rest = pieces * E + (int)threadIdx.x;  // behind the last whole piece
    if (target < 0 || (r.g == 0.0f && r.e == 0.0f && target < a.vocab)) {
#pragma unroll
      for (int p = 0; p < kBwdPieces; ++p) {
        const int piece = mine + p * kBwdThreads<F32>;
        if (piece < pieces) store_piece<F32>(out, piece, u32x4{});
      }
      if (last && rest < vocab) {
        if constexpr (F32) static_cast<float *>(out)[rest] = 0.0f;
        else static_cast<uint16_t *>(out)[rest] = 0;
      }
      continue;
    }
    u32x4 w[kBwdPieces];
#pragma unroll
    for (int p = 0; p < kBwdPieces; ++p) {
      const int piece = mine + p * kBwdThreads<F32>;
      w[p] = u32x4{};
      if (piece < pieces) w[p] = load_piece<F32>(z, piece);
    }
    r.m = a.row_max[row];
    r.log_sum = a.log_sum[row];
    if constexpr (ENTROPY) r.entropy = a.entropy[row];
    r.scale = a.scale;
    r.c = a.scale * 1.4426950408889634f;
    r.log2_sum = r.log_sum * 1.4426950408889634f;
    if (target >= a.vocab) r.g = __builtin_nanf("");
    const int at = target < vocab ? (int)target : vocab, chosen = at / E, place = at - chosen * E;
#pragma unroll
    for (int p = 0; p < kBwdPieces; ++p) {
      const int piece = mine + p * kBwdThreads<F32>;
      if (piece >= pieces) continue;
      float v[E], d[E];
      values<F32>(w[p], v);
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] = a.scale * gradient<ENTROPY>(r, v[i]);
      if (piece == chosen) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (i == place) d[i] = a.scale * chosen_gradient<ENTROPY>(r, v[i]);
      }
      u32x4 o;
      if constexpr (F32) o = u32x4{__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3])};
      else o = pack_bf16x8(d);
      store_piece<F32>(out, piece, o);
    }
    if (last && rest < vocab) {
      const float v = load_one<F32>(z, rest);
      const float d = a.scale * (rest == target ? chosen_gradient<ENTROPY>(r, v) : gradient<ENTROPY>(r, v));
      if constexpr (F32) static_cast<float *>(out)[rest] = d;
      else static_cast<uint16_t *>(out)[rest] = (uint16_t)pack_bf16(d, d);
    }
  }
}

int64_t segments_of(int64_t vocab, int f32) {
  const int64_t pieces = vocab / (f32 ? 4 : 8);
  return pieces == 0 ? 1 : (pieces + kSegment - 1) / kSegment;
}

// Few rows leave most of the chip idle, and a workgroup takes its segments one after the other.  Two ways out.  Wide:
// four times the waves take four segments at a time, one workgroup a row and so no more rows than CUs.  Split: every
// segment is a workgroup, for a second launch and the partials' way through memory.  bf16, us, whole, wide and split:
//   1 x 32000 (two segments) 6.1, 5.7, 8.2     1 x 65536 (four) 8.2, 6.7, 8.8      1 x 131072 (eight) 13.9, 10.9, 8.6
//   64 x 65536 9.3, 7.4, 8.0                   64 x 131072 15.5, 12.0, 8.3         128 x 131072 16.6, 12.6, 11.2
//   200 x 65536 10.0, 7.6, 10.3                200 x 131072 17.1, 12.9, 14.7       256 x 262144 (16) 31.7, 25.8, 28.1
//   300 x 65536 13.9, 12.6, 11.7               300 x 131072 24.8, 22.1, 18.8       512 x 131072 26.4, 25.3, 27.6
// f32: 16 x 32000 (four) 8.3, 5.7, 8.1, 200 x 131072 (16) 24.7, 19.2, 21.1.
// Between 257 and 512 rows the rule is not the best of the three: rows of up to four segments go whole (300 x 65536
// 13.9 where split takes 11.7), those of more split (512 x 131072 27.6 where wide takes 25.3).
bool wide_rows(int64_t rows, int64_t segments) {
  return rows <= 256 && segments > 1 && segments <= kMaxWide && (rows > 128 || segments <= 4);
}

bool split_rows(int64_t rows, int64_t segments) { return rows <= 512 && segments > 4 && !wide_rows(rows, segments); }

unsigned grid_of(int64_t units) { return (unsigned)(units < (1 << 22) ? units : (1 << 22)); }

}  // namespace

size_t logprobs_part_bytes(int64_t rows, int64_t vocab, int f32) {
  const int64_t segments = segments_of(vocab, f32);
  return split_rows(rows, segments) ? (size_t)rows * (size_t)segments * kWaves * 4 * sizeof(float) : 0;
}

hipError_t launch_logprobs(const LogprobsArgs &args, hipStream_t s) {
  if (args.rows == 0) return hipSuccess;
  LogprobsArgs a = args;
  const int64_t segments = segments_of(a.vocab, a.f32);
  if (wide_rows(a.rows, segments)) {
    const dim3 grid((unsigned)a.rows), block(kSide * kThreads);
    if (a.f32) {
      if (a.entropy) hipLaunchKernelGGL((logprobs_wide_kernel<true, true>), grid, block, 0, s, a, (int)segments);
      else hipLaunchKernelGGL((logprobs_wide_kernel<true, false>), grid, block, 0, s, a, (int)segments);
    } else {
      if (a.entropy) hipLaunchKernelGGL((logprobs_wide_kernel<false, true>), grid, block, 0, s, a, (int)segments);
      else hipLaunchKernelGGL((logprobs_wide_kernel<false, false>), grid, block, 0, s, a, (int)segments);
    }
    return hipGetLastError();
  }
  a.split = split_rows(a.rows, segments) ? 1 : 0;
  const dim3 grid(grid_of(a.split ? a.rows * segments : a.rows)), block(kThreads);
  if (a.f32) {
    if (a.entropy) hipLaunchKernelGGL((logprobs_kernel<true, true>), grid, block, 0, s, a, (int)segments);
    else hipLaunchKernelGGL((logprobs_kernel<true, false>), grid, block, 0, s, a, (int)segments);
  } else {
    if (a.entropy) hipLaunchKernelGGL((logprobs_kernel<false, true>), grid, block, 0, s, a, (int)segments);
    else hipLaunchKernelGGL((logprobs_kernel<false, false>), grid, block, 0, s, a, (int)segments);
  }
  if (a.split) {
    const dim3 joins((unsigned)((a.rows * kWaves + kWave - 1) / kWave));
    if (a.f32) hipLaunchKernelGGL(logprobs_join_kernel<true>, joins, dim3(kWave), 0, s, a, (int)segments);
    else hipLaunchKernelGGL(logprobs_join_kernel<false>, joins, dim3(kWave), 0, s, a, (int)segments);
  }
  return hipGetLastError();
}

namespace {

template <bool F32>
void launch_bwd(const LogprobsBwdArgs &a, hipStream_t s) {
  const int64_t pieces = a.vocab / kPiece<F32>;
  const int64_t chunks = pieces == 0 ? 1 : (pieces + kBwdChunk<F32> - 1) / kBwdChunk<F32>;
  const dim3 grid(grid_of(a.rows * chunks)), block(kBwdThreads<F32>);
  if (a.dentropy) hipLaunchKernelGGL((logprobs_bwd_kernel<F32, true>), grid, block, 0, s, a, (int)chunks);
  else hipLaunchKernelGGL((logprobs_bwd_kernel<F32, false>), grid, block, 0, s, a, (int)chunks);
}

}  // namespace

hipError_t launch_logprobs_bwd(const LogprobsBwdArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.f32) launch_bwd<true>(a, s);
  else launch_bwd<false>(a, s);
  return hipGetLastError();
}

}  // namespace hilore
