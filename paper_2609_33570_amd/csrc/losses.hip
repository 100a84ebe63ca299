// Clipped policy loss and preference loss with their gradients, on gfx950.
//
//   policy      -A r, or -A times the bound that the log ratio is past;  + beta kl - bonus entropy;  times a weight
//   preference  of h = L_chosen - L_rejected, L a sequence's sum of log-ratios:  softplus, hinge or square
//
// Small against the logits' passes (13 to 35 B a token): launches and the latencies inside them
// bound both.  Three steps each: sums by sequence, then the tokens (policy) or the pairs (preference), then the
// statistics or the tokens; every step is a launch, or all are one workgroup's phases where there is little to do.
// Partial sums of a step's workgroups are added by the next step in a fixed order, in fp64.
//
// Whole passes: policy 1024 tokens 7.3 us, 2^20 packed tokens in 512 sequences 21 to 22 us (steps 6.8, 13.0 and 3.9 under a
// trace; the bytes alone take 6); preference 16 x 211 tokens 8.2 us, 2^20 tokens in 768 sequences and 1152 listed
// pairs 16 us (4.6, 5.3 and 6.4).
#include "device_common.hpp"
#include "hilore_internal.hpp"

#include <type_traits>

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kSmall = 1024, kMaxWaves = kSmall / kWave;  // threads of the one workgroup of a small call
constexpr int kMaxGroups = 1024;  // workgroups of a launch, each with partial sums
constexpr int kMaxSums = 6;

typedef float f32x4 __attribute__((ext_vector_type(4)));
// Tensors may begin at any element.
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef uint32_t __attribute__((aligned(1))) u32_any;

// Valid tokens and sequences that have any, each below 2^31.
struct Counts {
  uint32_t tokens, sequences;
};

// Sum over aligned groups of W lanes (8 or 64), all of them receiving it.
template <int W>
__device__ __forceinline__ uint32_t lanes_sum_u32(uint32_t v) {
  static_assert(W == 8 || W == 64, "group size");
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kDppQuadXor1, 0xF, 0xF, true);
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kDppQuadXor2, 0xF, 0xF, true);
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kDppRowHalfMirror, 0xF, 0xF, true);
  if constexpr (W == 8) return v;
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kDppRowMirror, 0xF, 0xF, true);
  auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = p[0] + p[1];
  p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return p[0] + p[1];
}

// The sum of `groups` workgroups' counts, by every wave for itself: no barrier.
__device__ __forceinline__ Counts sum_counts(const Counts *part, int groups) {
  Counts n = {0, 0};
#pragma unroll 8
  for (int g = threadIdx.x & 63; g < groups; g += kWave) {
    n.tokens += part[g].tokens;
    n.sequences += part[g].sequences;
  }
  return Counts{lanes_sum_u32<kWave>(n.tokens), lanes_sum_u32<kWave>(n.sequences)};
}

// A workgroup's place in its step: `groups` of them take part, this is number `group`.  Its threads T are
// a constant of the step (blockDim would be a load that everything waits for).
struct Place {
  int group, groups;
};

template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 o = {(uint32_t)__builtin_amdgcn_mov_dpp((int)w.x, CTRL, 0xF, 0xF, true),
                   (uint32_t)__builtin_amdgcn_mov_dpp((int)w.y, CTRL, 0xF, 0xF, true)};
  return __builtin_bit_cast(double, o);
}

// Sum over aligned groups of W lanes (8 or 64), all of them receiving it, without LDS instructions.
template <int W>
__device__ __forceinline__ double lanes_sum64(double v) {
  static_assert(W == 8 || W == 64, "group size");
  v += dpp_f64<kDppQuadXor1>(v);
  v += dpp_f64<kDppQuadXor2>(v);
  v += dpp_f64<kDppRowHalfMirror>(v);
  if constexpr (W == 64) {
    v += dpp_f64<kDppRowMirror>(v);
    u32x2 w = __builtin_bit_cast(u32x2, v);
    auto x = __builtin_amdgcn_permlane16_swap(w.x, w.x, false, false);
    auto y = __builtin_amdgcn_permlane16_swap(w.y, w.y, false, false);
    v = __builtin_bit_cast(double, u32x2{x[0], y[0]}) + __builtin_bit_cast(double, u32x2{x[1], y[1]});
    w = __builtin_bit_cast(u32x2, v);
    x = __builtin_amdgcn_permlane32_swap(w.x, w.x, false, false);
    y = __builtin_amdgcn_permlane32_swap(w.y, w.y, false, false);
    v = __builtin_bit_cast(double, u32x2{x[0], y[0]}) + __builtin_bit_cast(double, u32x2{x[1], y[1]});
  }
  return v;
}

// N sums of each wave added over the workgroup, all threads receiving them.  `lds` has room for N sums of
// each wave.
template <int T, int N>
__device__ __forceinline__ void add_waves(double (&v)[N], double (*lds)[kMaxSums]) {
  constexpr int waves = T / kWave;
  __syncthreads();  // the sums before have been read
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

template <int T, int N>
__device__ __forceinline__ void group_sums(double (&v)[N], double (*lds)[kMaxSums]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lanes_sum64<64>(v[k]);
  add_waves<T>(v, lds);
}

// N sums of each wave (the same in all its lanes) added over the workgroup, to out[N].
template <int T, int N>
__device__ __forceinline__ void put_sums(const double (&v)[N], double (*lds)[kMaxSums], double *out) {
  __syncthreads();  // the sums before have been read
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) lds[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
  if (threadIdx.x >= N) return;
  double sum = lds[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < T / kWave; ++w) sum += lds[w][threadIdx.x];
  out[threadIdx.x] = sum;
}

// The sums of `groups` workgroups' N partial sums, by every wave for itself: no barrier.
template <int N>
__device__ __forceinline__ void sum_parts(const double *part, int groups, double (&v)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.0;
#pragma unroll 8
  for (int g = threadIdx.x & 63; g < groups; g += kWave)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += part[(int64_t)g * N + k];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = lanes_sum64<64>(v[k]);
}

// Tokens and sequences are numbered in 32 bits (both are below 2^31); an offset outside [0, tokens]
// counts as the nearer end.
__device__ __forceinline__ int offset(const SequencesArgs &q, int s) {
  const int64_t x = q.offsets[s];
  return (int)(x < 0 ? 0 : x > q.tokens ? q.tokens : x);
}

// Tokens [begin, end) of a sequence.
__device__ __forceinline__ void bounds(const SequencesArgs &q, int s, int &begin, int &end) {
  if (q.offsets) {
    begin = offset(q, s);
    end = offset(q, s + 1);
  } else {
    begin = s * (int)q.length;
    end = begin + (int)q.length;
  }
}

// The last sequences that begin at tokens t0 and t1 or before them, -1 where none does.  By a wave, all
// lanes with the same tokens: the lanes read 64 offsets at a time for each, so that 64^k sequences take k
// rounds of loads.  (1024 offsets at once, in one round, took 2 us longer of 13: more instructions.)
__device__ __forceinline__ void begins_before(const SequencesArgs &q, int t0, int t1, int &s0, int &s1) {
  const int lane = threadIdx.x & 63;
  const int t[2] = {t0, t1};
  int lo[2] = {0, 0}, n[2] = {(int)q.sequences, (int)q.sequences};  // the number that begin by then is in [lo, lo + n]
  while (n[0] > 0 || n[1] > 0) {
    int begin[2], step[2];
    bool read[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      step[k] = (int)(((uint32_t)n[k] + kWave - 1) / kWave);
      const int64_t i = (int64_t)(lane + 1) * step[k] - 1;
      read[k] = i < n[k];
      begin[k] = offset(q, read[k] ? lo[k] + (int)i : 0);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int before = __popcll(__ballot(read[k] && begin[k] <= t[k]));  // the offsets rise: the first ones read
      const int left = n[k] - before * step[k];
      lo[k] += before * step[k];
      n[k] = n[k] == 0 ? 0 : min(step[k] - 1, left);
    }
  }
  s0 = lo[0] - 1;
  s1 = lo[1] - 1;
}

// The last sequence of [lo, hi] that begins at token t or before it, lo - 1 where none does.
__device__ __forceinline__ int begins_between(const SequencesArgs &q, int t, int lo, int hi) {
  ++hi;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (offset(q, mid) <= t) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// For every sequence the number of its valid tokens and, with DIFFERENCE, the sum over them of
// x - y (x alone without y), to done(sequence, count, sum) in one thread.  W threads a sequence: 8 or 64
// lanes, or (0) the workgroup.
template <int T, int W, bool DIFFERENCE, class Done>
__device__ __forceinline__ void sum_sequences(const SequencesArgs &q, const float *x, const float *y, Place at, double (*lds)[kMaxSums],
                                              Done done) {
  constexpr int threads = W ? W : T, side = T / threads;
  constexpr int kAhead = W == 0 && T > kThreads ? 8 : 4;  // tokens of a thread in flight
  const int mine = (int)threadIdx.x % threads;
  // Loads without branches, which would each wait for their own: what is not there is read from
  // x and not used, past the end the last token again.
  const uint8_t *mask = q.mask ? q.mask : reinterpret_cast<const uint8_t *>(x);
  const float *from = y ? y : x;
  const bool all = !q.mask;
  // lanes of a wave stay together for the reduction: sequences past the last are empty
  for (int64_t base = (int64_t)at.group * side; base < q.sequences; base += (int64_t)at.groups * side) {
    const int s = (int)(base + (int)threadIdx.x / threads);
    const bool live = base + (int)threadIdx.x / threads < q.sequences;
    int begin = 0, end = 0;
    if (live) bounds(q, s, begin, end);
    uint32_t count = 0;
    double sum[1] = {0.0};
    for (int64_t t = (int64_t)begin + mine; t < end; t += kAhead * threads) {
      uint8_t m[kAhead];
      float u[kAhead], v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int k = t + i * threads < end ? (int)t + i * threads : end - 1;
        m[i] = mask[k];
        if constexpr (DIFFERENCE) {
          u[i] = x[k];
          v[i] = from[k];
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const bool ok = t + i * threads < end && (all || m[i] != 0);
        count += ok ? 1 : 0;
        if constexpr (DIFFERENCE) sum[0] += ok ? (double)(u[i] - (y ? v[i] : 0.0f)) : 0.0;
      }
    }
    if constexpr (W) {
      count = lanes_sum_u32<W>(count);
      if constexpr (DIFFERENCE) sum[0] = lanes_sum64<W>(sum[0]);
    } else {
      double both[2] = {(double)lanes_sum_u32<kWave>(count), DIFFERENCE ? lanes_sum64<kWave>(sum[0]) : 0.0};
      add_waves<T>(both, lds);
      count = (uint32_t)both[0];
      sum[0] = both[1];
    }
    if (mine == 0 && live) done(s, count, sum[0]);
  }
}

constexpr int kVector = 4;  // tokens of a lane; in a small call 1, which spreads them over more waves

// V neighbouring tokens of a lane from t on: their sequences and whether they are valid.
template <int V>
struct Tokens {
  int64_t t;
  int s[V];       // in no sequence: 0, and not inside
  bool inside[V], ok[V];
  bool whole;     // all of them are inside a sequence
};

// N arrays' values at a lane's tokens before `end`.  Whole waves of tokens are loaded as vectors, the last ones one
// by one (past the end the last token again).
template <int V, int N>
__device__ __forceinline__ void load(const float *const (&p)[N], int64_t first, int64_t t, int64_t end, float (&v)[N][V]) {
  if (V == 4 && first + V * kWave <= end) {
    f32x4 x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = *reinterpret_cast<const f32x4_any *>(p[k] + t);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) v[k][i] = x[k][i];
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) v[k][i] = p[k][t + i < end ? t + i : end - 1];
}

template <int V>
__device__ __forceinline__ void store(float *p, const Tokens<V> &k, const float (&v)[V]) {
  if constexpr (V == 4) {
    if (k.whole) {
      *reinterpret_cast<f32x4_any *>(p + k.t) = f32x4{v[0], v[1], v[2], v[3]};
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (k.inside[i]) p[k.t + i] = v[i];
}

// The mask's bytes at a lane's tokens before `end`.
template <int V>
__device__ __forceinline__ uint32_t mask_at(const SequencesArgs &q, int64_t first, int64_t t, int64_t end) {
  if (!q.mask) return 0x01010101u;
  if (V == 4 && first + V * kWave <= end) return *reinterpret_cast<const u32_any *>(q.mask + t);
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) mask |= (uint32_t)q.mask[t + i < end ? t + i : end - 1] << (8 * i);
  return mask;
}

template <int V>
__device__ __forceinline__ void set_valid(Tokens<V> &k, uint32_t mask) {
  k.whole = true;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    k.ok[i] = k.inside[i] && ((mask >> (8 * i)) & 0xFFu) != 0;
    k.whole = k.whole && k.inside[i];
  }
}

// A wave's tokens from `first` on, all of sequence s, which ends at `end` (first < end).
template <int V>
__device__ __forceinline__ Tokens<V> tokens_of(const SequencesArgs &q, int s, int64_t first, int64_t end) {
  Tokens<V> k;
  k.t = first + (int64_t)(threadIdx.x & 63) * V;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    k.s[i] = s;
    k.inside[i] = k.t + i < end;
  }
  set_valid(k, mask_at<V>(q, first, k.t, end));
  return k;
}

// A wave's tokens from `first` on (first < q.tokens), of whatever sequences (there is one at least: its ends are read).
template <int V>
__device__ __forceinline__ Tokens<V> tokens_at(const SequencesArgs &q, int64_t first) {
  Tokens<V> k;
  k.t = first + (int64_t)(threadIdx.x & 63) * V;
  const uint32_t mask = mask_at<V>(q, first, k.t, q.tokens);
  if (q.offsets) {
    const int64_t end = first + V * kWave < q.tokens ? first + V * kWave : q.tokens;
    int lo, hi;
    begins_before(q, (int)first, (int)end - 1, lo, hi);
    lo = lo < 0 ? 0 : lo;
    hi = hi < lo ? lo : hi;  // offsets that do not rise
    if (lo == hi) {          // one sequence: the whole wave reads its ends
      const int begin = offset(q, lo), last = offset(q, lo + 1);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        k.inside[i] = k.t + i < q.tokens && begin <= k.t + i && k.t + i < last;
        k.s[i] = lo;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int s = begins_between(q, k.t + i < q.tokens ? (int)k.t + i : (int)q.tokens - 1, lo, hi);
        k.s[i] = s < 0 ? 0 : s;
      }
#pragma unroll
      for (int i = 0; i < V; ++i)
        k.inside[i] = k.t + i < q.tokens && offset(q, k.s[i]) <= k.t + i && k.t + i < offset(q, k.s[i] + 1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      k.inside[i] = k.t + i < q.tokens;
      k.s[i] = k.inside[i] ? (int)((uint32_t)(k.t + i) / (uint32_t)q.length) : 0;
    }
  }
  set_valid(k, mask);
  return k;
}

// Calls tile(tokens, first, end) for this wave's tiles of V tokens a lane.  Workgroups share the tokens
// sequence by sequence, `chunks` of them to each, or in tiles of all tokens, whose sequences are searched
// for: that takes five dependent loads where the other way takes two, but no workgroup for a short sequence.
template <int T, int V, bool BY_SEQUENCE, class Tile>
__device__ __forceinline__ void each_tile(const SequencesArgs &q, Place at, int chunks, Tile tile) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (BY_SEQUENCE) {
    const int64_t units = q.sequences * chunks;
    for (int64_t unit = at.group; unit < units; unit += at.groups) {
      const int s = (int)(unit / chunks);
      int begin, end;
      bounds(q, s, begin, end);
      for (int64_t first = begin + (unit - (int64_t)s * chunks) * (T * V) + wave * (V * kWave); first < end; first += (int64_t)chunks * (T * V))
        tile(tokens_of<V>(q, s, first, end), first, (int64_t)end);
    }
  } else {
    const int64_t step = (int64_t)at.groups * T * V;
    for (int64_t first = (int64_t)at.group * T * V + wave * (V * kWave); first < q.tokens; first += step)
      tile(tokens_at<V>(q, first), first, q.tokens);
  }
}

// ----------------------------------------------------------------- policy --
// Valid tokens of each sequence and, for the sequences' ratios, their mean log ratio; partial
// sums of the valid tokens and of the sequences that have any.
template <int T, int W, bool RATIO>
__device__ __forceinline__ void policy_sequences(const PolicyArgs &a, Place at, Counts *part, double (*lds)[kMaxSums]) {
  Counts total = {0, 0};
  sum_sequences<T, W, RATIO>(a.seq, a.logp, a.old, at, lds, [&](int s, uint32_t count, double sum) {
    total.tokens += count;
    total.sequences += count > 0 ? 1 : 0;
    const double share = count > 0 ? 1.0 / (double)count : 0.0;
    a.share[s] = share;
    if constexpr (RATIO) a.mean_delta[s] = (float)(sum * share);
  });
  if constexpr (W) {  // else they are one thread's
    double both[2] = {(double)lanes_sum_u32<kWave>(total.tokens), (double)lanes_sum_u32<kWave>(total.sequences)};
    add_waves<T>(both, lds);
    total = Counts{(uint32_t)both[0], (uint32_t)both[1]};
  }
  if (threadIdx.x == 0) part[at.group] = total;
}

constexpr int kPolicySums = 6;  // policy, kl, entropy, loss, clipped, ratio

// exp(-x) - 1 + x, whose first terms cancel near 0, where a policy is beside its reference: x^2 / 2 times its series
// 2 (-x)^k / (k + 2)! below 1 (cut off at 2^-27), the sum from expm1 beyond.  Relative to the value within 2^-21
// everywhere; the sum alone was 1 % off at 1e-5.
__device__ __forceinline__ float k3(float x, float e) {
  float h = 2.0f / 39916800.0f;
  h = fmaf(h, -x, 2.0f / 3628800.0f);
  h = fmaf(h, -x, 2.0f / 362880.0f);
  h = fmaf(h, -x, 2.0f / 40320.0f);
  h = fmaf(h, -x, 2.0f / 5040.0f);
  h = fmaf(h, -x, 2.0f / 720.0f);
  h = fmaf(h, -x, 2.0f / 120.0f);
  h = fmaf(h, -x, 2.0f / 24.0f);
  h = fmaf(h, -x, 2.0f / 6.0f);
  h = fmaf(h, -x, 1.0f);
  return fabsf(x) < 1.0f ? 0.5f * x * x * h : e + x;
}

struct TokenLoss {
  float loss, policy, kl, dlogp, ratio;
  uint8_t flags;
};

__device__ __forceinline__ TokenLoss token_loss(const PolicyArgs &a, float delta, float adv, float x, float entropy) {
  TokenLoss o;
  o.ratio = expf(delta);
  bool chi = !(adv >= 0.0f ? delta > a.log_high : adv < 0.0f && delta < a.log_low);  // no bound hides a NaN
  float bound = adv >= 0.0f ? a.bound_high : a.bound_low;
  if (a.dual > 0.0f && adv < 0.0f && delta > a.log_dual) {
    chi = false;
    bound = a.dual;
  }
  // a response without advantage has no policy term, whatever its ratio
  o.policy = adv == 0.0f ? 0.0f : -adv * (chi ? o.ratio : bound);
  float slope = chi && adv != 0.0f ? -adv * o.ratio : 0.0f;
  o.kl = 0.0f;
  o.loss = o.policy;
  if (a.kl) {
    float dkl = 1.0f;
    o.kl = x;
    if (a.kl == 2) {
      o.kl = 0.5f * x * x;
      dkl = x;
    } else if (a.kl == 3) {
      const float e = expm1f(-x);
      o.kl = k3(x, e);
      dkl = -e;
    }
    // a term of weight 0 is watched in its statistic alone: exp(-x) may be past fp32
    if (a.beta != 0.0f) {
      o.loss += a.beta * o.kl;
      slope += a.beta * dkl;
    }
  }
  if (a.bonus != 0.0f) o.loss -= a.bonus * entropy;
  o.dlogp = slope;
  o.flags = (uint8_t)((chi ? 1 : 0) | (!chi && adv != 0.0f ? 2 : 0));
  return o;
}

template <int T, int V>
__device__ __forceinline__ void policy_tokens(const PolicyArgs &a, Place at, const Counts *counted, int counters, double *part,
                                              double (*lds)[kMaxSums]) {
  double each = 0.0;  // 1 / N
  bool have = false;
  double sum[kPolicySums] = {};
  // what is not there is read from what is, and not used: branches around the loads would each wait
  const float *const from[4] = {a.logp, a.old, a.kl ? a.ref : a.logp, a.entropy ? a.entropy : a.logp};
  const float *const mean = a.sequence_ratio ? a.mean_delta : reinterpret_cast<const float *>(a.share);
  each_tile<T, V, false>(a.seq, at, 0, [&](const Tokens<V> &k, int64_t first, int64_t end) {
    float in[4][V], adv[V], delta[V];
    double w64[V];
    const int64_t t = k.t;
    load<V>(from, first, t, end, in);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      delta[i] = mean[k.s[i]];
      w64[i] = a.share[k.s[i]];
      adv[i] = a.adv[a.adv_per_token ? (t + i < end ? t + i : end - 1) : k.s[i]];
    }
    if (!have) {  // behind the first loads, which need not wait for it
      const Counts n = sum_counts(counted, counters);
      each = 1.0 / (a.n_norm > 0.0 ? a.n_norm : (double)(a.sequence_mean ? n.sequences : n.tokens));
      have = true;
    }
    float dlogp[V], dent[V], loss[V];
    // The statistics of a wave's tokens are added in fp32, beyond them in fp64: at most 10 roundings (4 of a lane's tokens,
    // 6 over the lanes), as many as a token's loss itself has in fp32, and of their sizes' sum as those are.  In fp64 from
    // the tokens on a pass over 1024 tokens took 0.55 us longer (7.6), one over 2^20 0.65 (15.1 and 17.1).
    float some[kPolicySums] = {};
    uint32_t flags = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dlogp[i] = dent[i] = loss[i] = 0.0f;
      if (!k.ok[i]) continue;
      const float h = a.entropy ? in[3][i] : 0.0f;
      const TokenLoss o = token_loss(a, a.sequence_ratio ? delta[i] : in[0][i] - in[1][i], adv[i], in[0][i] - in[2][i], h);
      const float w = (float)(a.sequence_mean ? w64[i] * each : each);
      dlogp[i] = w * o.dlogp;
      dent[i] = -a.bonus * w;
      loss[i] = w * o.loss;
      flags |= (uint32_t)o.flags << (8 * i);
      some[0] = fmaf(w, o.policy, some[0]);
      some[1] = fmaf(w, o.kl, some[1]);
      some[2] = fmaf(w, h, some[2]);
      some[3] += loss[i];
      some[4] += (float)(o.flags >> 1);
      some[5] += o.ratio;
    }
#pragma unroll
    for (int j = 0; j < kPolicySums; ++j) sum[j] += (double)lanes_sum(some[j]);
    if (a.dlogp) store<V>(a.dlogp, k, dlogp);
    if (a.dentropy) store<V>(a.dentropy, k, dent);
    if (a.token_loss) store<V>(a.token_loss, k, loss);
    if (a.flags) {
      if (V == 4 && k.whole) {
        *reinterpret_cast<u32_any *>(a.flags + t) = flags;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (k.inside[i]) a.flags[t + i] = (uint8_t)(flags >> (8 * i));
      }
    }
  });
  if (a.stats) put_sums<T>(sum, lds, part + (int64_t)at.group * kPolicySums);
}

template <int T>
__device__ __forceinline__ void policy_fold(const PolicyArgs &a, const Counts *counted, int counters, const double *part, int groups,
                                            double (*lds)[kMaxSums]) {
  double v[kPolicySums] = {};
#pragma unroll 4
  for (int g = threadIdx.x; g < groups; g += T)
#pragma unroll
    for (int k = 0; k < kPolicySums; ++k) v[k] += part[(int64_t)g * kPolicySums + k];
  const Counts n = sum_counts(counted, counters);
  group_sums<T>(v, lds);
  if (threadIdx.x != 0) return;
  const double each = n.tokens > 0 ? (double)n.tokens : 1.0;
  a.stats[0] = (float)v[3];
  a.stats[1] = (float)v[0];
  a.stats[2] = (float)v[1];
  a.stats[3] = (float)v[2];
  a.stats[4] = (float)(v[4] / each);
  a.stats[5] = (float)(v[5] / each);
  a.stats[6] = (float)n.tokens;
  a.stats[7] = (float)n.sequences;
}

template <int T, int W, bool RATIO>
__global__ __launch_bounds__(T) void policy_sequences_kernel(const PolicyArgs a, Counts *part) {
  __shared__ double lds[T / kWave][kMaxSums];
  policy_sequences<T, W, RATIO>(a, Place{(int)blockIdx.x, (int)gridDim.x}, part, lds);
}

__global__ __launch_bounds__(kThreads) void policy_tokens_kernel(const PolicyArgs a, const Counts *counted, int counters, double *part) {
  __shared__ double lds[kWaves][kMaxSums];
  policy_tokens<kThreads, kVector>(a, Place{(int)blockIdx.x, (int)gridDim.x}, counted, counters, part, lds);
}

__global__ __launch_bounds__(kThreads) void policy_fold_kernel(const PolicyArgs a, const Counts *counted, int counters,
                                                               const double *part, int groups) {
  __shared__ double lds[kWaves][kMaxSums];
  policy_fold<kThreads>(a, counted, counters, part, groups, lds);
}

// All steps by one workgroup.
template <int W, bool RATIO>
__global__ __launch_bounds__(kSmall) void policy_small_kernel(const PolicyArgs a, Counts *counted, double *part) {
  __shared__ double lds[kMaxWaves][kMaxSums];
  const Place alone = {0, 1};
  policy_sequences<kSmall, W, RATIO>(a, alone, counted, lds);
  __syncthreads();
  policy_tokens<kSmall, 1>(a, alone, counted, 1, part, lds);
  __syncthreads();
  if (a.stats) policy_fold<kSmall>(a, counted, 1, part, 1, lds);
}

// ------------------------------------------------------------- preference --
// Valid tokens of each sequence and the sum (or mean) of its log-ratios.
template <int T, int W>
__device__ __forceinline__ void preference_sequences(const PreferenceArgs &a, Place at, double (*lds)[kMaxSums]) {
  sum_sequences<T, W, true>(a.seq, a.logp, a.ref, at, lds, [&](int s, uint32_t count, double sum) {
    const double value = a.length_mean && count > 0 ? sum / (double)count : sum;
    a.count[s] = count;
    a.value[s] = value;
    if (a.rewards) a.rewards[s] = (float)((double)a.beta * value);
  });
}

struct Pair {
  double used, loss, slope, h, chosen, rejected;  // slope: of the loss by h
};

__device__ __forceinline__ Pair pair_loss(const PreferenceArgs &a, int64_t win, int64_t lose) {
  Pair p{};
  if (win < 0 || lose < 0) return p;
  if (win >= a.seq.sequences || lose >= a.seq.sequences) {
    const double nan = __builtin_nan("");
    return Pair{nan, nan, nan, nan, nan, nan};
  }
  if (a.count[win] == 0 || a.count[lose] == 0) return p;
  const double beta = a.beta;
  p.used = 1.0;
  p.chosen = beta * a.value[win];
  p.rejected = beta * a.value[lose];
  p.h = a.value[win] - a.value[lose] - (double)a.margin;
  const double y = beta * p.h;
  if (a.loss == 0) {
    const double eps = a.smoothing, tail = log1p(exp(-fabs(y)));
    // softplus(-y) and softplus(y); their slopes are -sigmoid(-y) and sigmoid(y).  An infinite one of weight 0 adds
    // nothing: y is +inf where a token of the rejected has the log-probability -inf
    p.loss = (1.0 - eps) * (fmax(-y, 0.0) + tail);
    if (eps > 0.0) p.loss += eps * (fmax(y, 0.0) + tail);
    p.slope = beta * (eps / (1.0 + exp(-y)) - (1.0 - eps) / (1.0 + exp(y)));
  } else if (a.loss == 1) {
    p.loss = y < 1.0 ? 1.0 - y : 0.0;
    p.slope = y < 1.0 ? -beta : 0.0;
    if (y != y) p.loss = p.slope = y;
  } else {
    const double d = p.h - 0.5 / beta;
    p.loss = d * d;
    p.slope = 2.0 * d;
  }
  return p;
}

// The slope by each valid token's log-probability, of the one by the sequence's value.
__device__ __forceinline__ double of_token(const PreferenceArgs &a, int64_t s, double slope) {
  return a.length_mean && a.count[s] > 0 ? slope / (double)a.count[s] : slope;
}

constexpr int kPairSums = 6;  // used, loss, h > 0, beta h, chosen and rejected rewards

template <int T>
__device__ __forceinline__ void preference_pairs(const PreferenceArgs &a, Place at, double *part, double (*lds)[kMaxSums]) {
  double sum[kPairSums] = {};
  for (int64_t p = (int64_t)at.group * T + threadIdx.x; p < a.pairs; p += (int64_t)at.groups * T) {
    const Pair o = pair_loss(a, a.chosen ? a.chosen[p] : 2 * p, a.chosen ? a.rejected[p] : 2 * p + 1);
    if (a.pair_loss) a.pair_loss[p] = (float)o.loss;
    if (!a.chosen) {
      a.slope[2 * p] = of_token(a, 2 * p, o.slope);
      a.slope[2 * p + 1] = of_token(a, 2 * p + 1, -o.slope);
    }
    sum[0] += o.used;
    sum[1] += o.loss;
    sum[2] += o.h > 0.0 ? 1.0 : 0.0;
    sum[3] += (double)a.beta * o.h;
    sum[4] += o.chosen;
    sum[5] += o.rejected;
  }
  group_sums<T>(sum, lds);
  if (threadIdx.x == 0)
    for (int k = 0; k < kPairSums; ++k) part[(int64_t)at.group * kPairSums + k] = sum[k];
}

// With lists: the slope of each sequence over its pairs, a wave a sequence, which reads the lists.
template <int T>
__device__ __forceinline__ void preference_lists(const PreferenceArgs &a, Place at) {
  constexpr int waves = T / kWave;
  const int lane = threadIdx.x & 63;
  for (int64_t s = (int64_t)at.group * waves + (threadIdx.x >> 6); s < a.seq.sequences; s += (int64_t)at.groups * waves) {
    double slope = 0.0;
    constexpr int kAhead = 8;  // pairs of a lane in flight
    for (int64_t p = lane; p < a.pairs; p += kAhead * kWave) {
      int32_t win[kAhead], lose[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t u = p + i * kWave < a.pairs ? p + i * kWave : a.pairs - 1;
        win[i] = a.chosen[u];
        lose[i] = a.rejected[u];
      }
      uint32_t hits = 0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        hits |= p + i * kWave < a.pairs && (win[i] == (int32_t)s || lose[i] == (int32_t)s) ? 1u << i : 0u;
      for (; hits != 0; hits &= hits - 1) {
        int32_t c = win[0], r = lose[0];
        const int hit = __builtin_ctz(hits);
#pragma unroll
        for (int i = 1; i < kAhead; ++i) {
          c = hit == i ? win[i] : c;
          r = hit == i ? lose[i] : r;
        }
        const double d = pair_loss(a, c, r).slope;
        if (c == s) slope += d;
        if (r == s) slope -= d;
      }
    }
    slope = lanes_sum64<64>(slope);
    if (lane == 0) a.slope[s] = of_token(a, s, slope);
  }
}

template <int T, int V, bool BY_SEQUENCE>
__device__ __forceinline__ void preference_tokens(const PreferenceArgs &a, Place at, int chunks, const double *part, int groups) {
  double v[kPairSums];
  sum_parts<kPairSums>(part, groups, v);
  // a pair with a number out of range makes v[0] NaN, and so all that follows
  const double norm = a.n_norm > 0.0 ? a.n_norm + 0.0 * v[0] : v[0] == 0.0 ? 1.0 : v[0];
  if (at.group == 0 && threadIdx.x == 0 && a.stats) {
    for (int k = 1; k < kPairSums; ++k) a.stats[k - 1] = (float)(v[k] / norm);
    a.stats[5] = (float)v[0];
  }
  if (!a.dlogp || a.seq.sequences == 0) return;  // tokens of no sequence are left as they were
  const double each = 1.0 / norm;
  each_tile<T, V, BY_SEQUENCE>(a.seq, at, chunks, [&](const Tokens<V> &k, int64_t, int64_t) {
    double slope[V];
    float d[V];
    // without lists the last of an odd number of sequences is in no pair
#pragma unroll
    for (int i = 0; i < V; ++i) slope[i] = a.slope[k.s[i]];
#pragma unroll
    for (int i = 0; i < V; ++i)
      d[i] = k.ok[i] ? (float)((a.chosen || k.s[i] < 2 * a.pairs ? slope[i] : 0.0) * each) : 0.0f;
    store<V>(a.dlogp, k, d);
  });
}

template <int T, int W>
__global__ __launch_bounds__(T) void preference_sequences_kernel(const PreferenceArgs a) {
  __shared__ double lds[T / kWave][kMaxSums];
  preference_sequences<T, W>(a, Place{(int)blockIdx.x, (int)gridDim.x}, lds);
}

// The first `pairs` workgroups take the pairs, the others the sequences' lists.
__global__ __launch_bounds__(kThreads) void preference_pairs_kernel(const PreferenceArgs a, int pairs, double *part) {
  __shared__ double lds[kWaves][kMaxSums];
  if ((int)blockIdx.x < pairs) preference_pairs<kThreads>(a, Place{(int)blockIdx.x, pairs}, part, lds);
  else preference_lists<kThreads>(a, Place{(int)blockIdx.x - pairs, (int)gridDim.x - pairs});
}

template <int T, bool BY_SEQUENCE>
__global__ __launch_bounds__(T) void preference_tokens_kernel(const PreferenceArgs a, int chunks, const double *part, int groups) {
  preference_tokens<T, kVector, BY_SEQUENCE>(a, Place{(int)blockIdx.x, (int)gridDim.x}, chunks, part, groups);
}

template <int W>
__global__ __launch_bounds__(kSmall) void preference_small_kernel(const PreferenceArgs a, double *part) {
  __shared__ double lds[kMaxWaves][kMaxSums];
  const Place alone = {0, 1};
  preference_sequences<kSmall, W>(a, alone, lds);
  __syncthreads();
  preference_pairs<kSmall>(a, alone, part, lds);
  if (a.chosen && a.dlogp) preference_lists<kSmall>(a, alone);
  __syncthreads();
  preference_tokens<kSmall, 1, false>(a, alone, 0, part, 1);
}

int groups_of(int64_t work, int64_t each) {
  const int64_t need = (work + each - 1) / each;
  return (int)(need < kMaxGroups ? need : kMaxGroups);
}

// One workgroup does all of a call whose steps would each be little more than a launch.  Policy, one workgroup
// against three launches (12.6 us up to some 8000 tokens): 64 tokens 7.6 us, 1024 7.3 to 8.9, 2048 10.6, 4096 16.
// Preference (12.1): 1024 tokens 9.2, 3400 8.2, 4096 12 to 13.  With lists its 16 waves read them for a sequence
// each: 98 sequences took 20 us, by launches 11.
constexpr int kSmallPolicy = 2 * kSmall, kSmallPreference = 4 * kSmall;  // tokens
bool small_call(const SequencesArgs &q, int64_t tokens, bool lists) {
  return q.tokens > 0 && q.tokens <= tokens && q.sequences > 0 && q.sequences <= (lists ? kMaxWaves : kSmall);
}

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace

// Sets the workspace's pointers and returns its bytes.
size_t policy_workspace(PolicyArgs &a, void *base) {
  char *p = static_cast<char *>(base);
  size_t at = 0;
  a.share = reinterpret_cast<double *>(p + at);
  at += round256((size_t)a.seq.sequences * sizeof(double));
  a.mean_delta = reinterpret_cast<float *>(p + at);
  if (a.sequence_ratio) at += round256((size_t)a.seq.sequences * sizeof(float));
  a.part = reinterpret_cast<double *>(p + at);
  at += (size_t)kMaxGroups * (1 + kPolicySums) * sizeof(double);
  return at;
}

namespace {

// The workgroups of a step that sums sequences.
template <int T, int W>
int sequence_groups(const SequencesArgs &q) {
  return groups_of(q.sequences, W ? T / W : 1);
}

// Calls f(T, W) as constants for the sequences' mean length.  Policy passes over 2^19 tokens, us: length 64
// 17.6 by 8 lanes, 18.9 by 64; 128 18.2 and 16.9; 256 16.1 by 64 lanes, 17.9 by 256 threads; 512 17.2 and 16.4; over
// 2^20 tokens length 2048 20.6 by 256 threads, 21.4 by 1024; 4096 24.8 and 20.9.  The mean does not see one long
// sequence among short ones, which is walked by the lanes of a short one, in turn: 4095 of 64 tokens and one of 32768
// take 69 us (even ones 14), 511 of 2048 and one of 131072 42 (17), 32767 of 32 and one of 2^20 18 ms (31 us).
template <class F>
void by_length(const SequencesArgs &q, F f) {
  const int64_t mean = q.sequences ? q.tokens / q.sequences : 0;
  if (mean <= 64) f(std::integral_constant<int, kThreads>(), std::integral_constant<int, 8>());
  else if (mean <= 384) f(std::integral_constant<int, kThreads>(), std::integral_constant<int, 64>());
  else if (mean <= 2048) f(std::integral_constant<int, kThreads>(), std::integral_constant<int, 0>());
  else f(std::integral_constant<int, kSmall>(), std::integral_constant<int, 0>());
}

template <bool RATIO>
int policy_sums(const PolicyArgs &a, Counts *counted, hipStream_t s) {
  int groups = 0;
  by_length(a.seq, [&](auto t, auto w) {
    groups = sequence_groups<t(), w()>(a.seq);
    if (groups) hipLaunchKernelGGL((policy_sequences_kernel<t(), w(), RATIO>), dim3(groups), dim3(t()), 0, s, a, counted);
  });
  return groups;
}

template <int W>
void policy_small(const PolicyArgs &a, Counts *counted, double *part, hipStream_t s) {
  if (a.sequence_ratio) hipLaunchKernelGGL((policy_small_kernel<W, true>), dim3(1), dim3(kSmall), 0, s, a, counted, part);
  else hipLaunchKernelGGL((policy_small_kernel<W, false>), dim3(1), dim3(kSmall), 0, s, a, counted, part);
}

// Calls f(T, BY_SEQUENCE, workgroups, chunks) for the preference loss's step over the tokens.  Passes over
// 2^20 tokens, us: length 300 17.2 in tiles of all tokens, 18.3 by sequence; 600 17.3 and 16.1; 2048 15.7 and 13.8.
// The policy loss, whose tokens take longer than the search for their sequences, takes tiles (600: 22.3 and 26.3;
// 2048: 21.0 and 20.5; 8192: 20.8 and 22.1).  Chunks are those of the mean length, so that a long sequence among short
// ones is left to few workgroups; its sums take longer still (see by_length).
constexpr int kSequenceThreads = 512;
template <class F>
void by_tiles(const SequencesArgs &q, F f) {
  const int64_t mean = q.tokens / q.sequences, tile = kSequenceThreads * kVector;
  if (mean <= 512) {
    f(std::integral_constant<int, kThreads>(), std::false_type(), groups_of(q.tokens, kThreads * kVector), 0);
  } else {
    const int64_t chunks = (mean + tile - 1) / tile;
    f(std::integral_constant<int, kSequenceThreads>(), std::true_type(), groups_of(q.sequences * chunks, 1), (int)chunks);
  }
}

bool short_sequences(const SequencesArgs &q) { return q.sequences == 0 || q.tokens / q.sequences <= 64; }

}  // namespace

hipError_t launch_policy(const PolicyArgs &a, hipStream_t s) {
  Counts *counted = reinterpret_cast<Counts *>(a.part);
  double *part = a.part + kMaxGroups;
  if (a.seq.sequences == 0 && !a.stats) return hipSuccess;
  if (small_call(a.seq, kSmallPolicy, false)) {
    if (short_sequences(a.seq)) policy_small<8>(a, counted, part, s);
    else policy_small<64>(a, counted, part, s);
    return hipGetLastError();
  }
  const int counters = a.sequence_ratio ? policy_sums<true>(a, counted, s) : policy_sums<false>(a, counted, s);
  const int groups = counters ? groups_of(a.seq.tokens, kThreads * kVector) : 0;
  if (groups)
    hipLaunchKernelGGL(policy_tokens_kernel, dim3(groups), dim3(kThreads), 0, s, a, counted, counters, part);
  if (a.stats)
    hipLaunchKernelGGL(policy_fold_kernel, dim3(1), dim3(kThreads), 0, s, a, counted, counters, part, groups);
  return hipGetLastError();
}

size_t preference_workspace(PreferenceArgs &a, void *base) {
  char *p = static_cast<char *>(base);
  size_t at = 0;
  a.count = reinterpret_cast<uint32_t *>(p + at);
  at += round256((size_t)a.seq.sequences * sizeof(uint32_t));
  a.value = reinterpret_cast<double *>(p + at);
  at += round256((size_t)a.seq.sequences * sizeof(double));
  a.slope = reinterpret_cast<double *>(p + at);
  at += round256((size_t)a.seq.sequences * sizeof(double));
  a.part = reinterpret_cast<double *>(p + at);
  at += (size_t)kMaxGroups * kPairSums * sizeof(double);
  return at;
}

hipError_t launch_preference(const PreferenceArgs &a, hipStream_t s) {
  if (a.seq.sequences == 0 && a.pairs == 0 && !a.stats) return hipSuccess;
  if (small_call(a.seq, kSmallPreference, a.chosen != nullptr)) {
    if (short_sequences(a.seq)) hipLaunchKernelGGL(preference_small_kernel<8>, dim3(1), dim3(kSmall), 0, s, a, a.part);
    else hipLaunchKernelGGL(preference_small_kernel<64>, dim3(1), dim3(kSmall), 0, s, a, a.part);
    return hipGetLastError();
  }
  int sequences = 0;
  by_length(a.seq, [&](auto t, auto w) {
    sequences = sequence_groups<t(), w()>(a.seq);
    if (sequences) hipLaunchKernelGGL((preference_sequences_kernel<t(), w()>), dim3(sequences), dim3(t()), 0, s, a);
  });
  const int pairs = groups_of(a.pairs, kThreads);
  const int lists = a.chosen && a.dlogp ? groups_of(a.seq.sequences, kWaves) : 0;
  if (pairs + lists)
    hipLaunchKernelGGL(preference_pairs_kernel, dim3(pairs + lists), dim3(kThreads), 0, s, a, pairs, a.part);
  if (a.dlogp && sequences && a.seq.tokens > 0)
    by_tiles(a.seq, [&](auto t, auto by_sequence, int g, int chunks) {
      hipLaunchKernelGGL((preference_tokens_kernel<t(), by_sequence()>), dim3(g), dim3(t()), 0, s, a, chunks, a.part, pairs);
    });
  else if (a.stats)
    hipLaunchKernelGGL((preference_tokens_kernel<kThreads, false>), dim3(1), dim3(kThreads), 0, s, a, 0, a.part, pairs);
  return hipGetLastError();
}

}  // namespace hilore
