// Clipped policy loss and preference loss with their gradients, on gfx950.
//
// Small against the logits' passes: 13 to 30 B a token, so that the launches and their latencies
// count up to some 10^5 tokens.  Three launches each: sums by sequence, then the tokens (policy)
// or the pairs and then the tokens (preference), with partial sums of each workgroup that the next launch adds
// up in a fixed order, in fp64.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kMaxGroups = 1024;  // workgroups of a launch, each with partial sums
constexpr int kMaxSums = 8;

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

// N sums over the workgroup, all threads receiving them.  `lds` has room for N sums of each wave.
template <int N>
__device__ __forceinline__ void group_sums(double (&v)[N], double (*lds)[kMaxSums]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  const int waves = blockDim.x >> 6;
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

// The sums of `groups` workgroups' N partial sums, by this workgroup, in a fixed order.
template <int N>
__device__ __forceinline__ void sum_parts(const double *part, int groups, double (&v)[N], double (*lds)[kMaxSums]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.0;
  for (int g = threadIdx.x; g < groups; g += blockDim.x)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += part[(int64_t)g * N + k];
  group_sums<N>(v, lds);
}

__device__ __forceinline__ int64_t clamped(int64_t x, int64_t most) { return x < 0 ? 0 : x > most ? most : x; }

// Tokens [begin, end) of a sequence.
__device__ __forceinline__ void bounds(const SequencesArgs &q, int64_t s, int64_t &begin, int64_t &end) {
  if (q.offsets) {
    begin = clamped(q.offsets[s], q.tokens);
    end = clamped(q.offsets[s + 1], q.tokens);
  } else {
    begin = s * q.length;
    end = begin + q.length;
  }
}

// The last sequence in [lo, hi) that begins at token t or before it, lo - 1 where none does.
__device__ __forceinline__ int64_t begins_before(const SequencesArgs &q, int64_t t, int64_t lo, int64_t hi) {
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    if (q.offsets[mid] <= t) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// Sequences that a workgroup's tokens [first, first + n) can be of: found once, then each token
// searches among them.  Two values in LDS.
__device__ __forceinline__ void sequence_range(const SequencesArgs &q, int64_t first, int64_t n, int64_t *lds) {
  __syncthreads();
  if (threadIdx.x < 2) {
    const int64_t t = threadIdx.x == 0 ? first : first + n - 1;
    lds[threadIdx.x] = begins_before(q, t, 0, q.sequences);
  }
  __syncthreads();
}

// The sequence of a token, -1 where it is in none.
__device__ __forceinline__ int64_t sequence_of(const SequencesArgs &q, int64_t t, const int64_t *range) {
  if (!q.offsets) return (int64_t)((uint32_t)t / (uint32_t)q.length);
  const int64_t lo = range[0] < 0 ? 0 : range[0];
  const int64_t s = begins_before(q, t, lo, range[1] + 1);
  return s >= 0 && s < q.sequences && q.offsets[s] <= t && t < q.offsets[s + 1] ? s : -1;
}

__device__ __forceinline__ bool valid_token(const SequencesArgs &q, int64_t t) { return !q.mask || q.mask[t] != 0; }

// ----------------------------------------------------------------- policy --
// Valid tokens of each sequence and, for the sequences' ratios, their mean log ratio; partial
// sums of the valid tokens and of the sequences that have any.
__global__ __launch_bounds__(1024) void policy_sequences_kernel(const PolicyArgs a, double *part) {
  __shared__ double lds[16][kMaxSums];
  double total[2] = {0.0, 0.0};
  for (int64_t s = blockIdx.x; s < a.seq.sequences; s += gridDim.x) {
    int64_t begin, end;
    bounds(a.seq, s, begin, end);
    double sum[2] = {0.0, 0.0};
    for (int64_t t = begin + threadIdx.x; t < end; t += blockDim.x) {
      if (!valid_token(a.seq, t)) continue;
      sum[0] += 1.0;
      if (a.sequence_ratio) sum[1] += (double)(a.logp[t] - a.old[t]);
    }
    group_sums<2>(sum, lds);
    total[0] += sum[0];
    total[1] += sum[0] > 0.0 ? 1.0 : 0.0;
    if (threadIdx.x == 0) {
      a.count[s] = (uint32_t)sum[0];
      if (a.sequence_ratio) a.mean_delta[s] = sum[0] > 0.0 ? (float)(sum[1] / sum[0]) : 0.0f;
    }
  }
  if (threadIdx.x == 0) {
    part[blockIdx.x * 2] = total[0];
    part[blockIdx.x * 2 + 1] = total[1];
  }
}

constexpr int kPolicySums = 6;  // policy, kl, entropy, loss, clipped, ratio

struct TokenLoss {
  float loss, policy, kl, dlogp, ratio;
  uint8_t flags;
};

__device__ __forceinline__ TokenLoss token_loss(const PolicyArgs &a, float delta, float adv, float x, float entropy) {
  TokenLoss o;
  o.ratio = expf(delta);
  bool chi = adv >= 0.0f ? delta <= a.log_high : delta >= a.log_low;
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
      o.kl = e + x;
      dkl = -e;
    }
    o.loss += a.beta * o.kl;
    slope += a.beta * dkl;
  }
  if (a.entropy) o.loss -= a.bonus * entropy;
  o.dlogp = slope;
  o.flags = (uint8_t)((chi ? 1 : 0) | (!chi && adv != 0.0f ? 2 : 0));
  return o;
}

__global__ __launch_bounds__(kThreads) void policy_tokens_kernel(const PolicyArgs a, const double *counted, int counters,
                                                                 double *part) {
  __shared__ double lds[kWaves][kMaxSums];
  __shared__ int64_t range[2];
  double n[2];
  sum_parts<2>(counted, counters, n, lds);
  const double norm = a.n_norm > 0.0 ? a.n_norm : a.sequence_mean ? n[1] : n[0];
  double sum[kPolicySums] = {};
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < a.seq.tokens; first += (int64_t)gridDim.x * kThreads) {
    if (a.seq.offsets) {
      const int64_t left = a.seq.tokens - first;
      sequence_range(a.seq, first, left < kThreads ? left : kThreads, range);
    }
    const int64_t t = first + threadIdx.x;
    if (t >= a.seq.tokens) continue;
    const int64_t s = sequence_of(a.seq, t, range);
    if (s < 0) continue;
    if (!valid_token(a.seq, t)) {
      if (a.dlogp) a.dlogp[t] = 0.0f;
      if (a.dentropy) a.dentropy[t] = 0.0f;
      if (a.token_loss) a.token_loss[t] = 0.0f;
      if (a.flags) a.flags[t] = 0;
      continue;
    }
    const float delta = a.sequence_ratio ? a.mean_delta[s] : a.logp[t] - a.old[t];
    const float x = a.kl ? a.logp[t] - a.ref[t] : 0.0f, h = a.entropy ? a.entropy[t] : 0.0f;
    const TokenLoss o = token_loss(a, delta, a.adv[a.adv_per_token ? t : s], x, h);
    const double w64 = 1.0 / (a.sequence_mean ? norm * (double)a.count[s] : norm);
    const float w = (float)w64;
    if (a.dlogp) a.dlogp[t] = w * o.dlogp;
    if (a.dentropy) a.dentropy[t] = -a.bonus * w;
    if (a.token_loss) a.token_loss[t] = w * o.loss;
    if (a.flags) a.flags[t] = o.flags;
    sum[0] += w64 * (double)o.policy;
    sum[1] += w64 * (double)o.kl;
    sum[2] += w64 * (double)h;
    sum[3] += w64 * (double)o.loss;
    sum[4] += o.flags >> 1;
    sum[5] += (double)o.ratio;
  }
  if (!a.stats) return;
  group_sums<kPolicySums>(sum, lds);
  if (threadIdx.x == 0)
    for (int k = 0; k < kPolicySums; ++k) part[(int64_t)blockIdx.x * kPolicySums + k] = sum[k];
}

__global__ __launch_bounds__(kThreads) void policy_fold_kernel(const PolicyArgs a, const double *counted, int counters,
                                                               const double *part, int groups) {
  __shared__ double lds[kWaves][kMaxSums];
  double n[2], v[kPolicySums];
  sum_parts<2>(counted, counters, n, lds);
  sum_parts<kPolicySums>(part, groups, v, lds);
  if (threadIdx.x != 0) return;
  const double each = n[0] > 0.0 ? n[0] : 1.0;
  a.stats[0] = (float)v[3];
  a.stats[1] = (float)v[0];
  a.stats[2] = (float)v[1];
  a.stats[3] = (float)v[2];
  a.stats[4] = (float)(v[4] / each);
  a.stats[5] = (float)(v[5] / each);
  a.stats[6] = (float)n[0];
  a.stats[7] = (float)n[1];
}

// ------------------------------------------------------------- preference --
// Valid tokens of each sequence and the sum (or mean) of its log-ratios.
__global__ __launch_bounds__(1024) void preference_sequences_kernel(const PreferenceArgs a) {
  __shared__ double lds[16][kMaxSums];
  for (int64_t s = blockIdx.x; s < a.seq.sequences; s += gridDim.x) {
    int64_t begin, end;
    bounds(a.seq, s, begin, end);
    double sum[2] = {0.0, 0.0};
    for (int64_t t = begin + threadIdx.x; t < end; t += blockDim.x) {
      if (!valid_token(a.seq, t)) continue;
      sum[0] += 1.0;
      sum[1] += (double)(a.ref ? a.logp[t] - a.ref[t] : a.logp[t]);
    }
    group_sums<2>(sum, lds);
    if (threadIdx.x == 0) {
      const double value = a.length_mean && sum[0] > 0.0 ? sum[1] / sum[0] : sum[1];
      a.count[s] = (uint32_t)sum[0];
      a.value[s] = value;
      if (a.rewards) a.rewards[s] = (float)((double)a.beta * value);
    }
  }
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
    // softplus(-y) and softplus(y); their slopes are -sigmoid(-y) and sigmoid(y)
    p.loss = (1.0 - eps) * (fmax(-y, 0.0) + tail) + eps * (fmax(y, 0.0) + tail);
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

constexpr int kPairSums = 6;  // used, loss, h > 0, beta h, chosen and rejected rewards

// The first `pair_groups` workgroups take the pairs, with lists the others the sequences, a wave
// each, which reads the lists for its pairs.
__global__ __launch_bounds__(kThreads) void preference_pairs_kernel(const PreferenceArgs a, int pair_groups, double *part) {
  __shared__ double lds[kWaves][kMaxSums];
  if ((int)blockIdx.x < pair_groups) {
    double sum[kPairSums] = {};
    for (int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x; p < a.pairs; p += (int64_t)pair_groups * kThreads) {
      const Pair o = pair_loss(a, a.chosen ? a.chosen[p] : 2 * p, a.chosen ? a.rejected[p] : 2 * p + 1);
      if (a.pair_loss) a.pair_loss[p] = (float)o.loss;
      if (!a.chosen) {
        a.slope[2 * p] = o.slope;
        a.slope[2 * p + 1] = -o.slope;
      }
      sum[0] += o.used;
      sum[1] += o.loss;
      sum[2] += o.h > 0.0 ? 1.0 : 0.0;
      sum[3] += (double)a.beta * o.h;
      sum[4] += o.chosen;
      sum[5] += o.rejected;
    }
    group_sums<kPairSums>(sum, lds);
    if (threadIdx.x == 0)
      for (int k = 0; k < kPairSums; ++k) part[(int64_t)blockIdx.x * kPairSums + k] = sum[k];
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)(gridDim.x - pair_groups) * kWaves;
  for (int64_t s = (int64_t)(blockIdx.x - pair_groups) * kWaves + (threadIdx.x >> 6); s < a.seq.sequences; s += step) {
    double slope = 0.0;
    for (int64_t p = lane; p < a.pairs; p += kWave) {
      const int64_t win = a.chosen[p], lose = a.rejected[p];
      if (win != s && lose != s) continue;
      const double d = pair_loss(a, win, lose).slope;
      if (win == s) slope += d;
      if (lose == s) slope -= d;
    }
    slope = wave_sum(slope);
    if (lane == 0) a.slope[s] = slope;
  }
}

__global__ __launch_bounds__(kThreads) void preference_tokens_kernel(const PreferenceArgs a, const double *part, int groups) {
  __shared__ double lds[kWaves][kMaxSums];
  __shared__ int64_t range[2];
  double v[kPairSums];
  sum_parts<kPairSums>(part, groups, v, lds);
  // a pair with a number out of range makes v[0] NaN, and so all that follows
  const double norm = a.n_norm > 0.0 ? a.n_norm + 0.0 * v[0] : v[0] == 0.0 ? 1.0 : v[0];
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.stats) {
    for (int k = 1; k < kPairSums; ++k) a.stats[k - 1] = (float)(v[k] / norm);
    a.stats[5] = (float)v[0];
  }
  if (!a.dlogp) return;
  for (int64_t first = (int64_t)blockIdx.x * kThreads; first < a.seq.tokens; first += (int64_t)gridDim.x * kThreads) {
    if (a.seq.offsets) {
      const int64_t left = a.seq.tokens - first;
      sequence_range(a.seq, first, left < kThreads ? left : kThreads, range);
    }
    const int64_t t = first + threadIdx.x;
    if (t >= a.seq.tokens) continue;
    const int64_t s = sequence_of(a.seq, t, range);
    if (s < 0) continue;
    float d = 0.0f;
    if (valid_token(a.seq, t)) {
      // without lists the last of an odd number of sequences is in no pair
      const double slope = a.chosen || s < 2 * a.pairs ? a.slope[s] : 0.0;
      d = (float)(slope / (a.length_mean ? norm * (double)a.count[s] : norm));
    }
    a.dlogp[t] = d;
  }
}

int groups_of(int64_t work, int64_t each) {
  const int64_t need = (work + each - 1) / each;
  return (int)(need < kMaxGroups ? need : kMaxGroups);
}

// Threads of a workgroup that sums a sequence of `length` tokens on average.
int sequence_threads(int64_t length) { return length <= 64 ? 64 : length <= 1024 ? 256 : 1024; }

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

}  // namespace

// Sets the workspace's pointers and returns its bytes.
size_t policy_workspace(PolicyArgs &a, void *base) {
  char *p = static_cast<char *>(base);
  size_t at = 0;
  a.count = reinterpret_cast<uint32_t *>(p + at);
  at += round256((size_t)a.seq.sequences * sizeof(uint32_t));
  a.mean_delta = reinterpret_cast<float *>(p + at);
  if (a.sequence_ratio) at += round256((size_t)a.seq.sequences * sizeof(float));
  a.part = reinterpret_cast<double *>(p + at);
  at += (size_t)kMaxGroups * (2 + kPolicySums) * sizeof(double);
  return at;
}

hipError_t launch_policy(const PolicyArgs &a, hipStream_t s) {
  double *counted = a.part, *part = a.part + 2 * kMaxGroups;
  const int counters = groups_of(a.seq.sequences, 1), groups = groups_of(a.seq.tokens, kThreads);
  const int64_t mean = a.seq.sequences ? a.seq.tokens / a.seq.sequences : 0;
  if (!counters && !a.stats) return hipSuccess;
  if (counters)
    hipLaunchKernelGGL(policy_sequences_kernel, dim3(counters), dim3(sequence_threads(mean)), 0, s, a, counted);
  if (groups && counters)
    hipLaunchKernelGGL(policy_tokens_kernel, dim3(groups), dim3(kThreads), 0, s, a, counted, counters, part);
  if (a.stats)
    hipLaunchKernelGGL(policy_fold_kernel, dim3(1), dim3(kThreads), 0, s, a, counted, counters, part,
                       counters ? groups : 0);
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
  const int64_t mean = a.seq.sequences ? a.seq.tokens / a.seq.sequences : 0;
  const int sequences = groups_of(a.seq.sequences, 1), pairs = groups_of(a.pairs, kThreads);
  if (!sequences && !pairs && !a.stats) return hipSuccess;
  if (sequences)
    hipLaunchKernelGGL(preference_sequences_kernel, dim3(sequences), dim3(sequence_threads(mean)), 0, s, a);
  const int lists = a.chosen && a.dlogp ? groups_of(a.seq.sequences, kWaves) : 0;
  if (pairs + lists)
    hipLaunchKernelGGL(preference_pairs_kernel, dim3(pairs + lists), dim3(kThreads), 0, s, a, pairs, a.part);
  const int tokens = a.dlogp && sequences ? groups_of(a.seq.tokens, kThreads) : 0;
  if (tokens || a.stats)
    hipLaunchKernelGGL(preference_tokens_kernel, dim3(tokens ? tokens : 1), dim3(kThreads), 0, s, a, a.part, pairs);
  return hipGetLastError();
}

}  // namespace hilore
