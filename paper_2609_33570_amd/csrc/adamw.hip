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
// written, g read), 10 B with bf16 parameters and gradients and 8-bit states.  The step runs at
// 5.0 to 5.3 TB/s of those bytes (40M fp32 elements 210 us, 233M with 8-bit states 440 to 463, kernel
// times under a trace on different machines), the norm at 4.0.
#include "device_common.hpp"
#include "hilore_internal.hpp"

// Every rounding step is the one written: no implicit fused multiply-add.
#pragma clang fp contract(off)

namespace hilore {
namespace {

constexpr int kThreads = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// A lane's E consecutive elements as they lie in memory.  With `n` < E of them the others
// read as 0 and are not written (FULL: n >= E is known).
template <typename T, int E>
struct Lane {
  static constexpr int kBytes = E * (int)sizeof(T), kWords = kBytes / 4;
  uint32_t w[kWords];
};

template <bool FULL, typename T, int E>
__device__ __forceinline__ void load_lane(Lane<T, E> &v, const T *p, int64_t i, int n) {
  using L = Lane<T, E>;
  if (FULL || n >= E) {
    if constexpr (L::kBytes == 4) {
      v.w[0] = *reinterpret_cast<const uint32_t *>(p + i);
    } else if constexpr (L::kBytes == 8) {
      const u32x2 a = *reinterpret_cast<const u32x2 *>(p + i);
      v.w[0] = a.x; v.w[1] = a.y;
    } else {
#pragma unroll
      for (int k = 0; k < L::kBytes / 16; ++k) {
        const u32x4 a = *(reinterpret_cast<const u32x4 *>(p + i) + k);
        v.w[4 * k] = a.x; v.w[4 * k + 1] = a.y; v.w[4 * k + 2] = a.z; v.w[4 * k + 3] = a.w;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < L::kWords; ++k) v.w[k] = 0;
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (k < n) {
        constexpr int kPer = 4 / (int)sizeof(T);
        if constexpr (kPer == 1) v.w[k] = __builtin_bit_cast(uint32_t, p[i + k]);
        else v.w[k / kPer] |= (uint32_t)p[i + k] << (8 * (int)sizeof(T) * (k % kPer));
      }
  }
}

template <bool FULL, typename T, int E>
__device__ __forceinline__ void store_lane(const Lane<T, E> &v, T *p, int64_t i, int n) {
  using L = Lane<T, E>;
  if (FULL || n >= E) {
    if constexpr (L::kBytes == 4) {
      *reinterpret_cast<uint32_t *>(p + i) = v.w[0];
    } else if constexpr (L::kBytes == 8) {
      *reinterpret_cast<u32x2 *>(p + i) = u32x2{v.w[0], v.w[1]};
    } else {
#pragma unroll
      for (int k = 0; k < L::kBytes / 16; ++k)
        *(reinterpret_cast<u32x4 *>(p + i) + k) =
            u32x4{v.w[4 * k], v.w[4 * k + 1], v.w[4 * k + 2], v.w[4 * k + 3]};
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (k < n) {
        constexpr int kPer = 4 / (int)sizeof(T);
        if constexpr (kPer == 1) p[i + k] = __builtin_bit_cast(T, v.w[k]);
        else p[i + k] = (T)(v.w[k / kPer] >> (8 * (int)sizeof(T) * (k % kPer)));
      }
  }
}

template <int E>
__device__ __forceinline__ void values(const Lane<float, E> &l, float v[E]) {
#pragma unroll
  for (int k = 0; k < E; ++k) v[k] = __uint_as_float(l.w[k]);
}

template <int E>
__device__ __forceinline__ void values(const Lane<uint16_t, E> &l, float v[E]) {
#pragma unroll
  for (int k = 0; k < E; k += 2) {
    v[k] = bf16_lo(l.w[k / 2]);
    v[k + 1] = bf16_hi(l.w[k / 2]);
  }
}

// E4M3FN codes times their block's scale.
template <int E>
__device__ __forceinline__ void decode(const Lane<uint8_t, E> &l, float s, float v[E]) {
#pragma unroll
  for (int k = 0; k < E; k += 4) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)l.w[k / 4], false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)l.w[k / 4], true);
    v[k] = a.x * s; v[k + 1] = a.y * s; v[k + 2] = b.x * s; v[k + 3] = b.y * s;
  }
}

// Codes of a block's values (E of 256 in each lane) with 16 random bits each, and the block's
// scale.  KEEP: x >= 0, and what is above zero stays above it.  BIG: blocks up to fp32's
// largest; else up to 2^12, where 448 / amax 2^-120 is a normal number.  The two differ by a
// rounding of products below 2^-126, 2^-20 of the least code's spacing.
template <bool KEEP, bool BIG, int E>
__device__ __forceinline__ void encode(const float x[E], const uint32_t bits[E], float amax,
                                       Lane<uint8_t, E> &out, float &scale) {
  const bool none = amax < 0x1p-64f;
  float inv;
  if constexpr (BIG) {
    inv = 1.0f / amax;
  } else {  // one Newton step after the hardware's: 1 / amax to the bit for every fp32 in [2^-64, 2^12]
    inv = __builtin_amdgcn_rcpf(amax);
    inv = fmaf(fmaf(-amax, inv, 1.0f), inv, inv);
  }
  scale = none ? 0.0f : amax * (1.0f / 448.0f);
  const float r = none ? 0.0f : (448.0f * inv) * (BIG ? 1.0f : 0x1p-120f);
  const uint32_t least = none ? 0u : 1u;
#pragma unroll
  for (int k = 0; k < E; k += 4) {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y = fabsf(x[k + e]) * r;
      if constexpr (BIG) y *= 0x1p-120f;
      const uint32_t u = ((bits[k + e] << 4) + __float_as_uint(y)) >> 20;
      const uint32_t low = KEEP ? min(__float_as_uint(x[k + e]), least) : 0u;
      c[e] = max(min(u, 0x7Eu), low);
    }
    uint32_t w = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    if constexpr (!KEEP) {  // the signs: the four upper bytes' top bits
      const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(x[k + 1]), __float_as_uint(x[k]), 0x0C0C0703u);
      const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(x[k + 3]), __float_as_uint(x[k + 2]), 0x07030C0Cu);
      w |= (lo | hi) & 0x80808080u;
    }
    out.w[k / 4] = w;
  }
}

template <int E>
__device__ __forceinline__ float block_amax(const float x[E]) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < E; ++k) top = max(top, __float_as_uint(fabsf(x[k])));
  return __uint_as_float(lanes_max_u32<256 / E>(top));
}

// Roots of v >= 0: a Newton step after the hardware's reciprocal root, which is for normal
// numbers (the library's sqrtf, three times as long, for the others).  Over all normal numbers it is
// sqrtf but for 0.08 %, by one unit in the last place, none of them in [2^-64, 2^13).
template <int E>
__device__ __forceinline__ void roots(const float v[E], float r[E]) {
  bool other = false;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(v[k], 0x1p-126f));
    const float s = v[k] * y;
    r[k] = fmaf(fmaf(-s, s, v[k]), 0.5f * y, s);
    other |= __builtin_amdgcn_classf(v[k], 0x3 | 0x200 | 0x80 | 0x10);  // NaN, infinity, subnormal
  }
  if (other) {
#pragma unroll
    for (int k = 0; k < E; ++k) r[k] = sqrtf(v[k]);
  }
}

struct AdamwTensor {
  float *p;
  uint16_t *p16;
  const void *grad;
  void *m, *v;
  float *m_scales, *v_scales;
  int64_t n;
  float step_size, decay;
  uint32_t key_state, key_param;
  int grad16;
};

struct Scalars {
  float beta1, one_beta1, beta2, one_beta2, eps, inv_sqrt_c2, clip;
};

// The elements that a workgroup takes at once: 4 a lane with 32-bit states, 8 with 8-bit
// ones (a block is then half a wave), which makes the narrow operands' loads 8 and 16 bytes.
template <bool EIGHT, bool GRAD16, int PARAM>
struct Piece {
  static constexpr int E = EIGHT ? 8 : 4;
  Lane<float, E> p, m, v;
  Lane<uint16_t, E> p16;
  Lane<float, E> g;
  Lane<uint16_t, E> g16;
  Lane<uint8_t, E> mc, vc;
  float ms, vs;
};

template <bool FULL, bool EIGHT, bool GRAD16, int PARAM>
__device__ __forceinline__ void load_piece(Piece<EIGHT, GRAD16, PARAM> &x, const AdamwTensor &t,
                                           int64_t i, int n) {
  if constexpr (PARAM == 2) load_lane<FULL>(x.p16, (const uint16_t *)t.p16, i, n);
  else load_lane<FULL>(x.p, (const float *)t.p, i, n);
  if constexpr (GRAD16) load_lane<FULL>(x.g16, static_cast<const uint16_t *>(t.grad), i, n);
  else load_lane<FULL>(x.g, static_cast<const float *>(t.grad), i, n);
  if constexpr (EIGHT) {
    load_lane<FULL>(x.mc, static_cast<const uint8_t *>(t.m), i, n);
    load_lane<FULL>(x.vc, static_cast<const uint8_t *>(t.v), i, n);
    // a lane past the end still takes part in its block's largest value: with zeros, whatever
    // another block's scale may be
    x.ms = x.vs = 0.0f;
    if (FULL || n > 0) {
      x.ms = t.m_scales[i / kAdamwBlock];
      x.vs = t.v_scales[i / kAdamwBlock];
    }
  } else {
    load_lane<FULL>(x.m, static_cast<const float *>(t.m), i, n);
    load_lane<FULL>(x.v, static_cast<const float *>(t.v), i, n);
  }
}

// One step of a piece.  PARAM: 0 fp32, 1 fp32 with a bf16 copy, 2 bf16.
template <bool FULL, bool EIGHT, bool GRAD16, int PARAM>
__device__ __forceinline__ void step_piece(Piece<EIGHT, GRAD16, PARAM> &x, const AdamwTensor &t,
                                           int64_t i, int n, const Scalars &s) {
  constexpr int E = Piece<EIGHT, GRAD16, PARAM>::E;
  float p[E], g[E], m[E], v[E], r[E];
  if constexpr (PARAM == 2) values(x.p16, p);
  else values(x.p, p);
  if constexpr (GRAD16) values(x.g16, g);
  else values(x.g, g);
  if constexpr (EIGHT) {
    decode(x.mc, x.ms, m);
    decode(x.vc, x.vs, r);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = r[k] * r[k];
  } else {
    values(x.m, m);
    values(x.v, v);
  }
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float gk = g[k] * s.clip;
    m[k] = s.beta1 * m[k] + s.one_beta1 * gk;
    v[k] = s.beta2 * v[k] + s.one_beta2 * (gk * gk);
  }
  roots<E>(v, r);
#pragma unroll
  for (int k = 0; k < E; ++k)  // rcp is within 1 ulp, 2^-23 of the step that is taken from p;
                               // eps keeps its operand a normal number
    p[k] = p[k] * t.decay -
           (t.step_size * m[k]) * __builtin_amdgcn_rcpf(r[k] * s.inv_sqrt_c2 + s.eps);
  if constexpr (EIGHT) {
    uint32_t lo[E], hi[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const uint32_t w = mix32((uint32_t)(i + k) ^ t.key_state);
      lo[k] = w & 0xFFFFu;
      hi[k] = w >> 16;
    }
    const float am = block_amax<E>(m), ar = block_amax<E>(r);
    if (__builtin_expect(__any(!(am <= 0x1p12f) || !(ar <= 0x1p12f)), 0)) {
      encode<false, true, E>(m, lo, am, x.mc, x.ms);
      encode<true, true, E>(r, hi, ar, x.vc, x.vs);
    } else {
      encode<false, false, E>(m, lo, am, x.mc, x.ms);
      encode<true, false, E>(r, hi, ar, x.vc, x.vs);
    }
    store_lane<FULL>(x.mc, static_cast<uint8_t *>(t.m), i, n);
    store_lane<FULL>(x.vc, static_cast<uint8_t *>(t.v), i, n);
    if ((threadIdx.x & (kAdamwBlock / E - 1)) == 0 && (FULL || n > 0)) {
      t.m_scales[i / kAdamwBlock] = x.ms;
      t.v_scales[i / kAdamwBlock] = x.vs;
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) {
      x.m.w[k] = __float_as_uint(m[k]);
      x.v.w[k] = __float_as_uint(v[k]);
    }
    store_lane<FULL>(x.m, static_cast<float *>(t.m), i, n);
    store_lane<FULL>(x.v, static_cast<float *>(t.v), i, n);
  }
  if constexpr (PARAM != 2) {
#pragma unroll
    for (int k = 0; k < E; ++k) x.p.w[k] = __float_as_uint(p[k]);
    store_lane<FULL>(x.p, t.p, i, n);
  }
  if constexpr (PARAM == 1) {
#pragma unroll
    for (int k = 0; k < E; k += 2) x.p16.w[k / 2] = pack_bf16(p[k], p[k + 1]);
    store_lane<FULL>(x.p16, t.p16, i, n);
  }
  if constexpr (PARAM == 2) {
    uint32_t w[E];
    bool other = false;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      w[k] = __float_as_uint(p[k]) + (mix32((uint32_t)(i + k) ^ t.key_param) & 0xFFFFu);
      other |= __builtin_amdgcn_classf(p[k], 0x3 | 0x200 | 0x4);
    }
    if (other) {  // NaN and infinity have no bits to round
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (__builtin_amdgcn_classf(p[k], 0x3 | 0x200 | 0x4))
          w[k] = __float_as_uint(p[k]) | (p[k] != p[k] ? 0x400000u : 0u);
    }
#pragma unroll
    for (int k = 0; k < E; k += 2) x.p16.w[k / 2] = __builtin_amdgcn_perm(w[k + 1], w[k], 0x07060302u);
    store_lane<FULL>(x.p16, t.p16, i, n);
  }
}

// One chunk of one tensor: every load goes out before the first step.
template <bool FULL, bool EIGHT, bool GRAD16, int PARAM>
__device__ __forceinline__ void step_chunk(const AdamwTensor &t, int64_t begin, const Scalars &s) {
  constexpr int E = Piece<EIGHT, GRAD16, PARAM>::E;
  constexpr int kPieces = (int)kAdamwChunk / kThreads / E;
  Piece<EIGHT, GRAD16, PARAM> x[kPieces];
  const int64_t first = begin + (int64_t)threadIdx.x * E;
  const auto count = [&](int64_t i) {
    const int64_t left = t.n - i;
    return left >= E ? E : left > 0 ? (int)left : 0;
  };
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t i = first + k * kThreads * E;
    load_piece<FULL>(x[k], t, i, FULL ? E : count(i));
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int64_t i = first + k * kThreads * E;
    step_piece<FULL>(x[k], t, i, FULL ? E : count(i), s);
  }
}

template <bool EIGHT, bool GRAD16, int PARAM>
__device__ __forceinline__ void step_any(const AdamwTensor &t, int64_t begin, const Scalars &s) {
  if (begin + kAdamwChunk <= t.n) step_chunk<true, EIGHT, GRAD16, PARAM>(t, begin, s);
  else step_chunk<false, EIGHT, GRAD16, PARAM>(t, begin, s);
}

// Tensor of workgroup `b`: the last whose chunks begin at or before it (unused entries of
// `begin` are 2^32 - 1; one without elements begins where the next one does).  Every lane looks
// at one tensor of 64, so there is one load's wait, where a binary search has one a step (233M
// elements, 8 bit: 560 -> 430 us with the step's instructions cut; by unrolled scalar loads 463).
template <int N>
__device__ __forceinline__ int tensor_of(const uint32_t *begin, int count, uint32_t b) {
  int before = 0;
#pragma unroll
  for (int j = 0; j < N; j += kWave) {
    const int i = j + (int)(threadIdx.x & 63);
    const uint32_t first = begin[i < count ? i : 0];
    before += __popcll(__ballot((i < count) & (first <= b)));
  }
  return before - 1;
}

// Key of the random bits of tensor `index` of a call.
__device__ __forceinline__ uint32_t adamw_key(uint32_t seed, int index, uint32_t salt) {
  return mix32(seed + 0x9E3779B1u * (uint32_t)(index + 1) + salt);
}

// Global memory, not whatever address space: a pointer made of words says nothing of it, and the
// accesses would be flat ones (233M elements, 8 bit: 594 us a step with its norm, so 562).
template <typename T>
__device__ __forceinline__ T *global_at(uint64_t a) {
  return (T *)(__attribute__((address_space(1))) T *)a;
}

// Tensor k of a launch; its whole record is read at once (a shorter one with some of the words
// that follow it).
__device__ __forceinline__ AdamwTensor tensor_at(const AdamwBatch &a, int k, float clip) {
  const uint32_t *rec = a.w + a.cap + k * a.stride;
  uint32_t r[kAdamwRecord];
#pragma unroll
  for (int i = 0; i < kAdamwRecord; ++i) r[i] = rec[i];
  // all of them in one wait: each load on its own is a trip to the host's memory
  asm volatile("" ::"s"(r[0]), "s"(r[1]), "s"(r[2]), "s"(r[3]), "s"(r[4]), "s"(r[5]), "s"(r[6]), "s"(r[7]),
               "s"(r[8]), "s"(r[9]), "s"(r[10]), "s"(r[11]), "s"(r[12]), "s"(r[13]), "s"(a.w[k]), "s"(a.eps),
               "s"(a.first), "s"(clip));
  const auto pointer = [](uint32_t low, uint32_t upper) { return (uint64_t)(upper & 0xFFFFu) << 32 | low; };
  const bool both = a.has_p && a.has_p16;
  const bool scales = a.stride > (both ? 11 : 9);
  const uint64_t param = pointer(r[6], r[5] >> 16), second = pointer(r[9], r[10]);
  const uint32_t low_m = both ? r[11] : r[9], low_v = both ? r[12] : r[10], upper = both ? r[13] : r[11];
  AdamwTensor t;
  t.p = global_at<float>(a.has_p ? param : 0);
  t.p16 = global_at<uint16_t>(both ? second : a.has_p ? 0 : param);
  t.grad = global_at<const uint8_t>(pointer(r[0] & ~15u, r[3]));
  t.grad16 = (int)(r[0] & 1u);
  t.m = global_at<uint8_t>(pointer(r[1], r[3] >> 16));
  t.v = global_at<uint8_t>(pointer(r[2], r[5]));
  t.m_scales = global_at<float>(scales ? pointer(low_m, upper) : 0);
  t.v_scales = global_at<float>(scales ? pointer(low_v, upper >> 16) : 0);
  t.n = (int64_t)r[4];
  t.step_size = __uint_as_float(r[7]);
  t.decay = __uint_as_float(r[8]);
  t.key_state = adamw_key(a.seed, a.first + k, 0u);
  t.key_param = adamw_key(a.seed, a.first + k, 0x3C6EF372u);
  return t;
}

__device__ const float kNoClip[2] = {0.0f, 1.0f};

// One kernel for all kinds, since the tensors of a launch may differ in kind; its registers are
// those of the kind of most operands.  Bounded to five waves a SIMD, with 20 of them spilled there (a
// step with its norm: 28 adapters in 8 bit 16.3 -> 14.0 us, 233M elements 564 -> 554).  By the tensors'
// packing into fewer launches, 343 of 215 elements: 85 -> 65 us, 392 adapters of 40M elements 304 -> 268.
__global__ __launch_bounds__(kThreads, 5) void adamw_kernel(const AdamwBatch a) {
  // a uniform load, asked for before the tensors' first chunks are there
  const uintptr_t norm = reinterpret_cast<uintptr_t>(a.norm ? a.norm : kNoClip);
  const float clip = reinterpret_cast<const __attribute__((address_space(4))) float *>(norm)[1];
  const int k = __builtin_amdgcn_readfirstlane(tensor_of<128>(a.w, a.cap, blockIdx.x));
  const AdamwTensor t = tensor_at(a, k, clip);
  const int64_t begin = ((int64_t)blockIdx.x - a.w[k]) * kAdamwChunk;
  if (clip != clip) return;  // NaN: the step is skipped
  const Scalars s = {a.beta1, a.one_beta1, a.beta2,
                     a.one_beta2, a.eps, a.inv_sqrt_c2, clip};
  const int param = t.p ? (t.p16 ? 1 : 0) : 2;
  const int kind = (t.m_scales ? 6 : 0) + (t.grad16 ? 3 : 0) + param;
  switch (kind) {
    case 0: return step_any<false, false, 0>(t, begin, s);
    case 1: return step_any<false, false, 1>(t, begin, s);
    case 2: return step_any<false, false, 2>(t, begin, s);
    case 3: return step_any<false, true, 0>(t, begin, s);
    case 4: return step_any<false, true, 1>(t, begin, s);
    case 5: return step_any<false, true, 2>(t, begin, s);
    case 6: return step_any<true, false, 0>(t, begin, s);
    case 7: return step_any<true, false, 1>(t, begin, s);
    case 8: return step_any<true, false, 2>(t, begin, s);
    case 9: return step_any<true, true, 0>(t, begin, s);
    case 10: return step_any<true, true, 1>(t, begin, s);
    default: return step_any<true, true, 2>(t, begin, s);
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

// Sum of squares of one chunk of one gradient (16 KB; with 32 KB and 64 KB a gradient of 3 MB takes
// 5.5 and 7.2 us instead of 4.2, one of 466 MB 121 and 123 instead of 118), in fp64 (an fp32 square would
// overflow from 2^64 on and vanish below 2^-75).  All of a thread's loads go out first.
template <bool FULL, typename T>
__device__ __forceinline__ double chunk_squares(const T *g, int64_t n, int64_t begin) {
  constexpr int E = 16 / (int)sizeof(T), kLoads = (int)(kNormChunkBytes / kThreads / 16);
  Lane<T, E> x[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int64_t i = begin + (j * kThreads + (int)threadIdx.x) * E, left = n - i;
    load_lane<FULL>(x[j], g, i, left >= E ? E : left > 0 ? (int)left : 0);
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    float v[E];
    values(x[j], v);
#pragma unroll
    for (int e = 0; e < E; ++e) sum = fma((double)v[e], (double)v[e], sum);
  }
  return sum;
}

__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const NormBatch a) {
  __shared__ double lds[kThreads / kWave];
  const int k = tensor_of<kNormPerLaunch>(a.begin, kNormPerLaunch, blockIdx.x);
  const uint32_t low = a.grad[k], upper = a.upper[k / 2], n32 = a.n[k], before = a.begin[k];
  asm volatile("" ::"s"(low), "s"(upper), "s"(n32), "s"(before), "s"(a.part));  // in one wait
  const bool grad16 = low & 1u;
  const uint64_t at = (uint64_t)(upper >> (16 * (k & 1)) & 0xFFFFu) << 32 | (low & ~15u);
  const int64_t chunk = kNormChunkBytes / (grad16 ? 2 : 4);  // elements
  const int64_t begin = ((int64_t)blockIdx.x - before) * chunk, n = n32;
  const bool full = begin + chunk <= n;
  const float *g = global_at<const float>(at);
  const uint16_t *g16 = global_at<const uint16_t>(at);
  double sum = grad16 ? (full ? chunk_squares<true>(g16, n, begin) : chunk_squares<false>(g16, n, begin))
                        : (full ? chunk_squares<true>(g, n, begin) : chunk_squares<false>(g, n, begin));
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

constexpr int kFoldThreads = 1024;

__global__ __launch_bounds__(kFoldThreads) void norm_fold_kernel(const double *part, int64_t n,
                                                                 float max_norm, float *norm) {
  __shared__ double lds[kFoldThreads / kWave];
  double sum = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += kFoldThreads) sum += part[i];
  sum = group_sum(sum, lds);
  if (threadIdx.x == 0) {
    // The sum rounded to 24 bits, then fp32 operations (a 53-bit root of 24 bits rounds
    // to the same fp32 as theirs; fp32's exponents would not hold every sum).  These are the bits that
    // a trainer's own fp32 root, sum and quotient give on an exact sum, and the random rounding below
    // 8-bit states turns on single bits of the factor.  The roundings put the factor up to 3
    // units of 2^-24 from 64 bits (0.6 in the mean); one rounding at the end would put it 1 (0.36).
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
  hipLaunchKernelGGL(adamw_kernel, dim3(a.chunks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_norm_partial(const NormBatch &a, hipStream_t s) {
  hipLaunchKernelGGL(norm_partial_kernel, dim3(a.chunks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_norm_fold(const double *part, int64_t n, float max_norm, float *norm,
                            hipStream_t s) {
  hipLaunchKernelGGL(norm_fold_kernel, dim3(1), dim3(kFoldThreads), 0, s, part, n, max_norm, norm);
  return hipGetLastError();
}

}  // namespace hilore
