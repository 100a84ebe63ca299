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
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// ------------------------------------------------------------- large tiles --
// 256 tokens x 256 channels per workgroup of 4 waves (2 x 2), each wave 128 x 128 =
// 4 x 4 blocks of v_mfma_i32_32x32x32_i8, one wave a SIMD.  Both operands have k
// contiguous, so they are copied to LDS as they are by the buffer unit (16-byte
// LDS-DMA loads, no registers) in stages of 64 k: [256 rows][64 B] each, 16-byte
// chunk g of row r at position g ^ (r / 2 % 4), which spreads the 8 rows that one
// cycle of a fragment read takes over all banks.  Four stages are in flight.
constexpr int kTile = 256, kStageK = 64, kTileThreads = 256;
constexpr int kStageBytes = kTile * kStageK;  // of one operand (16 KB)
constexpr int kStageLoads = 8;                // LDS-DMA instructions of a wave per stage
constexpr int kGroupT = 8;
constexpr uint32_t kOob = 0x80000000u;        // a buffer offset past every range: loads 0

typedef __attribute__((address_space(3))) void lds_void;

struct TileLoad {
  uint32_t a[4], b[4];  // byte offset of the lane's chunk in its row of each load, at k = 0
  int g16;              // its first k within a stage
};

// Stage k0 of both operands into `la`, `lb`: load r of wave w writes rows 64 w + 16 r ..
// + 15, lane l the chunk at position l % 4 of row l / 4.  Chunks past k read as 0.
__device__ __forceinline__ void dma_stage(__amdgpu_buffer_rsrc_t ra, __amdgpu_buffer_rsrc_t rb,
                                          const TileLoad &tl, int k0, int k, uint8_t *la,
                                          uint8_t *lb, int wave) {
  const uint32_t past = k0 + tl.g16 < k ? 0u : kOob;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void *)(la + (wave * 64 + r * 16) * kStageK),
                                             16, (int)((tl.a[r] + (uint32_t)k0) | past), 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void *)(lb + (wave * 64 + r * 16) * kStageK),
                                             16, (int)((tl.b[r] + (uint32_t)k0) | past), 0, 0, 0);
  }
}

// The workgroup's barrier after this wave's LDS reads and all but its N newest vector-memory
// operations.  (__syncthreads would wait for every LDS-DMA load in flight.)
template <int N>
__device__ __forceinline__ void barrier_but_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));  // lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

struct TileFrags {
  i32x4 a[2][4], b[2][4];  // fragments of even and odd k-steps
};

// Fragments of k-step KS (32 k) of a stage: lane l takes chunk 2 KS + l / 32 of row l % 32
// of each 32-row block; oa, ob: the lane's offset in block 0 at KS = 0 and at KS = 1.
template <int KS>
__device__ __forceinline__ void read_block(TileFrags &f, const uint8_t *la, const uint8_t *lb,
                                           const uint32_t (&oa)[2], const uint32_t (&ob)[2],
                                           int i) {
  f.a[KS][i] = *reinterpret_cast<const i32x4 *>(la + oa[KS] + i * 32 * kStageK);
  f.b[KS][i] = *reinterpret_cast<const i32x4 *>(lb + ob[KS] + i * 32 * kStageK);
}

// The 16 products of k-step KS with the reads of the other k-step's fragments (from la, lb).
template <int KS>
__device__ __forceinline__ void mma16(i32x16 (&acc)[4][4], TileFrags &f, const uint8_t *la,
                                      const uint8_t *lb, const uint32_t (&oa)[2],
                                      const uint32_t (&ob)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) read_block<KS ^ 1>(f, la, lb, oa, ob, i);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[KS][i], f.a[KS][j], acc[i][j], 0, 0, 0);
  }
}

// The other k-step's 8 fragment reads after the first 8 MFMAs, so that they are there when
// the next region begins; the loads, if any, after the last 8.
template <bool LOADS>
__device__ __forceinline__ void schedule16() {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // 1 MFMA
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // 1 LDS read
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // 1 LDS-DMA load
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Stage s in (cur_a, cur_b), its first fragments in f: the products of its two k-steps.
// Between them the wave waits for its own loads of stage s + 1, and one barrier says that
// they have landed for all waves and that nobody reads stage s from LDS any more; the second
// k-step's products then cover the loads of stage s + 4 into its place and the first
// fragment reads of stage s + 1.
__device__ __forceinline__ void tile_stage(i32x16 (&acc)[4][4], TileFrags &f, uint8_t *cur_a,
                                           uint8_t *cur_b, const uint8_t *nxt_a,
                                           const uint8_t *nxt_b, __amdgpu_buffer_rsrc_t ra,
                                           __amdgpu_buffer_rsrc_t rb, const TileLoad &tl, int k4,
                                           int k, const uint32_t (&oa)[2],
                                           const uint32_t (&ob)[2], int wave) {
  mma16<0>(acc, f, cur_a, cur_b, oa, ob);
  schedule16<false>();
  barrier_but_vmcnt<2 * kStageLoads>();
  dma_stage(ra, rb, tl, k4, k, cur_a, cur_b, wave);
  mma16<1>(acc, f, nxt_a, nxt_b, oa, ob);
  schedule16<true>();
}

// A wave's 128 x 128 outputs.  Accumulator block (i, j): lane l holds token l % 32 of block j
// and, in register 4 q + e, channel 8 q + 4 (l / 32) + e of block i.  The values go through
// LDS, [64 tokens][256 B] in `lo` and in `hi` with 16-byte chunk c of a token at c ^ (token %
// 16), so that rows of the output are written 256 bytes at a time.  WIDE: as fp32, 64 channels
// at a time (fp32 outputs, and bf16 ones that are added to: one rounding); else as bf16.
template <bool WIDE>
__device__ __forceinline__ void tile_store(const i32x16 (&acc)[4][4], const Int8Args &a,
                                           uint8_t *lo, uint8_t *hi, int64_t t0, int64_t n0,
                                           int lane) {
  const int h = lane >> 5, tok = lane & 31;
  float sa[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t t = t0 + j * 32 + tok;
    sa[j] = t < a.tokens ? a.a_scales[t] : 0.0f;
  }
#pragma unroll
  for (int half = 0; half < (WIDE ? 2 : 1); ++half) {
#pragma unroll
    for (int i = WIDE ? 2 * half : 0; i < (WIDE ? 2 * half + 2 : 4); ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t n = n0 + i * 32 + q * 8 + h * 4;
        f32x4 sw = {1.0f, 1.0f, 1.0f, 1.0f};
        float bias[4] = {};
        if (n < a.n) {
          if (a.w_scales) sw = *reinterpret_cast<const f32x4 *>(a.w_scales + n);
          if (a.bias) {
            const u32x2 b = *reinterpret_cast<const u32x2 *>(a.bias + n);
            bias[0] = bf16_lo(b.x); bias[1] = bf16_hi(b.x);
            bias[2] = bf16_lo(b.y); bias[3] = bf16_hi(b.y);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = ((float)acc[i][j][4 * q + e] * sa[j]) * sw[e] + bias[e];
          uint8_t *row = (j < 2 ? lo : hi) + ((j & 1) * 32 + tok) * 256;
          if constexpr (WIDE) {
            const int c = (i & 1) * 8 + q * 2 + h;
            *reinterpret_cast<f32x4 *>(row + ((c ^ (tok & 15)) << 4)) = f32x4{v[0], v[1], v[2], v[3]};
          } else {
            const int c = i * 4 + q;
            *reinterpret_cast<u32x2 *>(row + ((c ^ (tok & 15)) << 4) + h * 8) =
                u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
          }
        }
      }
    }
    // a row of 16 chunks by 16 lanes, 4 rows at a time
    const int c = lane & 15, sub = lane >> 4;
#pragma unroll 4
    for (int it = 0; it < 32; ++it) {
      const int r = it * 4 + sub;
      const int64_t t = t0 + r;
      const u32x4 w = *reinterpret_cast<const u32x4 *>((r < 64 ? lo : hi) + (r & 63) * 256 +
                                                       ((c ^ (r & 15)) << 4));
      if (t >= a.tokens) continue;
      if constexpr (WIDE) {
        const int64_t n = n0 + half * 64 + c * 4;
        if (n >= a.n) continue;
        f32x4 v = __builtin_bit_cast(f32x4, w);
        if (a.out_f32) {
          f32x4 *o = reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + t * a.ldo + n);
          *o = a.accumulate ? *o + v : v;
        } else {
          u32x2 *o = reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + n);
          const u32x2 p = *o;  // added to: a plain bf16 output is not WIDE
          *o = u32x2{pack_bf16(bf16_lo(p.x) + v.x, bf16_hi(p.x) + v.y),
                     pack_bf16(bf16_lo(p.y) + v.z, bf16_hi(p.y) + v.w)};
        }
      } else {
        const int64_t n = n0 + c * 8;
        if (n < a.n) *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + n) = w;
      }
    }
  }
}

template <bool WIDE>
__global__ __launch_bounds__(kTileThreads, 1) void int8_tile_kernel(const Int8Args a, int tiles_t,
                                                                    int tiles_n) {
  __shared__ __attribute__((aligned(16))) uint8_t a0[kStageBytes], b0[kStageBytes];
  __shared__ __attribute__((aligned(16))) uint8_t a1[kStageBytes], b1[kStageBytes];
  __shared__ __attribute__((aligned(16))) uint8_t a2[kStageBytes], b2[kStageBytes];
  __shared__ __attribute__((aligned(16))) uint8_t a3[kStageBytes], b3[kStageBytes];

  // each XCD takes a contiguous run of tiles, in groups 8 token tiles tall, so that its CUs
  // share rows of both operands in their L2
  int id = blockIdx.x;
  {
    const int n = tiles_t * tiles_n, x = id & 7, q = n >> 3, r = n & 7;
    id = x * q + (x < r ? x : r) + (id >> 3);
  }
  const int per_group = kGroupT * tiles_n;
  const int first_t = (id / per_group) * kGroupT;
  const int gt = tiles_t - first_t < kGroupT ? tiles_t - first_t : kGroupT;
  const int tile_t = __builtin_amdgcn_readfirstlane(first_t + (id % per_group) % gt);
  const int tile_n = __builtin_amdgcn_readfirstlane((id % per_group) / gt);
  const int64_t t0 = (int64_t)tile_t * kTile, n0 = (int64_t)tile_n * kTile;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int wt = wave >> 1, wn = wave & 1;

  const int64_t rows_t = a.tokens - t0 < kTile ? a.tokens - t0 : kTile;
  const int64_t rows_n = a.n - n0 < kTile ? a.n - n0 : kTile;
  const __amdgpu_buffer_rsrc_t ra =
      __builtin_amdgcn_make_buffer_rsrc((void *)(a.a + t0 * a.k), 0, (int)(rows_t * a.k), 0x00020000);
  const __amdgpu_buffer_rsrc_t rb =
      __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + n0 * a.k), 0, (int)(rows_n * a.k), 0x00020000);
  TileLoad tl;
  {
    const int row = lane >> 2;
    tl.g16 = ((lane & 3) ^ ((row >> 1) & 3)) * 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int x = wave * 64 + r * 16 + row;  // rows past the operand lie past its range
      tl.a[r] = (uint32_t)x * (uint32_t)a.k + (uint32_t)tl.g16;
      tl.b[r] = tl.a[r];
    }
  }
  uint32_t oa[2], ob[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int r = lane & 31, g = 2 * ks + (lane >> 5);
    const uint32_t o = (uint32_t)(r * kStageK + ((g ^ ((r >> 1) & 3)) << 4));
    oa[ks] = o + (uint32_t)(wt * 128 * kStageK);
    ob[ks] = o + (uint32_t)(wn * 128 * kStageK);
  }

  i32x16 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x16{};

  const int k = a.k, stages = (k + kStageK - 1) / kStageK;
  dma_stage(ra, rb, tl, 0, k, a0, b0, wave);
  dma_stage(ra, rb, tl, kStageK, k, a1, b1, wave);
  dma_stage(ra, rb, tl, 2 * kStageK, k, a2, b2, wave);
  dma_stage(ra, rb, tl, 3 * kStageK, k, a3, b3, wave);
  barrier_but_vmcnt<3 * kStageLoads>();
  TileFrags f;
#pragma unroll
  for (int i = 0; i < 4; ++i) read_block<0>(f, a0, b0, oa, ob, i);
  int k4 = 4 * kStageK;
  for (int s = 4; s <= stages; s += 4, k4 += 4 * kStageK) {
    tile_stage(acc, f, a0, b0, a1, b1, ra, rb, tl, k4, k, oa, ob, wave);
    tile_stage(acc, f, a1, b1, a2, b2, ra, rb, tl, k4 + kStageK, k, oa, ob, wave);
    tile_stage(acc, f, a2, b2, a3, b3, ra, rb, tl, k4 + 2 * kStageK, k, oa, ob, wave);
    tile_stage(acc, f, a3, b3, a0, b0, ra, rb, tl, k4 + 3 * kStageK, k, oa, ob, wave);
  }
  // one to three stages left, rounded up to two or four (a stage past k is zeros)
  if ((stages & 3) != 0) {
    tile_stage(acc, f, a0, b0, a1, b1, ra, rb, tl, k4, k, oa, ob, wave);
    tile_stage(acc, f, a1, b1, a2, b2, ra, rb, tl, k4 + kStageK, k, oa, ob, wave);
    if ((stages & 3) == 3) {
      tile_stage(acc, f, a2, b2, a3, b3, ra, rb, tl, k4 + 2 * kStageK, k, oa, ob, wave);
    }
  }
  barrier_but_vmcnt<0>();  // loads past the last stage still write LDS

  // the wave's own 32 KB of LDS: two of the stage buffers
  uint8_t *const lo = wave == 0 ? a0 : wave == 1 ? a1 : wave == 2 ? a2 : a3;
  uint8_t *const hi = wave == 0 ? b0 : wave == 1 ? b1 : wave == 2 ? b2 : b3;
  tile_store<WIDE>(acc, a, lo, hi, t0 + wt * 128, n0 + wn * 128, lane);
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
  if (a.tokens > 64) {
    const int tiles_t = (int)((a.tokens + kTile - 1) / kTile), tiles_n = (int)((a.n + kTile - 1) / kTile);
    if (a.out_f32 || a.accumulate)
      hipLaunchKernelGGL(int8_tile_kernel<true>, dim3(tiles_t * tiles_n), dim3(kTileThreads), 0, s, a, tiles_t, tiles_n);
    else
      hipLaunchKernelGGL(int8_tile_kernel<false>, dim3(tiles_t * tiles_n), dim3(kTileThreads), 0, s, a, tiles_t, tiles_n);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(int8_kernel, dim3((unsigned)(((a.n + 63) / 64) * ((a.tokens + 63) / 64))),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hilore
