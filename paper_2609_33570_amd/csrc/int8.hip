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
constexpr int kQuantThreads = 1024;  // at most
constexpr int64_t kQuantHeld = 4 * 8 * kQuantThreads;  // longest row held in registers

// 8 values of x * factor at col.
__device__ __forceinline__ void load_scaled8(const uint16_t *x, const float *factor, int64_t col,
                                             float v[8]) {
  unpack_bf16x8(*reinterpret_cast<const u32x4 *>(x + col), v);
  if (factor) {
    const f32x4 lo = *reinterpret_cast<const f32x4 *>(factor + col);
    const f32x4 hi = *reinterpret_cast<const f32x4 *>(factor + col + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] *= lo[i];
      v[4 + i] *= hi[i];
    }
  }
}

// A workgroup rounds a row at a time: its largest magnitude, then its codes.  Bound by HBM (3 B
// an element) for many tokens, by latency for few.  V > 0: the row stays in registers in
// between, V pieces of 8 values a thread; V = 0: longer rows are read twice.
template <int V>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const QuantArgs a) {
  __shared__ uint32_t lds[2][kQuantThreads / kWave];
  const int waves = blockDim.x / kWave;
  const int64_t stride = (int64_t)blockDim.x * 8, first = (int64_t)threadIdx.x * 8;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x, turn ^= 1) {
    const uint16_t *x = a.x + row * a.ldx;
    float v[V > 0 ? V : 1][8];
    uint32_t top = 0;
    if constexpr (V > 0) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (first + j * stride < a.k) {
          load_scaled8(x, a.factor, first + j * stride, v[j]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
        }
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(fabsf(v[j][i])));
    } else {
      for (int64_t col = first; col < a.k; col += stride) {
        load_scaled8(x, a.factor, col, v[0]);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(fabsf(v[0][i])));
      }
    }
    top = group_max_u32<32>(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, kWave));
    if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < waves; ++w) top = max(top, lds[turn][w]);
    float scale;
    const float r = token_scale(__uint_as_float(top), scale);
    if (threadIdx.x == 0) a.scales[row] = scale;
    int8_t *codes = a.codes + row * a.k;
    if constexpr (V > 0) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (first + j * stride < a.k)
          *reinterpret_cast<u32x2 *>(codes + first + j * stride) = token_codes8(v[j], r);
    } else {
      for (int64_t col = first; col < a.k; col += stride) {
        load_scaled8(x, a.factor, col, v[0]);
        *reinterpret_cast<u32x2 *>(codes + col) = token_codes8(v[0], r);
      }
    }
  }
}

// ------------------------------------------------------------------ product --
// Four neighbouring values of the output (n % 4 == 0): the exact sums, scaled, with bias,
// added or written.
__device__ __forceinline__ void finish4(const Int8Args &a, int64_t t, int64_t n, i32x4 sum) {
  const float sa = a.a_scales[t];
  f32x4 v = {(float)sum.x * sa, (float)sum.y * sa, (float)sum.z * sa, (float)sum.w * sa};
  if (a.w_scales) v *= *reinterpret_cast<const f32x4 *>(a.w_scales + n);
  if (a.bias) {
    const u32x2 b = *reinterpret_cast<const u32x2 *>(a.bias + n);
    v += f32x4{bf16_lo(b.x), bf16_hi(b.x), bf16_lo(b.y), bf16_hi(b.y)};
  }
  if (a.out_f32) {
    f32x4 *o = reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + t * a.ldo + n);
    *o = a.accumulate ? *o + v : v;
  } else {
    u32x2 *o = reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + n);
    if (a.accumulate) {
      const u32x2 p = *o;
      v += f32x4{bf16_lo(p.x), bf16_hi(p.x), bf16_lo(p.y), bf16_hi(p.y)};
    }
    *o = u32x2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
  }
}

constexpr uint32_t kOob = 0x80000000u;  // a buffer offset past every range: loads 0

typedef __attribute__((address_space(3))) void lds_void;

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

// --------------------------------------------------------------- few tokens --
// Up to 64 tokens: the product streams the weights once.  A workgroup owns 16 NB channels
// and a range of k (a part); its waves take k-steps of 64 G bytes in turn and add their sums
// in LDS.  Both operands pass through the wave's own LDS by LDS-DMA, 64 G bytes of a row by 4 G
// neighbouring lanes: straight into v_mfma_i32_16x16x64_i8's registers every lane would
// read another row, and the address unit, which takes a cycle for each 128-byte line, not
// the memory, would set the pace (64 x 18944 x 3584: 27.8 us).  Four slots, three in
// flight; no barriers.  Several parts leave their sums in the workspace for int8_join_kernel.
constexpr int kSlots = 4;

// Rows of one slot: 16 NB channels, then 16 TB tokens, 64 G bytes each; 16-byte chunk c of row
// r lies at c ^ swz(r).  A 16-byte read serves 16 lanes a cycle, quads 0, 3, 5, 6 of each half
// wave and then 1, 2, 4, 7: rows 0..3 and 12..15 at one chunk and 4..11 at the next, or the
// reverse.  With these swz all 16 meet different banks.
template <int G>
__device__ __forceinline__ int few_swz(int row) {
  static_assert(G == 1 || G == 2, "bytes of a row in a slot");
  return G == 1 ? (0x78 >> (2 * ((row >> 2) & 3))) & 3  // 0, 2, 3, 1 for rows 0-3, 4-7, 8-11, 12-15
                : (row & 2) | ((row >> 1) & 4);
}

template <int TB, int NB, int G>
struct FewLoad {
  static constexpr int kRows = 16 / G;  // rows of one load
  static constexpr int kLoads = (TB + NB) * G;
  static constexpr int kSlotBytes = kLoads * 1024;
  uint32_t first;  // the lane's row of load 0, times k
  uint32_t step;   // kRows k
  int chunk[2];    // the lane's first byte within a slot's k, in even and odd loads
};

template <int TB, int NB, int G>
__device__ __forceinline__ void dma_few(const FewLoad<TB, NB, G> &f, __amdgpu_buffer_rsrc_t rw,
                                        __amdgpu_buffer_rsrc_t rx, int k, int end, uint8_t *slot) {
  uint32_t off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    off[i] = k + f.chunk[i] < end ? f.first + (uint32_t)(k + f.chunk[i]) : kOob;
#pragma unroll
  for (int j = 0; j < NB * G; ++j)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void *)(slot + j * 1024), 16,
                                             (int)(off[j & 1] + j * f.step), 0, 0, 0);
#pragma unroll
  for (int j = 0; j < TB * G; ++j)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(slot + (NB * G + j) * 1024), 16,
                                             (int)(off[j & 1] + j * f.step), 0, 0, 0);
}

// The products of one slot; `at`: the lane's fragment offset of each k-step of 64.
template <int TB, int NB, int G>
__device__ __forceinline__ void mma_few(i32x4 (&acc)[NB][TB], const uint8_t *slot,
                                        const uint32_t (&at)[G]) {
#pragma unroll
  for (int g = 0; g < G; ++g) {
    i32x4 w[NB], x[TB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
      w[i] = *reinterpret_cast<const i32x4 *>(slot + at[g] + i * (16 * 64 * G));
#pragma unroll
    for (int j = 0; j < TB; ++j)
      x[j] = *reinterpret_cast<const i32x4 *>(slot + at[g] + (NB + j) * (16 * 64 * G));
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
  }
}

// One slot's turn: the loads of the slot three turns ahead, then the wait for this one's.
template <int TB, int NB, int G>
__device__ __forceinline__ void few_turn(i32x4 (&acc)[NB][TB], const FewLoad<TB, NB, G> &f,
                                         __amdgpu_buffer_rsrc_t rw, __amdgpu_buffer_rsrc_t rx,
                                         int k_ahead, int end, const uint8_t *cur, uint8_t *ahead,
                                         const uint32_t (&at)[G]) {
  constexpr int N = (kSlots - 1) * FewLoad<TB, NB, G>::kLoads;
  static_assert(N < 64, "vmcnt is 6 bits");
  // the reads of `ahead`'s last turn have been waited for by its products
  dma_few(f, rw, rx, k_ahead, end, ahead);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  mma_few<TB, NB, G>(acc, cur, at);
  __builtin_amdgcn_sched_barrier(0);
}

template <int TB, int NB, int G, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void int8_few_kernel(const Int8Args a, int parts) {
  using Load = FewLoad<TB, NB, G>;
  constexpr int kSlot = Load::kSlotBytes;
  __shared__ __attribute__((aligned(16))) uint8_t s0[WAVES * kSlot], s1[WAVES * kSlot];
  __shared__ __attribute__((aligned(16))) uint8_t s2[WAVES * kSlot], s3[WAVES * kSlot];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int tile = blockIdx.x / parts, part = blockIdx.x - tile * parts;
  const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane(tile) * (16 * NB);
  const int64_t rows = a.n - n0 < 16 * NB ? a.n - n0 : 16 * NB;
  const __amdgpu_buffer_rsrc_t rw =
      __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + n0 * a.k), 0, (int)(rows * a.k), 0x00020000);
  const __amdgpu_buffer_rsrc_t rx =
      __builtin_amdgcn_make_buffer_rsrc((void *)a.a, 0, (int)(a.tokens * a.k), 0x00020000);
  // this part's k-steps of 64 G
  const int steps = (a.k + 64 * G - 1) / (64 * G);  // <= 2^11, of at most 2^9 parts
  const int g0 = (int)((unsigned)(steps * part) / (unsigned)parts);
  const int g1 = (int)((unsigned)(steps * (part + 1)) / (unsigned)parts);
  const int end = g1 * 64 * G < a.k ? g1 * 64 * G : a.k;

  Load f;
  {
    const int row = lane / (4 * G);
    f.first = (uint32_t)row * (uint32_t)a.k;
    f.step = (uint32_t)Load::kRows * (uint32_t)a.k;
#pragma unroll
    for (int i = 0; i < 2; ++i)  // 16 rows are one load (G = 1) or two
      f.chunk[i] = ((lane & (4 * G - 1)) ^ few_swz<G>((row + i * Load::kRows) & 15)) * 16;
  }
  uint32_t at[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int r = lane & 15, c = g * 4 + (lane >> 4);
    at[g] = (uint32_t)(r * 64 * G + ((c ^ few_swz<G>(r)) << 4));
  }
  i32x4 acc[NB][TB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = i32x4{};

  uint8_t *const p0 = s0 + wave * kSlot, *const p1 = s1 + wave * kSlot;
  uint8_t *const p2 = s2 + wave * kSlot, *const p3 = s3 + wave * kSlot;
  constexpr int kTurn = WAVES * 64 * G;
  int k = (g0 + wave) * 64 * G;
  dma_few(f, rw, rx, k, end, p0);
  dma_few(f, rw, rx, k + kTurn, end, p1);
  dma_few(f, rw, rx, k + 2 * kTurn, end, p2);
  for (; k < end; k += 4 * kTurn) {  // loads past the end read nothing and give zeros
    few_turn(acc, f, rw, rx, k + 3 * kTurn, end, p0, p3, at);
    few_turn(acc, f, rw, rx, k + 4 * kTurn, end, p1, p0, at);
    few_turn(acc, f, rw, rx, k + 5 * kTurn, end, p2, p1, at);
    few_turn(acc, f, rw, rx, k + 6 * kTurn, end, p3, p2, at);
  }
  // sums of the waves: 1 KB per accumulator block, in the wave's place of s0, then of s1
  barrier_but_vmcnt<0>();
  constexpr int kPerSlot = kSlot / 1024;
  static_assert(NB * TB <= 2 * kPerSlot, "sums fit two slots");
  const auto place = [&](int w, int b) {
    uint8_t *p = b < kPerSlot ? s0 + w * kSlot + b * 1024 : s1 + w * kSlot + (b - kPerSlot) * 1024;
    return reinterpret_cast<i32x4 *>(p) + lane;
  };
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) *place(wave, i * TB + j) = acc[i][j];
  __syncthreads();
  // accumulator block (i, j): lane l holds token l % 16 of block j, channels 4 (l / 16) .. of i
  for (int b = wave; b < NB * TB; b += WAVES) {
    i32x4 sum = *place(0, b);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += *place(w, b);
    const int64_t t = (b % TB) * 16 + (lane & 15), n = n0 + (b / TB) * 16 + (lane >> 4) * 4;
    if (t >= a.tokens || n >= a.n) continue;
    if (parts == 1) finish4(a, t, n, sum);
    else *reinterpret_cast<i32x4 *>(a.part + ((int64_t)part * a.tokens + t) * a.n + n) = sum;
  }
}

// The sums of `parts` partial products ([part][token][channel] in the workspace).
__global__ __launch_bounds__(256) void int8_join_kernel(const Int8Args a, int parts) {
  const uint32_t quads = (uint32_t)a.n / 4, all = (uint32_t)a.tokens * quads;
  // < 2^31: 64 tokens of 2^24 quads, or 1024 tiles, more of which are not split
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const i32x4 *p = reinterpret_cast<const i32x4 *>(a.part) + i;
    i32x4 sum = *p;
#pragma unroll 8
    for (int s = 1; s < parts; ++s) sum += p[(int64_t)s * all];
    const uint32_t t = i / quads;
    finish4(a, t, (int64_t)(i - t * quads) * 4, sum);
  }
}

// ------------------------------------------------------------------- tiles --
// 64 B tokens x 64 B channels (B = 4: 256, B = 2: 128) per workgroup of 4 waves (2 x 2), each
// wave B x B blocks of v_mfma_i32_32x32x32_i8, one wave a SIMD.  Both operands have k
// contiguous, so they are copied to LDS as they are by the buffer unit (16-byte LDS-DMA loads,
// no registers) in stages of 64 k: [64 B rows][64 bytes] each, 16-byte chunk g of row r at
// position g ^ (r / 4 % 4), which spreads the 16 rows that one cycle of a fragment read takes
// over all banks.  Four stages are in flight.
// A large product is bound by the matrix units at the clock their power allows: 16384 x 3584 x 18944
// takes 1040 to 1090 us on different machines, 2.04 to 2.15 POP/s; the outputs' way through LDS (5 us a tile) is not covered by products.
constexpr int kStageK = 64, kTileThreads = 256;
constexpr int kTurnK = 4 * kStageK;  // a turn of the ring
constexpr int kGroupT = 16, kBlockT = 8, kBlockN = 4;  // tiles

template <int B>
struct Tile {
  static constexpr int kSide = 64 * B;
  static constexpr int kStageBytes = kSide * kStageK;  // of one operand
  static constexpr int kStageLoads = 2 * B;            // LDS-DMA instructions of a wave per stage
  static constexpr int kRow = 32 * B;                  // bytes of a token that a wave writes at a time
  static constexpr int kPerCu = B == 2 ? 2 : 1;        // workgroups, by their LDS
};

template <int B>
struct TileLoad {
  uint32_t row[B];  // byte offset of the lane's chunk in its row of each load, at k = 0
  int g16;          // its first k within a stage
};

struct TileSource {  // the operands' rows of one tile
  __amdgpu_buffer_rsrc_t a, b;
};

// Stage k0 of both operands into `la`, `lb`: load r of wave w writes rows 16 (B w + r) ..
// + 15, lane l the chunk at position l % 4 of row l / 4.  Chunks past `end` read as 0.
template <int B>
__device__ __forceinline__ void dma_stage(const TileSource &src, const TileLoad<B> &tl, int k0,
                                          int end, uint8_t *la, uint8_t *lb, int wave) {
  const uint32_t past = k0 + tl.g16 < end ? 0u : kOob;
#pragma unroll
  for (int r = 0; r < B; ++r) {
    const int off = (int)((tl.row[r] + (uint32_t)k0) | past), to = (wave * B + r) * 16 * kStageK;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src.a, (lds_void *)(la + to), 16, off, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src.b, (lds_void *)(lb + to), 16, off, 0, 0, 0);
  }
}

template <int B>
struct TileFrags {
  i32x4 a[2][B], b[2][B];  // fragments of even and odd k-steps
};

// Fragments of k-step KS (32 k) of a stage: lane l takes chunk 2 KS + l / 32 of row l % 32
// of each 32-row block; oa, ob: the lane's offset in block 0 at KS = 0 and at KS = 1.
template <int KS, int B>
__device__ __forceinline__ void read_block(TileFrags<B> &f, const uint8_t *la, const uint8_t *lb,
                                           const uint32_t (&oa)[2], const uint32_t (&ob)[2],
                                           int i) {
  f.a[KS][i] = *reinterpret_cast<const i32x4 *>(la + oa[KS] + i * 32 * kStageK);
  f.b[KS][i] = *reinterpret_cast<const i32x4 *>(lb + ob[KS] + i * 32 * kStageK);
}

// The products of k-step KS with the reads of the other k-step's fragments (from la, lb), a
// read after each of the first 2 B MFMAs, so that they are there when the next region begins;
// LOADS: an LDS-DMA load after each of the others (B = 2: after every read).
template <int KS, bool LOADS, int B>
__device__ __forceinline__ void mma_step(i32x16 (&acc)[B][B], TileFrags<B> &f, const uint8_t *la,
                                         const uint8_t *lb, const uint32_t (&oa)[2],
                                         const uint32_t (&ob)[2]) {
#pragma unroll
  for (int i = 0; i < B; ++i) read_block<KS ^ 1>(f, la, lb, oa, ob, i);
#pragma unroll
  for (int i = 0; i < B; ++i) {
#pragma unroll
    for (int j = 0; j < B; ++j)
      acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[KS][i], f.a[KS][j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < B * B; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                        // 1 MFMA
    if (i < 2 * B) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);         // 1 LDS read
    if (LOADS && (B == 2 || i >= 2 * B)) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Stage s in (cur_a, cur_b), its first fragments in f: the products of its two k-steps.
// Between them the wave waits for its own loads of stage s + 1, and one barrier says that
// they have landed for all waves and that nobody reads stage s from LDS any more; the second
// k-step's products then cover the loads of stage s + 4 into its place and the first
// fragment reads of stage s + 1.
template <int B>
__device__ __forceinline__ void tile_stage(i32x16 (&acc)[B][B], TileFrags<B> &f, uint8_t *cur_a,
                                           uint8_t *cur_b, const uint8_t *nxt_a,
                                           const uint8_t *nxt_b, const TileSource &src,
                                           const TileLoad<B> &tl, int k4, int end,
                                           const uint32_t (&oa)[2], const uint32_t (&ob)[2],
                                           int wave) {
  mma_step<0, false>(acc, f, cur_a, cur_b, oa, ob);
  barrier_but_vmcnt<2 * Tile<B>::kStageLoads>();
  dma_stage(src, tl, k4, end, cur_a, cur_b, wave);
  mma_step<1, true>(acc, f, nxt_a, nxt_b, oa, ob);
}

// One accumulator value, where it is asked for: left to itself the compiler copies all 256 at
// once and spills what the next tile needs.  (The compiler does not see the read, so its
// distance from the last MFMA is tile_store's to keep.)
__device__ __forceinline__ int acc_value(int a) {
  int v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return v;
}

// Scales and bias of one tile in LDS, copied there while the tile is at work.
template <int B>
struct TileScales {
  float sa[Tile<B>::kSide], sw[Tile<B>::kSide];
  uint16_t bias[Tile<B>::kSide];
};

// Rows of a tile of S from `at` on: 0 in a quarter (see below) past the operand.
template <int S>
__device__ __forceinline__ int64_t rows_left(int64_t rows, int64_t at) {
  const int64_t left = rows - at;
  return left < S ? (left > 0 ? left : 0) : S;
}

template <int B>
__device__ __forceinline__ void dma_scales(const Int8Args &a, int64_t t0, int64_t n0,
                                           TileScales<B> &s, int wave, int lane) {
  constexpr int S = Tile<B>::kSide;
  const int64_t rows_t = rows_left<S>(a.tokens, t0), rows_n = rows_left<S>(a.n, n0);
  const auto copy = [&](const void *from, int64_t bytes, void *to) {
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(from), 0, (int)bytes, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)((uint8_t *)to + wave * 256), 4,
                                             (wave * 64 + lane) * 4, 0, 0, 0);
  };
  if (wave < B) copy(a.a_scales + t0, rows_t * 4, s.sa);
  if (a.w_scales && wave < B) copy(a.w_scales + n0, rows_n * 4, s.sw);
  if (a.bias && wave < B / 2) copy(a.bias + n0, rows_n * 2, s.bias);
}

// What becomes of a tile's sums: a bf16 output; an fp32 one, or a bf16 one that is added to
// (in fp32, one rounding); raw sums of a part of k in the workspace.
enum Store : int { kStoreBf16, kStoreWide, kStorePart };

// One piece of work: a tile, or the part of k from `begin` to `end` of one.
struct TileWork {
  int64_t t0, n0;
  int part, begin, end;
};

// A wave's 32 B x 32 B outputs.  Accumulator block (i, j): lane l holds token l % 32 of block j
// and, in register 4 q + e, channel 8 q + 4 (l / 32) + e of block i.  The values go through the
// wave's LDS, 32 tokens of kRow bytes at a time with their 16-byte chunks permuted so that 16
// tokens cover all banks, so that the output is written in whole rows of kRow bytes.
template <int MODE, int B>
__device__ __forceinline__ void tile_store(const i32x16 (&acc)[B][B], const Int8Args &a,
                                           const TileScales<B> &s, uint8_t *lds, const TileWork &w,
                                           int wt, int wn, int lane) {
  constexpr int kRow = Tile<B>::kRow, kChunks = kRow / 16, kWave = 32 * B;
  constexpr int kChannels = kRow / (MODE == kStoreBf16 ? 2 : 4);
  asm volatile("s_nop 15\n\ts_nop 15");  // more than the 18 states from an MFMA to a read of its result
  asm volatile("" : "+v"(lane));  // else the addresses below are formed once and kept, 100 registers
  const int h = lane >> 5, tok = lane & 31;
  const int c = lane % kChunks, sub = lane / kChunks;
  const auto at = [](int row, int chunk) {
    return row * kRow + ((chunk ^ (row / (16 / kChunks) % kChunks)) << 4);
  };
#pragma unroll
  for (int j = 0; j < B; ++j) {
    const float sa = MODE == kStorePart ? 1.0f : s.sa[wt * kWave + j * 32 + tok];
#pragma unroll
    for (int c0 = 0; c0 < kWave; c0 += kChannels) {
#pragma unroll
      for (int qq = 0; qq < kChannels / 8; ++qq) {
        const int i = (c0 + qq * 8) / 32, q = (c0 + qq * 8) % 32 / 8;
        i32x4 sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = acc_value(acc[i][j][4 * q + e]);
        if constexpr (MODE == kStorePart) {
          *reinterpret_cast<i32x4 *>(lds + at(tok, qq * 2 + h)) = sum;
          continue;
        }
        const int ch = wn * kWave + i * 32 + q * 8 + h * 4;
        f32x4 v = {(float)sum.x * sa, (float)sum.y * sa, (float)sum.z * sa, (float)sum.w * sa};
        if (a.w_scales) v *= *reinterpret_cast<const f32x4 *>(s.sw + ch);
        if (a.bias) {
          const u32x2 b = *reinterpret_cast<const u32x2 *>(s.bias + ch);
          v += f32x4{bf16_lo(b.x), bf16_hi(b.x), bf16_lo(b.y), bf16_hi(b.y)};
        }
        if constexpr (MODE == kStoreWide) {
          *reinterpret_cast<f32x4 *>(lds + at(tok, qq * 2 + h)) = v;
        } else {
          *reinterpret_cast<u32x2 *>(lds + at(tok, qq) + h * 8) =
              u32x2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
        }
      }
#pragma unroll
      for (int r = sub; r < 32 + sub; r += 64 / kChunks) {
        const int64_t t = w.t0 + wt * kWave + j * 32 + r;
        const int64_t n = w.n0 + wn * kWave + c0 + c * (kChannels / kChunks);
        const u32x4 o4 = *reinterpret_cast<const u32x4 *>(lds + at(r, c));
        if (t >= a.tokens || n >= a.n) continue;
        if constexpr (MODE == kStorePart) {
          *reinterpret_cast<u32x4 *>(a.part + ((int64_t)w.part * a.tokens + t) * a.n + n) = o4;
        } else if constexpr (MODE == kStoreWide) {
          f32x4 v = __builtin_bit_cast(f32x4, o4);
          if (a.out_f32) {
            f32x4 *o = reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + t * a.ldo + n);
            *o = a.accumulate ? *o + v : v;
          } else {
            u32x2 *o = reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + n);
            const u32x2 p = *o;  // added to: a plain bf16 output is kStoreBf16
            *o = u32x2{pack_bf16(bf16_lo(p.x) + v.x, bf16_hi(p.x) + v.y),
                       pack_bf16(bf16_lo(p.y) + v.z, bf16_hi(p.y) + v.w)};
          }
        } else {
          *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + t * a.ldo + n) = o4;
        }
      }
    }
  }
}

// Piece `id` of the order of work: parts slowest, then groups 16 token tiles tall, in them blocks
// of 8 x 4 tiles.  An XCD's workgroups have a block and share its rows in their L2, and the blocks
// at work at a time make up 16 x 16 tiles, whose rows come from memory once for all XCDs (with
// rows of tiles to each XCD of their own 16384 x 3584 x 18944 takes 1166 us, so 1080).
// QUARTERS: the tiles are of 256 x 256 and a piece is a quarter of one.
template <int B, bool QUARTERS>
__device__ __forceinline__ TileWork work_of(const Int8Args &a, int id, int tiles_t, int tiles_n,
                                            int parts) {
  const int tiles = tiles_t * tiles_n;
  TileWork w;
  const int quarter = id & 3;
  if constexpr (QUARTERS) id >>= 2;
  w.part = __builtin_amdgcn_readfirstlane(id / tiles);
  id -= w.part * tiles;
  const int group = id / (kGroupT * tiles_n), t_first = group * kGroupT;
  const int gt = tiles_t - t_first < kGroupT ? tiles_t - t_first : kGroupT;
  id -= t_first * tiles_n;
  const int column = id / (gt * kBlockN), n_first = column * kBlockN;
  const int gn = tiles_n - n_first < kBlockN ? tiles_n - n_first : kBlockN;
  id -= n_first * gt;
  const int block = id / (kBlockT * gn);
  const int bt = gt - block * kBlockT < kBlockT ? gt - block * kBlockT : kBlockT;
  id -= block * kBlockT * gn;
  const int t = t_first + block * kBlockT + id % bt, n = n_first + id / bt;
  w.t0 = (int64_t)__builtin_amdgcn_readfirstlane(QUARTERS ? 2 * t + (quarter & 1) : t) * Tile<B>::kSide;
  w.n0 = (int64_t)__builtin_amdgcn_readfirstlane(QUARTERS ? 2 * n + (quarter >> 1) : n) * Tile<B>::kSide;
  const int turns = (a.k + kTurnK - 1) / kTurnK;  // <= 2^9, of at most 2^8 parts
  w.begin = turns * w.part / parts * kTurnK;
  const int end = turns * (w.part + 1) / parts * kTurnK;
  w.end = end < a.k ? end : a.k;
  return w;
}

template <int B>
__device__ __forceinline__ TileSource tile_source(const Int8Args &a, const TileWork &w) {
  constexpr int S = Tile<B>::kSide;
  const int64_t rows_t = rows_left<S>(a.tokens, w.t0), rows_n = rows_left<S>(a.n, w.n0);
  TileSource s;
  s.a = __builtin_amdgcn_make_buffer_rsrc((void *)(a.a + w.t0 * a.k), 0, (int)(rows_t * a.k), 0x00020000);
  s.b = __builtin_amdgcn_make_buffer_rsrc((void *)(a.w + w.n0 * a.k), 0, (int)(rows_n * a.k), 0x00020000);
  return s;
}

// A workgroup stays for its pieces of all rounds.  Their stages follow one another in the ring
// without a gap: while a piece's last four are multiplied, the next one's first four
// are loaded, and they land while the outputs are written.
// It has the pieces from `first` to `first` + `pieces`.
template <int B, int MODE, bool QUARTERS>
__global__ __launch_bounds__(kTileThreads, Tile<B>::kPerCu) void int8_tile_kernel(
    const Int8Args a, int tiles_t, int tiles_n, int parts, int first, int pieces) {
  constexpr int kBytes = Tile<B>::kStageBytes;
  __shared__ __attribute__((aligned(16))) uint8_t a0[kBytes], b0[kBytes], a1[kBytes], b1[kBytes];
  __shared__ __attribute__((aligned(16))) uint8_t a2[kBytes], b2[kBytes], a3[kBytes], b3[kBytes];
  __shared__ __attribute__((aligned(16))) uint8_t rows[4][32 * Tile<B>::kRow];
  __shared__ __attribute__((aligned(16))) TileScales<B> scales[2];

  // every round of the grid takes the next gridDim.x pieces, XCD x (workgroups are dealt round
  // robin) an eighth of them; -1: no more
  const int x = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const auto piece = [&](int begin) {
    const int count = pieces - begin < (int)gridDim.x ? pieces - begin : (int)gridDim.x;
    const int per = count >> 3, more = count & 7;
    return slot < per + (x < more ? 1 : 0) ? first + begin + x * per + (x < more ? x : more) + slot : -1;
  };
  int begin = 0, id = piece(0);  // the grid is at most the pieces: every workgroup has one

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int wt = wave >> 1, wn = wave & 1;

  TileLoad<B> tl;
  {
    const int row = lane >> 2;
    tl.g16 = ((lane & 3) ^ ((row >> 2) & 3)) * 16;
#pragma unroll
    for (int r = 0; r < B; ++r)  // rows past the operand lie past its range
      tl.row[r] = (uint32_t)((wave * B + r) * 16 + row) * (uint32_t)a.k + (uint32_t)tl.g16;
  }
  uint32_t oa[2], ob[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int r = lane & 31, g = 2 * ks + (lane >> 5);
    const uint32_t o = (uint32_t)(r * kStageK + ((g ^ ((r >> 2) & 3)) << 4));
    oa[ks] = o + (uint32_t)(wt * 32 * B * kStageK);
    ob[ks] = o + (uint32_t)(wn * 32 * B * kStageK);
  }

  TileWork w = work_of<B, QUARTERS>(a, id, tiles_t, tiles_n, parts), next = w;
  TileSource src = tile_source<B>(a, w);
  dma_stage(src, tl, w.begin, w.end, a0, b0, wave);
  dma_stage(src, tl, w.begin + kStageK, w.end, a1, b1, wave);
  dma_stage(src, tl, w.begin + 2 * kStageK, w.end, a2, b2, wave);
  dma_stage(src, tl, w.begin + 3 * kStageK, w.end, a3, b3, wave);
  barrier_but_vmcnt<3 * Tile<B>::kStageLoads>();
  TileFrags<B> f;
#pragma unroll
  for (int i = 0; i < B; ++i) read_block<0>(f, a0, b0, oa, ob, i);

  int turn = 0;
  for (;;) {
    i32x16 acc[B][B];
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
      for (int j = 0; j < B; ++j) acc[i][j] = i32x16{};
    // the other ones are still being read by waves that have not passed this piece's first
    // barrier
    if constexpr (MODE != kStorePart) dma_scales(a, w.t0, w.n0, scales[turn], wave, lane);
    // a turn of four stages (the last ones past the end are zeros); `at`: what is loaded meanwhile
    bool more_work = true;
    for (int k = w.begin + kTurnK;; k += kTurnK) {
      const bool done = k >= w.end;
      int at = k;
      if (done) {
        begin += (int)gridDim.x;
        id = begin < pieces ? piece(begin) : -1;
        more_work = id >= 0;
        if (more_work) {
          next = work_of<B, QUARTERS>(a, id, tiles_t, tiles_n, parts);
          src = tile_source<B>(a, next);
          at = next.begin;
        } else {
          at = next.end = 0;  // nothing more: zeros
        }
      }
      const int end = next.end;
      tile_stage(acc, f, a0, b0, a1, b1, src, tl, at, end, oa, ob, wave);
      tile_stage(acc, f, a1, b1, a2, b2, src, tl, at + kStageK, end, oa, ob, wave);
      tile_stage(acc, f, a2, b2, a3, b3, src, tl, at + 2 * kStageK, end, oa, ob, wave);
      tile_stage(acc, f, a3, b3, a0, b0, src, tl, at + 3 * kStageK, end, oa, ob, wave);
      if (done) break;
    }
    tile_store<MODE>(acc, a, scales[turn], rows[wave], w, wt, wn, lane);
    turn ^= 1;
    if (!more_work) break;
    w = next;
  }
  barrier_but_vmcnt<0>();  // loads past the last piece still write LDS
}

}  // namespace

hipError_t launch_quantize_tokens(const QuantArgs &a, hipStream_t s) {
  if (a.tokens == 0) return hipSuccess;
  // few tokens: as many threads as there are pieces; many: two pieces a thread (16384 x 3584
  // with 1 / 2 / 4: 42.5 / 34.5 / 37.4 us, x 8192 with 2 / 4: 68.8 / 75.3; 5.1 to 5.9 TB/s
  // over operands in turn that no cache holds; 46 us and 3.8 TB/s in front of a product, under a trace)
  const int64_t pieces = (a.k + 7) / 8;
  const int v = a.k > kQuantHeld ? 0
                : a.tokens < 1024 ? (pieces <= 1024 ? 1 : pieces <= 2048 ? 2 : 4)
                                  : (pieces <= 256 ? 1 : pieces <= 1024 ? 2 : 4);
  int64_t threads = v == 0 ? kQuantThreads : ((pieces + v - 1) / v + kWave - 1) / kWave * kWave;
  if (threads < kWave) threads = kWave;
  const dim3 grid((unsigned)(a.tokens < (1 << 20) ? a.tokens : 1 << 20)), block((unsigned)threads);
  if (v == 1) hipLaunchKernelGGL(quantize_kernel<1>, grid, block, 0, s, a);
  else if (v == 2) hipLaunchKernelGGL(quantize_kernel<2>, grid, block, 0, s, a);
  else if (v == 4) hipLaunchKernelGGL(quantize_kernel<4>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(quantize_kernel<0>, grid, block, 0, s, a);
  return hipGetLastError();
}

namespace {

// How a product of up to kFewTokens tokens runs.  A workgroup of 128 KB of LDS has a CU to
// itself and waits 2 to 3 us for its first operands, so what counts is that the workgroups
// fill the chip once: k is split into as many parts as whole blocks of channels fit 256
// CUs (16 tokens, 18944 x 3584: 1 / 2 parts 16.5 / 21.9 us),
// but a part keeps 2048 k for the price of the second launch (4.5 us).  Up to 16 tokens the
// 16-channel blocks of more than 256 CUs' worth go as 32-channel workgroups of 48 KB
// instead, three to a CU (1 x 3584 x 4608 7.6 -> 5.1 us, x 18944 21.6 -> 15.5).
constexpr int kFewTokens = 64;
struct FewPlan {
  int channels, parts;  // channels of a workgroup
};

// 33 to 64 tokens times large weights go as tiles: 64 x 3584 x 18944 takes 25.5 us as tiles and 32.2
// here, x 18944 x 3584 23.2 and 25.5, but x 3584 x 4608 13.9 and 11.7, x 896 x 128 7.3 and 5.5.
bool runs_few(int64_t tokens, int64_t k, int64_t n) {
  return tokens <= 32 || (tokens <= kFewTokens && k * n <= (int64_t)1 << 25);
}

FewPlan few_plan(int64_t tokens, int64_t k, int64_t n) {
  FewPlan p{};
  p.channels = tokens > 32 ? 64 : tokens > 16 || n > 16 * 256 ? 32 : 16;
  const int64_t tiles = (n + p.channels - 1) / p.channels;
  int64_t parts = 256 / tiles;
  if (parts > k / 2048) parts = k / 2048;
  p.parts = parts < 1 ? 1 : (int)parts;
  return p;
}

void launch_join(const Int8Args &a, int parts, hipStream_t s) {
  const int64_t groups = (a.tokens * (a.n / 4) + 255) / 256;
  hipLaunchKernelGGL(int8_join_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s,
                     a, parts);
}

template <int TB, int NB, int G, int WAVES>
void launch_few(const Int8Args &a, const FewPlan &p, hipStream_t s) {
  const int64_t tiles = (a.n + 16 * NB - 1) / (16 * NB);
  hipLaunchKernelGGL((int8_few_kernel<TB, NB, G, WAVES>), dim3((unsigned)(tiles * p.parts)),
                     dim3(WAVES * 64), 0, s, a, p.parts);
  if (p.parts > 1) launch_join(a, p.parts, s);
}

// How a product runs that the few-token kernel does not take: in tiles of 256 x 256 or 128 x 128,
// of all of k or of one of several parts of it.  The larger tile reads half as much per product
// and wins where there are tiles for all CUs; the smaller one, parts of k, or both, where there
// are not: 700 x 3584 x 3584 takes 18.4 us in small tiles and 44.0 in large ones,
// 3000 x 3584 x 3584 54.7 and 50.8; 128 x 18944 x 3584 118 us whole and 28 in nine parts.  The
// plan with the least estimated time is taken.  The estimate, in us, was fitted to both sides and
// 1, 2 and 4 parts at 39 shapes of 65 to 16384 tokens; it takes one within about 5 % of the fastest.
// Where 256 x 256 tiles leave a last round with at most 64, those may go as quarters of 128 x 128,
// one to a CU, in a launch of their own (4200 x 4112 x 4104, 33 tiles: 136 -> 102 us,
// 1789 x 4864 x 18944, 6: 215 -> 191).  Half a round stays as it is (16384 x 18944 x 3584 1069, as
// quarters 1104): under the power limit half the CUs run faster.
struct TilePlan {
  int side, parts;
  int64_t quartered;  // of the last tiles of 256 x 256
};

constexpr int kMaxParts = 32;

TilePlan tile_plan(int64_t tokens, int64_t k, int64_t n) {
  const int64_t turns = (k + kTurnK - 1) / kTurnK;
  const double far = k * n > (int64_t)1 << 25 ? 1.4 : 1.0;  // weights from beyond the caches
  TilePlan best{256, 1, 0};
  double least = 0.0;
  for (const int side : {256, 128}) {
    const double stage = (side == 256 ? 0.55 : 0.22) * far, ends = side == 256 ? 5.0 : 2.0;
    const int64_t tiles = ((tokens + side - 1) / side) * ((n + side - 1) / side), rest = tiles % 256;
    for (int parts = 1; parts == 1 || (parts <= turns && parts <= kMaxParts); ++parts) {
      const int64_t rounds = (tiles * parts + 255) / 256;
      double us = ends + (double)rounds * ((double)((turns + parts - 1) / parts) * 4 * stage + ends);
      if (parts > 1) us += 3.0 + parts * (0.5 + (double)tokens * (double)n * 8 / 6e6);
      if (least == 0.0 || us < least) {
        least = us;
        best = TilePlan{side, parts, 0};
      }
      if (side == 256 && parts == 1 && rest > 0 && rest <= 64 && rest < tiles) {
        const double whole = (double)(turns * 4) * stage + ends;
        const double quarter = (double)(turns * 4) * 0.22 * far + 2.0;
        us = ends + (double)(rounds - 1) * whole + 6.0 + (double)((4 * rest + 255) / 256) * quarter;
        if (us < least) {
          least = us;
          best = TilePlan{256, 1, rest};
        }
      }
      if (rounds > 4) break;  // work enough for every CU
    }
  }
  return best;
}

template <int B, bool QUARTERS>
void launch_tiles(const Int8Args &a, int64_t first, int64_t pieces, int parts, hipStream_t s) {
  constexpr int S = QUARTERS ? 256 : Tile<B>::kSide;
  const int tiles_t = (int)((a.tokens + S - 1) / S), tiles_n = (int)((a.n + S - 1) / S);
  constexpr int64_t kResident = 256 * Tile<B>::kPerCu;
  const dim3 grid((unsigned)(pieces < kResident ? pieces : kResident)), block(kTileThreads);
  if (parts > 1) {
    if constexpr (!QUARTERS) {
      hipLaunchKernelGGL((int8_tile_kernel<B, kStorePart, false>), grid, block, 0, s, a, tiles_t, tiles_n,
                         parts, 0, (int)pieces);
      launch_join(a, parts, s);
    }
  } else if (a.out_f32 || a.accumulate) {
    hipLaunchKernelGGL((int8_tile_kernel<B, kStoreWide, QUARTERS>), grid, block, 0, s, a, tiles_t, tiles_n, 1,
                       (int)first, (int)pieces);
  } else {
    hipLaunchKernelGGL((int8_tile_kernel<B, kStoreBf16, QUARTERS>), grid, block, 0, s, a, tiles_t, tiles_n, 1,
                       (int)first, (int)pieces);
  }
}

}  // namespace

size_t int8_part_bytes(int64_t tokens, int64_t k, int64_t n) {
  if (tokens <= 0 || n <= 0) return 0;
  const int parts = runs_few(tokens, k, n) ? few_plan(tokens, k, n).parts : tile_plan(tokens, k, n).parts;
  return parts > 1 ? (size_t)parts * (size_t)tokens * (size_t)n * sizeof(int32_t) : 0;
}

hipError_t launch_int8(const Int8Args &a, hipStream_t s) {
  if (a.tokens == 0 || a.n == 0) return hipSuccess;
  if (runs_few(a.tokens, a.k, a.n)) {
    const FewPlan p = few_plan(a.tokens, a.k, a.n);
    if (a.tokens <= 16 && p.channels == 16) launch_few<1, 1, 2, 8>(a, p, s);
    else if (a.tokens <= 16) launch_few<1, 2, 1, 4>(a, p, s);
    else if (a.tokens <= 32) launch_few<2, 2, 2, 4>(a, p, s);
    else launch_few<4, 4, 1, 4>(a, p, s);
    return hipGetLastError();
  }
  const TilePlan p = tile_plan(a.tokens, a.k, a.n);
  const int64_t tiles = ((a.tokens + p.side - 1) / p.side) * ((a.n + p.side - 1) / p.side);
  if (p.side == 128) {
    launch_tiles<2, false>(a, 0, tiles * p.parts, p.parts, s);
  } else {
    launch_tiles<4, false>(a, 0, (tiles - p.quartered) * p.parts, p.parts, s);
    if (p.quartered > 0) launch_tiles<2, true>(a, (tiles - p.quartered) * 4, p.quartered * 4, 1, s);
  }
  return hipGetLastError();
}

}  // namespace hilore
