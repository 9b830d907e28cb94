// 4-bit floating point with a scale for each small block of a row: quantisation, and the product of two such operands.
//
// A value is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times its block's scale: for MXFP4 a power of two for
// 32 values, for NVFP4 an e4m3 number for 16 values, times a power of two for the whole tensor.  That last one is a
// power of two, not any number, because a block's scale has a mantissa of its own: the tensor's only has to bring
// scales into e4m3's range, and as it is, no step of the quantisation depends on how a product or a quotient is rounded
// (a quotient within half a step of fp32 of a border between two values is that border).
//
// Scales lie as the tensor cores take them: in groups of 128 rows x 4 blocks, 512 bytes each, where row r and block b
// are at (r % 32) * 16 + (r / 32) * 4 + b; groups along a row follow one another.
#include <algorithm>
#include <cmath>

#include "layer.cuh"
#include "sm100_ptx.cuh"

namespace sparsp {

__host__ __device__ constexpr int fp4_block(int format) { return format == SPARSP_MXFP4 ? 32 : 16; }
// groups of four blocks along a row
__host__ __device__ inline int64_t fp4_groups(int64_t cols, int format) {
  const int span = 4 * fp4_block(format);
  return (cols + span - 1) / span;
}
int64_t fp4_scales_bytes(const sparsp_fp4& f) { return (f.rows + 127) / 128 * fp4_groups(f.cols, f.format) * 512; }

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// ---- quantisation ---------------------------------------------------------------------------------------------------
// A thread has eight values of a row, neighbouring lanes a block; a warp has up to four pieces of 256 values of a row, all
// of whose loads are on their way before the first is used.  Bound by HBM and by instructions at once, about 12 a value in
// mxfp4 and 14 in nvfp4: 75600 x 5120 bf16 with the values written too, 303 us = 5.8 TB/s, nvfp4 315 us.

// 2^k for -127 <= k <= 127, exact
__device__ __forceinline__ float power_of_two(int k) {
  return k == -127 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)(k + 127) << 23);
}
__device__ __forceinline__ float from_e4m3(uint32_t code) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code));
  return __half2float(__ushort_as_half((uint16_t)h));
}
__device__ __forceinline__ uint32_t to_e4m3(float x) {
  uint16_t h;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(0.0f), "f"(x));
  return h;
}
// eight values in half steps of e2m1, ties to the even code, what is beyond 6 becomes 6; the first in the low bits
__device__ __forceinline__ uint32_t to_e2m1(const float (&x)[8]) {
  uint32_t r;
  asm("{\n\t"
      ".reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t"
      "}"
      : "=r"(r)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}
__device__ __forceinline__ void from_e2m1(uint32_t codes, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t h;
    // (a byte by itself: taken out of a wider register by mov, the conversion sees its neighbours)
    asm("{\n\t"
        ".reg .b8 a, b;\n\t"
        "mov.b16 {a, b}, %1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "}"
        : "=r"(h)
        : "h"((uint16_t)(codes >> 8 * i & 0xffu)));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
    x[2 * i] = v.x;
    x[2 * i + 1] = v.y;
  }
}

// Eight values as they lie in memory: one 16-byte access, two for fp32.
template <typename T>
struct Eight {
  static constexpr int kParts = sizeof(T) / 2, kEach = 8 / kParts;
  Vec<T, kEach> part[kParts];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) part[i] = load_once<T, kEach>(p + i * kEach);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kParts; ++i) part[i].clear();
  }
  __device__ __forceinline__ float operator[](int i) const { return part[i / kEach][i % kEach]; }
  __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) part[i].set(x + i * kEach);
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < kParts; ++i) store_vec<T, kEach>(p + i * kEach, part[i]);
  }
};

// The block's scale from its largest magnitude (as bits, so that NaN is above infinity and infinity above the rest):
// its code, its value, and what takes a value to e2m1's range.
template <int kFormat>
struct BlockScale {
  uint32_t code;
  float value, inverse, part = 0.0f;  // NVFP4: `part` is the scale without the tensor's power of two
  __device__ __forceinline__ BlockScale(uint32_t most, int exponent) {
    const bool finite = most < 0x7f800000u;
    if constexpr (kFormat == SPARSP_MXFP4) {
      // the least power of two with most <= 6 times it: most = m 2^E goes to E - 2 for m <= 1.5, else to E - 1
      const int c = max((int)((most + 0x3fffffu) >> 23) - 2, 0);
      code = finite ? c : 0xffu;
      value = finite ? power_of_two(c - 127) : __uint_as_float(0x7fc00000u);
      inverse = finite ? power_of_two(127 - c) : 0.0f;
    } else {
      // most / 6, correctly rounded: the product with the rounded 1/6, corrected by what it leaves (Markstein's division)
      // of what stays finite: from 2688 on the scale is 448 anyway
      const float x = fminf(__uint_as_float(most) * power_of_two(-exponent), 1e30f), sixth = 1.0f / 6.0f, q = x * sixth;
      code = finite ? to_e4m3(fmaf(fmaf(-6.0f, q, x), sixth, q)) : 0x7fu;
      part = finite ? from_e4m3(code) : 0.0f;
      value = finite ? part * power_of_two(exponent) : __uint_as_float(0x7fc00000u);
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(part));  // (a step of fp32 off is near enough, see OverScale)
      if (part == 0.0f) inverse = 0.0f;
    }
  }
};

// x over the scale, on the right side of every border between two values.
// NVFP4: a border is a multiple of 2^-2 and met exactly or missed by a step of x's type, 2^-13 at least for 16-bit types:
// a quotient rounded to a multiple of 2^-13, as the sum with 1.5 * 2^10 is, is on the border where x is and otherwise on
// x's side of it.  fp32 misses by less: there the quotient is corrected by what it leaves, which is off by far less than
// half a step (75600 x 5120 bf16 with values 361 us that way, 335 this way at the time).
template <typename T, int kFormat>
struct OverScale {
  float inverse, part, tensor;
  __device__ __forceinline__ OverScale(const BlockScale<kFormat>& s, int exponent)
      : inverse(s.inverse), part(s.part), tensor(kFormat == SPARSP_NVFP4 ? power_of_two(-exponent) : 1.0f) {
    if (sizeof(T) == 2 && kFormat == SPARSP_NVFP4) inverse *= tensor;
  }
  // for a quotient that is zero where x is negative or -0
  static __device__ __forceinline__ float with_sign_of(float x, float q) {
    return __uint_as_float(__float_as_uint(q) | (__float_as_uint(x) & 0x80000000u));
  }
  __device__ __forceinline__ float operator()(float x) const {
    if constexpr (kFormat == SPARSP_MXFP4) {
      return x * inverse;
    } else if constexpr (sizeof(T) == 2) {
      return with_sign_of(x, fmaf(x, inverse, 1536.0f) - 1536.0f);
    } else {
      x *= tensor;
      const float q = fminf(fmaxf(x * inverse, -8.0f), 8.0f);  // (nothing infinite in the next step)
      return with_sign_of(x, fmaf(fmaf(-q, part, x), inverse, q));
    }
  }
};

// The largest magnitude of eight values, as the bits of an fp32 value.  Of 16-bit types two at a time; a NaN is NaN.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Eight<T>& v) {
  if constexpr (sizeof(T) == 2) {
    uint32_t m = v.part[0].w[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const uint32_t w = v.part[0].w[i] & 0x7fff7fffu;
      if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w));
      else
        asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m) : "r"(w));
    }
    Vec<T, 8> both;
    both.w[0] = m;
    return max(__float_as_uint(both[0]) & 0x7fffffffu, __float_as_uint(both[1]) & 0x7fffffffu);
  } else {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
    return most;
  }
}

struct QuantizeParams {
  const void* x;
  uint8_t* codes;
  uint8_t* scales;
  void* values;
  int64_t rows, all_rows, ld, groups;  // all_rows: a multiple of 128
  int32_t cols, chunks, pieces, exponent;  // pieces: of 256 values, of a chunk
};
constexpr int kQuantizeUnroll = 4;  // pieces of a warp at a time, at most

template <typename T, int kFormat>
__global__ void __launch_bounds__(256) quantize_kernel(QuantizeParams p) {
  enter_grid(p.x);
  constexpr int kBlock = fp4_block(kFormat), kLanes = kBlock / 8;
  const int lane = threadIdx.x & 31;
  const int64_t units = p.all_rows * p.chunks, step = (int64_t)gridDim.x * 8;
  for (int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); unit < units; unit += step) {
    const int64_t row = unit / p.chunks;
    const int first = (int)(unit - row * p.chunks) * (p.pieces * 256) + lane * 8;
    const bool there = row < p.rows;
    const T* from = static_cast<const T*>(p.x) + row * p.ld;
    Eight<T> v[kQuantizeUnroll];
#pragma unroll
    for (int i = 0; i < kQuantizeUnroll; ++i) {
      if (there && i < p.pieces && first + i * 256 < p.cols)
        v[i].load(from + first + i * 256);
      else
        v[i].clear();
    }
    uint8_t* to_scales = p.scales + (row >> 7) * p.groups * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4;
#pragma unroll
    for (int i = 0; i < kQuantizeUnroll; ++i) {
      if (i >= p.pieces) break;
      const int col = first + i * 256;
      uint32_t most = largest(v[i]);
#pragma unroll
      for (int d = 1; d < kLanes; d *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
      const BlockScale<kFormat> s(most, p.exponent);
      const int block = col / kBlock;
      if (lane % kLanes == 0 && block < p.groups * 4) to_scales[(int64_t)(block >> 2) * 512 + (block & 3)] = (uint8_t)s.code;
      if (!there || col >= p.cols) continue;
      const OverScale<T, kFormat> over(s, p.exponent);
      float q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = over(v[i][e]);
      const uint32_t codes = to_e2m1(q);
      *reinterpret_cast<uint32_t*>(p.codes + (row * p.cols + col) / 2) = codes;
      if (p.values != nullptr) {
        from_e2m1(codes, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] *= s.value;
        v[i].set(q);
        v[i].store(static_cast<T*>(p.values) + row * p.ld + col);
      }
    }
  }
}

int launch_fp4_quantize(const sparsp_fp4& f, const void* X, uint8_t* codes, uint8_t* scales, void* values,
                        cudaStream_t st) {
  QuantizeParams p = {};
  p.x = X;
  p.codes = codes;
  p.scales = scales;
  p.values = values;
  p.rows = f.rows;
  p.all_rows = align_up(f.rows, 128);
  p.ld = f.stride_x;
  p.groups = fp4_groups(f.cols, f.format);
  p.cols = f.cols;
  const int pieces = ceil_div(p.groups * 4 * fp4_block(f.format), 256);
  p.chunks = ceil_div(pieces, kQuantizeUnroll);
  p.pieces = ceil_div(pieces, p.chunks);
  p.exponent = f.exponent;
  const int64_t ctas = (p.all_rows * p.chunks + 7) / 8;
  // as many CTAs as there is work (75600 x 5120 bf16 nvfp4 315 us; eight for each SM, which take what is left by turns, 340)
  const dim3 grid((unsigned)std::min<int64_t>(ctas, 0x7fffffff));
  SPARSP_WITH_TYPE(f.dtype, T, {
    auto kern = f.format == SPARSP_MXFP4 ? quantize_kernel<T, SPARSP_MXFP4> : quantize_kernel<T, SPARSP_NVFP4>;
    SPARSP_CUDA_OK(launch_kernel(kern, grid, 256, 0, st, p));
  });
  return SPARSP_OK;
}

// ---- product --------------------------------------------------------------------------------------------------------
// C = A B^T + bias.  A pair of CTAs (a cluster of two, tcgen05 cta_group::2) makes a tile of 256 rows x BN columns: each
// loads 128 rows of A and half of B's rows by TMA, the even CTA issues the MMAs for both, and each finds its 128 rows,
// all columns, in its own tensor memory.  Scales go from shared to tensor memory by tcgen05.cp before the MMAs that
// read them: a CTA has those of its rows of A and of all of the tile's rows of B.
//
// Two accumulators of 256 columns would fill tensor memory and leave none for scales.  They overlap by 64: the tile
// after begins as soon as these 64 have been read, which is done first: 400 clocks after the last product, of 12000 that
// a tile of 5120 elements of K takes.  (Results by 16 warps with 32 columns each, bias read where it is added and
// arrivals that wait for earlier stores: 1500 clocks.)
//
// Bound by what copies of scales leave of the tensor cores, and by power: one launch of 8192 x 13824 x 5120 at 1.72 GHz
// keeps them busy for 78 % of its cycles in mxfp4 (6 copies a stage) and for 69 % in nvfp4 (12); copied half a stage at
// a time, in places taken by turns: no different.  75600 x 13824 x 5120 nvfp4 2.29 ms = 4.7 PFLOP/s, mxfp4 2.1.
struct ProductParams {
  const void* bias;
  int32_t rows, cols, depth;
  int32_t m_tiles, n_tiles, band, k_blocks;
  float factor;
  uint32_t idesc;
  int32_t* status;
  long long wait_limit, tile_limit;  // of a wait for one stage, and for a tile's products
};

constexpr int kDeep = 256;  // K elements of a stage: one 128-byte swizzled row
constexpr int kResultWarps = 8;
constexpr int kProductThreads = 32 * (kResultWarps + 2);
constexpr int kRows = 128;  // of one CTA
constexpr long long kWaitLimit = 200000000LL;  // of a wait in a kernel: about 0.1 s of SM clocks
constexpr long long kStageLimit = 8192;  // ... and what a stage adds to that of its tile (it takes 300 to 1200 clocks)
constexpr int kPairs = kSms / 2;

template <int kFormat, typename T, int BN>
struct ProductCfg {
  static constexpr int kGroups = kDeep / (4 * fp4_block(kFormat));  // of four blocks, of a stage
  static constexpr int kA = kRows * 128, kB = BN / 2 * 128;
  static constexpr int kTilesB = BN / 128;  // of scales
  static constexpr int kScalesA = kGroups * 512, kScalesB = kTilesB * kGroups * 512;
  static constexpr int kStage = kA + kB + kScalesA + kScalesB;
  static constexpr int kTurn = 4096;            // a warp's results on their way out: 32 rows of 128 bytes
  static constexpr int kMine = BN / 2;          // columns of a warp
  static constexpr int kBias = kMine * 4;       // ... and their bias
  static constexpr int kStages = (227 * 1024 - 1024 - 256 - kResultWarps * (kTurn + kBias)) / kStage;
  static constexpr int kOffOut = kStages * kStage, kOffBias = kOffOut + kResultWarps * kTurn;
  static constexpr int kOffBars = kOffBias + kResultWarps * kBias;
  static constexpr int kBars = 2 * kStages + 7;
  static constexpr int kDynamic = kOffBars + kBars * 8 + 16 + 1024;  // the tiles are aligned to 1024 bytes
  static constexpr int kScaleCols = kGroups * (4 + 4 * kTilesB);     // of tensor memory: 4 of A, 4 or 8 of B a group
  static constexpr int kScaleSets = 64 / kScaleCols;
  static constexpr int kAccStep = BN == 256 ? 192 : 128;
  static_assert(kStage % 1024 == 0, "tiles stay 1024 bytes apart");
};
constexpr int kScaleAt = 448;  // column of tensor memory: behind accumulators at 0 and 192 (of 256) or 128 (of 128)

// Instruction descriptor: e2m1 operands, both K-major; bit 23 says that scales are powers of two.
static uint32_t fp4_instruction(int format, int M, int N) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((format == SPARSP_MXFP4 ? 1u : 0u) << 23) |
         ((uint32_t)(M >> 4) << 24);
}

// 32 rows x 128 bytes of a warp, on their way out through its own shared memory (16-byte pieces of a row in turned
// places, so that lanes do not meet in a bank) as one TMA tile, which leaves out what lies beyond the tensor.
template <typename T, int N>
__device__ __forceinline__ void write_out(const CUtensorMap* to, uint8_t* mine, const float (&x)[N], int first, int lane,
                                          int col, int row, int cols, int rows) {
  constexpr int kEach = 16 / sizeof(T);
  Vec<T, kEach> piece[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) piece[i].set(x + first + i * kEach);
  if (lane == 0) ptx::tma_store_wait_read();
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) store_vec<T, kEach>(reinterpret_cast<T*>(mine + lane * 128 + ((i ^ (lane & 7)) << 4)), piece[i]);
  ptx::fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0 && col < cols && row < rows) {
    ptx::tma_store_2d(to, mine, col, row);
    ptx::tma_store_commit();
  }
}

template <typename T, int kFormat, int BN>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                   const __grid_constant__ CUtensorMap msa, const __grid_constant__ CUtensorMap msb,
                   const __grid_constant__ CUtensorMap mc, ProductParams p) {
  using namespace ptx;
  using C = ProductCfg<kFormat, T, BN>;
  constexpr bool kOverlap = BN == 256;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kOffBars);  // of the even CTA: both CTAs' tiles have arrived
  uint64_t* empty = full + C::kStages;                               // the stage has been multiplied
  uint64_t* acc_full = empty + C::kStages;                           // [2]
  uint64_t* acc_read = acc_full + 2;                                 // [2] of the even CTA: both have read all of theirs
  uint64_t* shared_read = acc_read + 2;  // [2] ... the 64 columns that this accumulator shares with the other
  uint64_t* drained = shared_read + 2;   // every product has ended
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  volatile int* s_abort = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + a, 1);
      mbar_init(acc_read + a, 2 * kResultWarps);
      mbar_init(shared_read + a, 2 * 4);
    }
    mbar_init(drained, 1);
    *s_abort = 0;
    mbar_init_fence();
  }
  if (warp == kResultWarps + 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  enter_grid(p.bias);  // (the next launch may begin: tensor memory is ours, so its CTAs cannot have taken it before)

  const int tiles = p.m_tiles * p.n_tiles, pairs = gridDim.x >> 1;
  auto tile_at = [&](int tile, int& m, int& n) {
    const int per_band = p.band * p.n_tiles, b = tile / per_band, in = tile - b * per_band;
    const int height = min(p.band, p.m_tiles - b * p.band);
    n = in / height;
    m = b * p.band + in - n * height;
  };

  if (warp == kResultWarps) {
    // ---- loads ----
    if (elect_one()) {
      int s = 0;
      uint32_t round = 0;
      for (int tile = blockIdx.x >> 1; tile < tiles && !*s_abort; tile += pairs) {
        int m, n;
        tile_at(tile, m, n);
        for (int k = 0; k < p.k_blocks; ++k) {
          mbar_wait_bounded_inline(empty + s, round ^ 1u, s_abort, 21, p.wait_limit);
          if (*s_abort) break;
          if (rank == 0) mbar_expect_tx(full + s, 2 * C::kStage);
          uint8_t* at = smem + s * C::kStage;
          const uint32_t bar = cluster_addr(full + s, 0);
          tma_load_pair(at, &ma, bar, k * 128, (m * 2 + (int)rank) * kRows);
          tma_load_pair(at + C::kA, &mb, bar, k * 128, (n * 2 + (int)rank) * (BN / 2));
          tma_load_pair_3d(at + C::kA + C::kB, &msa, bar, 0, k * C::kGroups, m * 2 + (int)rank);
          tma_load_pair_3d(at + C::kA + C::kB + C::kScalesA, &msb, bar, 0, k * C::kGroups, n * C::kTilesB);
          if (++s == C::kStages) {
            s = 0;
            round ^= 1u;
          }
        }
      }
      if (*s_abort && rank == 0) {  // copies still in flight are waited for, within the same limit
        const long long t0 = clock64();
        for (int q = 0; q < C::kStages; ++q) {
          const uint32_t phase = q < s ? round : round ^ 1u;
          while (!mbar_try_wait(full + q, phase) && clock64() - t0 < p.wait_limit) {
          }
        }
      }
    }
  } else if (warp == kResultWarps + 1) {
    // ---- products, for both CTAs ----
    if (rank == 0 && elect_one()) {
      const uint32_t base = smem_u32(smem);
      const uint64_t da = make_smem_desc(base, 16u, 1024u), db = make_smem_desc(base + C::kA, 16u, 1024u);
      const uint64_t dsa = make_scale_desc(base + C::kA + C::kB), dsb = make_scale_desc(base + C::kA + C::kB + C::kScalesA);
      int s = 0, acc = 0, set = 0;
      uint32_t round = 0, acc_round = 0;
      for (int tile = blockIdx.x >> 1; tile < tiles && !*s_abort; tile += pairs) {
        // this accumulator's last tile has been read, and of the other's, which is read now, what the two share
        mbar_wait_bounded_inline(acc_read + acc, acc_round ^ 1u, s_abort, 22, p.wait_limit);
        if (kOverlap)
          mbar_wait_bounded_inline(shared_read + (acc ^ 1), acc == 0 ? acc_round ^ 1u : acc_round, s_abort, 23, p.wait_limit);
        tc_fence_after();
        for (int k = 0; k < p.k_blocks; ++k) {
          if (!mbar_wait_bounded_inline(full + s, round, s_abort, 24, p.wait_limit)) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)((s * C::kStage) >> 4);
          const uint32_t sa = tmem + kScaleAt + set * C::kScaleCols, sb = sa + 4 * C::kGroups;
#pragma unroll
          for (int g = 0; g < C::kGroups; ++g) {
            copy_scales_pair(sa + 4 * g, dsa + off + g * 32);
#pragma unroll
            for (int t = 0; t < C::kTilesB; ++t)
              copy_scales_pair(sb + 4 * (C::kTilesB * g + t), dsb + off + (C::kGroups * t + g) * 32);
          }
          const int steps = min(4, (p.depth - k * kDeep + 63) / 64);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (kk >= steps) break;
            const int g = kk * C::kGroups / 4;
            // MXFP4: a group of four blocks serves two instructions, the second half of it the second
            const uint32_t half = C::kGroups == 2 && (kk & 1) ? (2u << 4) | (2u << 29) : 0u;
            mma_fp4_pair<kFormat == SPARSP_MXFP4>(tmem + acc * C::kAccStep, da + off + kk * 2, db + off + kk * 2,
                                                  p.idesc | half, sa + 4 * g, sb + 4 * C::kTilesB * g, k > 0 || kk > 0);
          }
          mma_commit_pair(empty + s);
          set = set + 1 == C::kScaleSets ? 0 : set + 1;
          if (++s == C::kStages) {
            s = 0;
            round ^= 1u;
          }
        }
        mma_commit_pair(acc_full + acc);
        acc ^= 1;
        if (acc == 0) acc_round ^= 1u;
      }
      mma_commit_pair(drained);
    }
  } else {
    // ---- results: warp w has the lanes of quarter w % 4, and half of the columns, 64 at a time ----
    const int quarter = warp & 3, side = warp >> 2;
    uint8_t* mine = smem + C::kOffOut + warp * C::kTurn;
    float* held_bias = reinterpret_cast<float*>(smem + C::kOffBias + warp * C::kBias);
    const T* bias = static_cast<const T*>(p.bias);
    if (bias == nullptr)
      for (int i = lane; i < C::kMine; i += 32) held_bias[i] = 0.0f;
    int acc = 1;
    uint32_t acc_round = 1;
    for (int tile = blockIdx.x >> 1; tile < tiles; tile += pairs) {
      acc ^= 1;
      if (acc == 0) acc_round ^= 1u;
      int m, n;
      tile_at(tile, m, n);
      const int row = (m * 2 + (int)rank) * kRows + quarter * 32, col = n * BN + side * C::kMine;
      if (bias != nullptr) {  // while the products are made
        __syncwarp();
#pragma unroll
        for (int i = 0; i < C::kMine; i += 32) held_bias[i + lane] = col + i + lane < p.cols ? to_float(bias[col + i + lane]) : 0.0f;
      }
      __syncwarp();
      mbar_wait_bounded_inline(acc_full + acc, acc_round, s_abort, 25, p.tile_limit);
      if (__any_sync(0xffffffffu, *s_abort != 0)) break;  // (the same for all lanes)
      tc_fence_after();
      const uint32_t from = tmem + acc * C::kAccStep + side * C::kMine + ((uint32_t)(quarter * 32) << 16);
      // first the columns that both accumulators share: the last of one, the first of the other
      const int flip = kOverlap && acc == 0 ? 1 : 0;
#pragma unroll 1
      for (int h = 0; h < C::kMine / 64; ++h) {
        const int at = (h ^ flip) * 64;
        float x[64];
        tmem_ld32(from + at, reinterpret_cast<uint32_t*>(x));
        tmem_ld32(from + at + 32, reinterpret_cast<uint32_t*>(x + 32));
        tmem_ld_wait(x);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kOverlap && h == 0 && side == flip) mbar_arrive_cluster_relaxed(cluster_addr(shared_read + acc, 0));
          if (h == C::kMine / 64 - 1) mbar_arrive_cluster_relaxed(cluster_addr(acc_read + acc, 0));
        }
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
          const float4 b = *reinterpret_cast<const float4*>(held_bias + at + i);
          x[i] = fmaf(x[i], p.factor, b.x);
          x[i + 1] = fmaf(x[i + 1], p.factor, b.y);
          x[i + 2] = fmaf(x[i + 2], p.factor, b.z);
          x[i + 3] = fmaf(x[i + 3], p.factor, b.w);
        }
#pragma unroll
        for (int i = 0; i < 64; i += 128 / (int)sizeof(T))
          write_out<T>(&mc, mine, x, i, lane, col + at + i, row, p.cols, p.rows);
      }
    }
    if (lane == 0) tma_store_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  // Products use both CTAs' memory until they have ended: after a wait that ran out nobody else has waited for them.
  if (warp == kResultWarps + 1 && elect_one()) {
    const long long t0 = clock64();
    while (!mbar_try_wait(drained, 0) && clock64() - t0 < p.wait_limit) {
    }
  }
  __syncwarp();
  cluster_sync();  // the other CTA's arrivals and products here have ended
  if (warp == kResultWarps + 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
  if (threadIdx.x == 0) report_abort(s_abort, p.status);
}

// ---- product of a few rows ------------------------------------------------------------------------------------------
// With up to 128 rows the call is one pass over B, and a 256-row tile of A would be mostly padding.  Here B's rows are the
// rows of the tile and A's its columns: D = B A^T, 128 rows by the rows of A, rounded up to 16.  A CTA has whole tiles,
// where there are some for half of the SMs: these load as fast as memory gives.  With fewer, a cluster of CTAs shares
// out a tile's K, and each adds some of the rows from the others' shared memory.  Bound by HBM and by a start and an end of
// 5 us: 148 tiles of 5120 values 13.0 us, 296 21.3, the 240 of 1 x 30720 x 5120 nvfp4 19.5, for 92 SMs have two and 56
// one.  (Stages of all tiles shared out evenly, pieces joined through global memory by the CTA that came last: 21.5 us, and
// 15 instead of 6 for 100 x 7680 x 1920.  Loads of several stages next to each other, as a feed-forward's weights want: no
// different.)
struct FewParams {
  const void* bias;
  void* c;
  int64_t ld_c;
  int32_t rows, cols, depth, columns;
  int32_t tiles, k_blocks, pieces, stages, stage_bytes;  // pieces: CTAs of a cluster
  float factor;
  uint32_t idesc;
  int32_t* status;
  long long wait_limit, tile_limit;  // of a wait for one stage, and for a tile's products
};
constexpr int kFewRows = 128;  // (us, this way and by pairs: 16 x 7680 x 1920 4.9 and 6.4, 128 x 6.1 and 6.8; 1 x 30720 x 5120 18.8
                               // and 31.5, 128 x 21.1 and 24.6; 64 x 5120 x 5120 8.5 and 8.5, 128 x 9.7 and 8.9)
constexpr int kFewWarps = 8;  // of results
constexpr int kFewThreads = 64 + 32 * kFewWarps;
constexpr int kFewSmem = 220 * 1024;
constexpr int kFewScalesAt = 256;  // column of tensor memory: two accumulators of 128, then scales

template <typename T, int kFormat>
__global__ void __launch_bounds__(kFewThreads, 1)
    few_rows_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                    const __grid_constant__ CUtensorMap msa, const __grid_constant__ CUtensorMap msb, FewParams p) {
  using namespace ptx;
  constexpr int kGroups = kDeep / (4 * fp4_block(kFormat)), kScales = kGroups * 512;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  __shared__ uint64_t full[16], empty[16], acc_full[2], acc_read[2], drained;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  volatile int* s_abort = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + a, 1);
      mbar_init(acc_read + a, kFewWarps);
    }
    mbar_init(&drained, 1);
    *s_abort = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  enter_grid(p.bias);  // (after tensor memory is ours, as above)
  const int N = p.columns;
  float* sums = reinterpret_cast<float*>(smem);  // [rows of A][128], after the products
  // tiles [t0, t1), blocks of K [k0, k1) of each
  int t0 = blockIdx.x, t1 = t0 + 1, k0 = 0, k1 = p.k_blocks;
  if (p.pieces > 1) {
    t0 = blockIdx.x / p.pieces;
    t1 = t0 + 1;
    const int piece = blockIdx.x - t0 * p.pieces;
    k0 = p.k_blocks * piece / p.pieces;
    k1 = p.k_blocks * (piece + 1) / p.pieces;
  } else {
    t0 = (int)((int64_t)p.tiles * blockIdx.x / gridDim.x);
    t1 = (int)((int64_t)p.tiles * (blockIdx.x + 1) / gridDim.x);
  }

  if (warp == 0) {
    if (elect_one()) {
      int s = 0;
      uint32_t round = 0;
      for (int tile = t0; tile < t1 && !*s_abort; ++tile) {
        for (int k = k0; k < k1; ++k) {
          mbar_wait_bounded_inline(empty + s, round ^ 1u, s_abort, 31, p.wait_limit);
          if (*s_abort) break;
          uint8_t* at = smem + s * p.stage_bytes;
          mbar_expect_tx(full + s, p.stage_bytes);
          tma_load_2d(at, &mb, full + s, k * 128, tile * kRows);
          tma_load_3d(at + kRows * 128 + N * 128, &msb, full + s, 0, k * kGroups, tile);
          tma_load_2d(at + kRows * 128, &ma, full + s, k * 128, 0);
          tma_load_3d(at + kRows * 128 + N * 128 + kScales, &msa, full + s, 0, k * kGroups, 0);
          if (++s == p.stages) {
            s = 0;
            round ^= 1u;
          }
        }
      }
      if (*s_abort) {  // copies still in flight are waited for, within the same limit
        const long long t0 = clock64();
        for (int q = 0; q < p.stages; ++q) {
          const uint32_t phase = q < s ? round : round ^ 1u;
          while (!mbar_try_wait(full + q, phase) && clock64() - t0 < p.wait_limit) {
          }
        }
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t base = smem_u32(smem), scales = base + kRows * 128 + N * 128;
      const uint64_t db = make_smem_desc(base, 16u, 1024u), da = make_smem_desc(base + kRows * 128, 16u, 1024u);
      const uint64_t dsb = make_scale_desc(scales), dsa = make_scale_desc(scales + kScales);
      int s = 0, acc = 0, set = 0;
      uint32_t round = 0, acc_round = 0;
      for (int tile = t0; tile < t1 && !*s_abort; ++tile) {
        mbar_wait_bounded_inline(acc_read + acc, acc_round ^ 1u, s_abort, 32, p.wait_limit);
        for (int k = k0; k < k1; ++k) {
          if (!mbar_wait_bounded_inline(full + s, round, s_abort, 33, p.wait_limit)) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)((s * p.stage_bytes) >> 4);
          const uint32_t sb = tmem + kFewScalesAt + set * (8 * kGroups), sa = sb + 4 * kGroups;
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            copy_scales(sb + 4 * g, dsb + off + g * 32);
            copy_scales(sa + 4 * g, dsa + off + g * 32);
          }
          const int steps = min(4, (p.depth - k * kDeep + 63) / 64);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (kk >= steps) break;
            const int g = kk * kGroups / 4;
            const uint32_t half = kGroups == 2 && (kk & 1) ? (2u << 4) | (2u << 29) : 0u;
            mma_fp4<kFormat == SPARSP_MXFP4>(tmem + acc * 128, db + off + kk * 2, da + off + kk * 2, p.idesc | half,
                                             sb + 4 * g, sa + 4 * g, k > k0 || kk > 0);
          }
          mma_commit(empty + s);
          set ^= 1;
          if (++s == p.stages) {
            s = 0;
            round ^= 1u;
          }
        }
        mma_commit(acc_full + acc);
        acc ^= 1;
        if (acc == 0) acc_round ^= 1u;
      }
      mma_commit(&drained);
      const long long t0 = clock64();
      while (!mbar_try_wait(&drained, 0) && clock64() - t0 < p.wait_limit) {
      }
    }
  } else {
    // warp w has the lanes of quarter w % 4, and every other 16 columns
    const int quarter = warp & 3, side = (warp - 2) >> 2, in_tile = quarter * 32 + lane;
    T* c = static_cast<T*>(p.c);
    int acc = 0;
    uint32_t acc_round = 0;
    for (int tile = t0; tile < t1; ++tile) {
      mbar_wait_bounded_inline(acc_full + acc, acc_round, s_abort, 34, p.tile_limit);
      tc_fence_after();
      const int col = tile * kRows + in_tile;
      const bool in = col < p.cols;
      const float bias = p.bias != nullptr && in ? to_float(static_cast<const T*>(p.bias)[col]) : 0.0f;
      for (int n = side * 16; n < p.rows; n += 32) {
        float x[16];
        tmem_ld16(tmem + acc * 128 + n + ((uint32_t)(quarter * 32) << 16), reinterpret_cast<uint32_t*>(x));
        tmem_ld_wait(x);
        if (p.pieces > 1) {  // (all of this CTA's products have ended: their stages are free)
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[(n + i) * kRows + in_tile] = x[i];
        } else if (in) {
          T* to = c + (int64_t)n * p.ld_c + col;
#pragma unroll
          for (int i = 0; i < 16; ++i, to += p.ld_c)
            if (n + i < p.rows) *to = from_float<T>(fmaf(x[i], p.factor, bias));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_read + acc);
      acc ^= 1;
      if (acc == 0) acc_round ^= 1u;
    }
  }
  __syncwarp();
  if (p.pieces > 1) {
    cluster_sync();
    if (warp >= 2) {
      const int in_tile = (threadIdx.x - 64) & 127, col = t0 * kRows + in_tile;
      const float bias = p.bias != nullptr && col < p.cols ? to_float(static_cast<const T*>(p.bias)[col]) : 0.0f;
      // each half of the warps of each CTA has some of the rows, four at a time
      const int share = 2 * (int)cluster_rank() + (int)(threadIdx.x - 64) / 128;
      for (int n = share * 4; n < p.rows; n += 8 * p.pieces) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int q = 0; q < p.pieces; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += ld_cluster(smem_u32(sums + (n + i) * kRows + in_tile), q);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < p.rows && col < p.cols)
            static_cast<T*>(p.c)[(n + i) * p.ld_c + col] = from_float<T>(fmaf(sum[i], p.factor, bias));
      }
    }
    cluster_sync();  // nobody's memory goes before it has been read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (threadIdx.x == 0) report_abort(s_abort, p.status);
}

// [rows][bytes] in boxes of 128 bytes x 128 rows, swizzled
static int make_codes_map(CUtensorMap* out, const void* base, int64_t rows, int64_t bytes, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)bytes};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  return encode_tmap(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// scales: [tiles of 128 rows][groups][512 bytes] in boxes of some groups of some tiles
static int make_scales_map(CUtensorMap* out, const void* base, int64_t rows, int64_t groups, int box_groups, int box_tiles) {
  const cuuint64_t dims[3] = {128, (cuuint64_t)groups, (cuuint64_t)((rows + 127) / 128)};
  const cuuint64_t strides[2] = {512, (cuuint64_t)groups * 512};
  const cuuint32_t box[3] = {128, (cuuint32_t)box_groups, (cuuint32_t)box_tiles};
  return encode_tmap(out, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}
static int make_result_map(CUtensorMap* out, int dtype, const void* base, int64_t rows, int64_t cols, int64_t ld) {
  const int e = element_bytes(dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * e};
  const cuuint32_t box[2] = {128u / (unsigned)e, 32};
  return encode_tmap(out,
                     dtype == SPARSP_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                     : dtype == SPARSP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                            : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                     2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

static int few_columns(int64_t rows) { return (int)align_up(std::min<int64_t>(std::max<int64_t>(rows, 1), kFewRows), 16); }
int64_t fp4_product_workspace_bytes(const sparsp_fp4_gemm&) { return kStatusWords * 4; }

template <typename T, int kFormat>
static int launch_few_rows(const sparsp_fp4_gemm& f, const void* A, const void* As, const void* B, const void* Bs,
                           const void* bias, void* C, char* ws, cudaStream_t st) {
  constexpr int kGroups = kDeep / (4 * fp4_block(kFormat));
  const int64_t groups = fp4_groups(f.depth, kFormat);
  FewParams p = {};
  p.bias = bias;
  p.c = C;
  p.ld_c = f.stride_c;
  p.rows = (int32_t)f.rows;
  p.cols = f.cols;
  p.depth = f.depth;
  p.columns = few_columns(f.rows);
  p.tiles = ceil_div(f.cols, kRows);
  p.k_blocks = ceil_div(f.depth, kDeep);
  p.stage_bytes = (kRows + p.columns) * 128 + 2 * kGroups * 512;
  p.stages = std::min(16, (kFewSmem - 1024) / p.stage_bytes);
  p.factor = std::ldexp(1.0f, f.exponent);
  p.idesc = fp4_instruction(kFormat, 128, p.columns);
  p.status = reinterpret_cast<int32_t*>(ws);
  p.wait_limit = kWaitLimit;
  p.tile_limit = kWaitLimit + kStageLimit * p.k_blocks;
  CUtensorMap ma, mb, msa, msb;
  int rc;
  if ((rc = make_codes_map(&ma, A, f.rows, f.depth / 2, p.columns)) != SPARSP_OK) return rc;
  if ((rc = make_codes_map(&mb, B, f.cols, f.depth / 2, kRows)) != SPARSP_OK) return rc;
  if ((rc = make_scales_map(&msa, As, f.rows, groups, kGroups, 1)) != SPARSP_OK) return rc;
  if ((rc = make_scales_map(&msb, Bs, f.cols, groups, kGroups, 1)) != SPARSP_OK) return rc;
  // 290 ns a block of K, and for sums that meet 1400 ns and 40 a row, which the pieces share (7680 x 1920, rows and us in
  // one and in two pieces: 1 4.9 5.1, 32 5.0 6.0, 128 6.0 8.8; 5120 x 5120: 1 8.4 6.6, 64 8.9 8.6, 128 9.7 10.5; 1280 x
  // 5120, also in four: 32 8.4 7.4 5.8, 128 9.4 10.1 7.5).  Clusters of four find room on 128 SMs, of two on all.
  auto cost = [&](int pieces) { return 290 * p.k_blocks / pieces + (pieces > 1 ? 1400 + 40 * p.rows / pieces : 0); };
  p.pieces = 1;
  if (p.tiles * 2 <= kSms && p.k_blocks >= 2 && cost(2) < cost(1)) p.pieces = 2;
  if (p.tiles * 4 <= 128 && p.k_blocks >= 4 && cost(4) < cost(p.pieces)) p.pieces = 4;
  auto kern = few_rows_kernel<T, kFormat>;
  const int smem = std::max(p.stages * p.stage_bytes, p.columns * kRows * 4) + 1024;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, smem));
  SPARSP_CUDA_OK(launch_clusters(kern, dim3((unsigned)std::min(p.tiles * p.pieces, kSms)), p.pieces, kFewThreads,
                                 (size_t)smem, st, ma, mb, msa, msb, p));
  return SPARSP_OK;
}

template <typename T, int kFormat, int BN>
static int launch_pairs(const sparsp_fp4_gemm& f, const void* A, const void* As, const void* B, const void* Bs,
                        const void* bias, void* C, char* ws, cudaStream_t st) {
  using Cfg = ProductCfg<kFormat, T, BN>;
  const int64_t groups = fp4_groups(f.depth, kFormat);
  CUtensorMap ma, mb, msa, msb, mc;
  int rc;
  if ((rc = make_codes_map(&ma, A, f.rows, f.depth / 2, kRows)) != SPARSP_OK) return rc;
  if ((rc = make_codes_map(&mb, B, f.cols, f.depth / 2, BN / 2)) != SPARSP_OK) return rc;
  if ((rc = make_scales_map(&msa, As, f.rows, groups, Cfg::kGroups, 1)) != SPARSP_OK) return rc;
  if ((rc = make_scales_map(&msb, Bs, f.cols, groups, Cfg::kGroups, Cfg::kTilesB)) != SPARSP_OK) return rc;
  if ((rc = make_result_map(&mc, f.dtype, C, f.rows, f.cols, f.stride_c)) != SPARSP_OK) return rc;
  ProductParams p = {};
  p.bias = bias;
  p.rows = (int32_t)f.rows;
  p.cols = f.cols;
  p.depth = f.depth;
  p.m_tiles = ceil_div(f.rows, 256);
  p.n_tiles = ceil_div(f.cols, BN);
  // row tiles in a band, whose tiles go column by column: those at work at one time share rows of A and of B in L2 (75600 x
  // 13824 x 5120 and x 5120 x 13824 nvfp4, bands of 4 2425 and 2162 us, 8 2373 and 2236, 16 2291 and 2190, 37 2284 and 2486)
  p.band = 16;
  p.k_blocks = ceil_div(f.depth, kDeep);
  p.factor = std::ldexp(1.0f, f.exponent);
  p.idesc = fp4_instruction(kFormat, 256, BN);
  p.status = reinterpret_cast<int32_t*>(ws);
  p.wait_limit = kWaitLimit;
  p.tile_limit = kWaitLimit + kStageLimit * p.k_blocks;
  auto kern = product_kernel<T, kFormat, BN>;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, Cfg::kDynamic));
  const unsigned grid = 2u * (unsigned)std::min(p.m_tiles * p.n_tiles, kPairs);
  SPARSP_CUDA_OK(launch_clusters(kern, dim3(grid), 2, kProductThreads, Cfg::kDynamic, st, ma, mb, msa, msb, mc, p));
  return SPARSP_OK;
}

// Tiles of 128 columns where these make fewer rounds: a round of them takes 0.7 of one of 256, for each value that they load
// serves fewer products (us, 256 and 128 columns: 226 x 7680 x 1920 6.8 and 6.1, 1003 x 1160 x 5120 10.6 and 8.9, one round of
// either; 1000 x 7680 x 1920, two and four rounds, 11.1 and 13.2; 2000 x 5120 x 5120, three and five, 28.5 and 30.1).
static bool narrow_tiles(const sparsp_fp4_gemm& f) {
  const int64_t m = ceil_div(f.rows, 256);
  return 128 * 7 * ceil_div(m * ceil_div(f.cols, 128), kPairs) < 256 * 5 * ceil_div(m * ceil_div(f.cols, 256), kPairs);
}

template <typename T, int kFormat>
static int launch_product(const sparsp_fp4_gemm& f, const void* A, const void* As, const void* B, const void* Bs,
                          const void* bias, void* C, char* ws, cudaStream_t st) {
  if (f.rows <= kFewRows) return launch_few_rows<T, kFormat>(f, A, As, B, Bs, bias, C, ws, st);
  return narrow_tiles(f) ? launch_pairs<T, kFormat, 128>(f, A, As, B, Bs, bias, C, ws, st)
                         : launch_pairs<T, kFormat, 256>(f, A, As, B, Bs, bias, C, ws, st);
}

int launch_fp4_product(const sparsp_fp4_gemm& f, const void* A, const void* As, const void* B, const void* Bs,
                       const void* bias, void* C, char* ws, cudaStream_t st) {
  if ((int64_t)ceil_div(f.rows, 256) * ceil_div(f.cols, 128) > (1 << 30)) {
    set_error("%d x %d tiles are too many", ceil_div(f.rows, 256), ceil_div(f.cols, 128));
    return SPARSP_ERR_UNSUPPORTED;
  }
  SPARSP_WITH_TYPE(f.dtype, T, {
    return f.format == SPARSP_MXFP4 ? launch_product<T, SPARSP_MXFP4>(f, A, As, B, Bs, bias, C, ws, st)
                                    : launch_product<T, SPARSP_NVFP4>(f, A, As, B, Bs, bias, C, ws, st);
  });
}

}  // namespace sparsp
