// Gated feed-forward: H = a(X Wg^T) * (X Wu^T) in one kernel, and its backward pass.
//
// All three products are one matrix kernel.  A pair of CTAs (a cluster of two, tcgen05 cta_group::2) makes a 256-row
// tile of the result: each CTA loads 128 of its rows of A and half of its columns of B by TMA, the even CTA issues the
// MMAs for both, and each finds its 128 rows, all columns, as fp32 in its own tensor memory.
//   forward   A = X (K-major), B = half a tile of Wg's rows in one CTA and the same rows of Wu in the other: the tile's
//             columns are gate and up of the same features, and the activation and the product happen between tensor
//             memory and the store.
//   dX        A = dG then dU (K-major), B = Wg then Wu as they lie (MN-major): the sum over both is one accumulation.
//   dW        A = dG^T or dU^T (MN-major), B = X (MN-major); summed over tokens.
// dG and dU, which the last two read, are made element by element before them, rounded to 16 bits.  Where there are few
// tokens those roundings do not average out over many results, and time goes into the weights, not into products: then
// both are in two parts, the rounded value and what it leaves, one 128 rows behind the other.  dX takes the two parts
// as the two halves of its 256-row tile and adds them when the pieces of K are added, dW as more tokens.
//
// Bound by the tensor cores and by power where all sizes are large.  A single launch of 8192 x 5120 x 6912 bf16, both
// projections kept, has them busy for 97.9 % of its cycles, at 1.38 GHz.  In a loop of seconds, at 980 to 990 W: 37800
// x 5120 x 13824, both kept, 8.09 ms = 1320 TFLOP/s at a median of 1.21 GHz, so that the 8.85 million clocks of its
// products are 91 % of the time; backward 20.1 ms = 1065 TFLOP/s at 1.00 GHz, 88 % (17.1 to 20.3 ms over GPUs and
// shorter loops).
#include <algorithm>
#include <cmath>

#include "layer.cuh"
#include "sm100_ptx.cuh"

namespace sparsp {

enum GemmMode { kForward, kInput, kWeights };

struct GemmParams {
  void* out[2];           // kForward: H;  kInput: dX;  kWeights: dWg, dWu
  void* keep[2];          // kForward: gate, up or NULL
  float* partial;         // sums of pieces of K
  int64_t ld_out;         // elements from row to row of out and keep
  int32_t rows, cols;     // of the result (kForward: tokens, hidden; kInput: tokens, dim; kWeights: hidden, dim)
  int32_t m_tiles, n_tiles, band;
  int32_t whole, shares;  // see Walk
  int32_t two_parts;      // dG and dU are in two parts
  int32_t alternate;      // half the warps of a CTA take every other tile's results
  int32_t k_blocks;       // of 64, of one (A, B); kInput has two of them
  int32_t activation;
  uint32_t idesc;
  int32_t* status;
  long long wait_limit;
};

constexpr int kStageK = 64;           // K elements of a stage: one 128-byte swizzled row
constexpr int kEpilogueWarps = 16;    // four for each quarter of the lanes (256 x 2048 x 9472: 16.7 us, 18.3 with two)
constexpr int kGemmThreads = 32 * (kEpilogueWarps + 2);
constexpr int kTileRows = 128;        // of one CTA
constexpr int kFewTokens = 128;       // up to so many tokens go their own ways

// BN: columns of the accumulator, and of B over both CTAs.
template <int BN>
struct GemmCfg {
  static constexpr int kA = kTileRows * 128, kB = BN / 2 * 128;  // bytes a stage of one CTA
  static constexpr int kStage = kA + kB;
  static constexpr int kStages = 196608 / kStage > 8 ? 8 : 196608 / kStage;
  static constexpr int kOffOut = kStages * kStage;  // each epilogue warp's 32 rows x 32 columns on their way out
  static constexpr int kOffBars = kOffOut + kEpilogueWarps * 2048;
  static constexpr int kBars = 2 * kStages + 5;
  static constexpr int kBytes = kOffBars + kBars * 8 + 16;
  static constexpr int kDynamic = kBytes + 1024;  // the tiles are aligned to 1024 bytes
};

// 1 / (1 + 2^t): with t = -x log2 e, the logistic function of x.  Far out on either side it is 1 or 0.
__device__ __forceinline__ float logistic2(float t) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + ptx::ex2(t)));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kTanhA = 2.0f * 0.7978845608028654f, kTanhB = 0.044715f;  // (1 + tanh(u)) / 2 = logistic(2 u)

// (1 + erf(x / sqrt 2)) / 2, and e = exp(-x^2 / 2), which the slope needs too: with z = |x| / sqrt 2 and t = 1 / (1 +
// 3/8 z), the way of Abramowitz and Stegun 7.1.26, erfc(z) / 2 is e times a polynomial in t, fitted here to the least
// largest relative error: 2^-20 for every x whose e is above zero.  Their five terms, made for a small absolute error,
// are off by 0.05 % at x = -4 and 0.4 % at -6, which 16-bit results show.  A forward call of 16384 x 64 x 9472 takes
// 168 us (160 with five terms, 217 with the library's erff; in pairs of values by f32x2 instructions 167).
__device__ __forceinline__ float normal_below(float x, float& e) {
  const float z = fabsf(x) * 0.70710678118654752f;
  e = ptx::ex2(z * z * -kLog2e);
  float t;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(z, 0.375f, 1.0f)));
  float q = fmaf(t, -0.06754766983f, 0.19396793736f);
  q = fmaf(t, q, -0.06479728835f);
  q = fmaf(t, q, 0.14152977980f);
  q = fmaf(t, q, 0.08333265443f);
  q = fmaf(t, q, 0.10784451822f);
  q = fmaf(t, q, 0.10566972979f) * t * e;
  return x < 0.0f ? q : 1.0f - q;
}

// a(x), and a(x) with a'(x).  a(x) is within 2^-16 of itself as far down as x = -6 (roundings of the exponent's
// argument).
template <int kKind>
__device__ __forceinline__ float activate(float x) {
  if constexpr (kKind == SPARSP_ACT_SILU) return x * logistic2(-kLog2e * x);
  if constexpr (kKind == SPARSP_ACT_GELU_TANH)
    return x * logistic2(x * fmaf(x * x, -kLog2e * kTanhA * kTanhB, -kLog2e * kTanhA));
  float e;
  return x * normal_below(x, e);
}
template <int kKind>
__device__ __forceinline__ void activate(float x, float& a, float& slope) {
  if constexpr (kKind == SPARSP_ACT_SILU) {
    const float s = logistic2(-kLog2e * x);
    a = x * s;
    slope = s * (1.0f + x * (1.0f - s));
  } else if constexpr (kKind == SPARSP_ACT_GELU_TANH) {
    const float s = logistic2(x * fmaf(x * x, -kLog2e * kTanhA * kTanhB, -kLog2e * kTanhA));
    a = x * s;
    const float t = s * (1.0f - s);
    slope = t == 0.0f ? s : s + x * t * kTanhA * (1.0f + 3.0f * kTanhB * x * x);  // far out x * x may be infinite
  } else {
    float e;
    const float c = normal_below(x, e);
    a = x * c;
    slope = c + x * 0.3989422804014327f * e;
  }
}
// Runs f with the kind as a constant.
template <typename F>
__device__ __forceinline__ void with_activation(int kind, F f) {
  if (kind == SPARSP_ACT_SILU)
    f(std::integral_constant<int, SPARSP_ACT_SILU>());
  else if (kind == SPARSP_ACT_GELU_TANH)
    f(std::integral_constant<int, SPARSP_ACT_GELU_TANH>());
  else
    f(std::integral_constant<int, SPARSP_ACT_GELU>());
}
// h = a(g) u
template <int N>
__device__ __forceinline__ void gate_product(int kind, const float (&g)[N], const float (&u)[N], float (&h)[N]) {
  with_activation(kind, [&](auto k) {
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = activate<decltype(k)::value>(g[i]) * u[i];
  });
}

// One thread, before shared and tensor memory are given back: waits, within a limit, for the products issued here.
__device__ __forceinline__ void wait_drained(uint64_t* drained, long long limit) {
  const long long t0 = clock64();
  while (!ptx::mbar_try_wait(drained, 0) && clock64() - t0 < limit) {
  }
}

// A warp's 32 rows x 32 columns to global memory: staged in its own 2 KB (64-byte swizzle: a row's 16-byte pieces in
// turned places, so that lanes do not meet in a bank) and stored as one TMA tile, which writes whole sectors and leaves
// out what lies beyond the tensor.  16-byte stores from the registers, a row each, cost a forward call of 37800 x 5120
// x 13824 that keeps its projections 9305 us.
template <typename T>
__device__ __forceinline__ void write_out(const CUtensorMap* to, uint8_t* mine, const float (&x)[32], int lane, int col,
                                          int row, int cols, int rows) {
  uint32_t words[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) words[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
  if (lane == 0) ptx::tma_store_wait_read();
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 4; ++e)
    *reinterpret_cast<uint4*>(mine + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
        make_uint4(words[4 * e], words[4 * e + 1], words[4 * e + 2], words[4 * e + 3]);
  ptx::fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0 && col < cols && row < rows) {
    ptx::tma_store_2d(to, mine, col, row);
    ptx::tma_store_commit();
  }
}

// Tiles go in bands of `band` row tiles, column by column inside a band, so that the tiles at work at one time share
// both their rows of A and their columns of B in L2 (37800 x 5120 x 13824: bands of 4 to 24 are alike within 1 %).
__device__ __forceinline__ void tile_at(const GemmParams& p, int tile, int& m, int& n) {
  const int per_band = p.band * p.n_tiles;
  const int b = tile / per_band, in = tile - b * per_band;
  const int height = min(p.band, p.m_tiles - b * p.band);
  n = in / height;
  m = b * p.band + in - n * height;
}

// What a pair of CTAs works on.  The first `whole` tiles go to the pairs round by round; of the K blocks of the rest,
// which would leave pairs without a tile, each of the first `shares` pairs has an equal run, so that a tile's sums are
// in pieces that gemm_join_kernel adds.  A run is no longer than a tile and touches two at most.
struct Walk {
  int tile, k0, k1, slot;  // at work: tile, blocks of K, and where to put the sums (-1: the whole tile is done)
  int next_whole, pairs, whole, blocks, lo, hi, next_slot;
  bool always;  // sums go through a slot even where a pair has all of a tile
  __device__ __forceinline__ Walk(const GemmParams& p, int blocks, int pair, int pairs, bool adds_halves)
      : next_whole(pair), pairs(pairs), whole(p.whole), blocks(blocks), lo(0), hi(0), next_slot(2 * pair),
        always(adds_halves) {
    if (pair < p.shares) {
      lo = share_begin(p, blocks, pair);
      hi = share_begin(p, blocks, pair + 1);
    }
  }
  // first of the rest's K blocks that pair q has
  static __device__ __forceinline__ int share_begin(const GemmParams& p, int blocks, int q) {
    return (int)((int64_t)(p.m_tiles * p.n_tiles - p.whole) * blocks * q / p.shares);
  }
  __device__ __forceinline__ bool next() {
    if (next_whole < whole) {
      tile = next_whole;
      next_whole += pairs;
      k0 = 0;
      k1 = blocks;
      slot = -1;
      return true;
    }
    if (lo >= hi) return false;
    const int r = lo / blocks;
    tile = whole + r;
    k0 = lo - r * blocks;
    k1 = min(blocks, k0 + hi - lo);
    slot = k1 - k0 == blocks && !always ? -1 : next_slot;
    ++next_slot;
    lo += k1 - k0;
    return true;
  }
};

// One product, by pairs of CTAs `pair` of `pairs`; maps: A (two), B (two), results (up to three).
template <typename T, int kMode, int BN>
__device__ __forceinline__ void gemm_tiles(const CUtensorMap& a0, const CUtensorMap& a1, const CUtensorMap& b0,
                                           const CUtensorMap& b1, const CUtensorMap& o0, const CUtensorMap& o1,
                                           const CUtensorMap& o2, const GemmParams p, const int pair,
                                           const int pairs) {
  using namespace ptx;
  using C = GemmCfg<BN>;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kOffBars);  // of the even CTA: both CTAs' tiles have arrived
  uint64_t* empty = full + C::kStages;                               // the stage has been multiplied
  uint64_t* acc_full = empty + C::kStages;                           // [2]
  uint64_t* acc_empty = acc_full + 2;                                // [2] of the even CTA: both have read theirs
  uint64_t* drained = acc_empty + 2;                                 // every product has ended
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
      mbar_init(acc_empty + a, p.alternate ? kEpilogueWarps : 2 * kEpilogueWarps);
    }
    mbar_init(drained, 1);
    *s_abort = 0;
    mbar_init_fence();
  }
  if (warp == kEpilogueWarps + 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  enter_grid();  // (the next launch may begin: tensor memory is ours, so its CTAs cannot have taken it before)

  Walk walk(p, p.k_blocks * (kMode == kInput ? 2 : 1), pair, pairs, kMode == kInput && p.two_parts);
  constexpr bool kAMn = kMode == kWeights, kBMn = kMode != kForward;

  if (warp == kEpilogueWarps) {
    // ---- loads ----
    if (elect_one()) {
      uint32_t full_of_even[C::kStages];
#pragma unroll
      for (int s = 0; s < C::kStages; ++s) full_of_even[s] = cluster_addr(full + s, 0);
      int s = 0;
      uint32_t round = 0;
      while (!*s_abort && walk.next()) {
        int m, n;
        tile_at(p, walk.tile, m, n);
        const int half_m = p.m_tiles / 2;  // kWeights: the tiles of dWg, then those of dWu
        const CUtensorMap* ta = &a0;
        int row = (m * 2 + (int)rank) * kTileRows;
        if (kMode == kWeights && m >= half_m) {
          ta = &a1;
          row -= half_m * 2 * kTileRows;
        }
        for (int k = walk.k0; k < walk.k1; ++k) {
          mbar_wait_bounded_inline(empty + s, round ^ 1u, s_abort, 1, p.wait_limit);
          if (*s_abort) break;
          if (rank == 0) mbar_expect_tx(full + s, 2 * C::kStage);
          uint8_t* A = smem + s * C::kStage;
          uint8_t* B = A + C::kA;
          uint32_t bar = 0;
#pragma unroll
          for (int q = 0; q < C::kStages; ++q)
            if (q == s) bar = full_of_even[q];
          const bool second = kMode == kInput && k >= p.k_blocks;
          const bool left = kMode == kWeights && p.two_parts && k >= p.k_blocks / 2;  // what the rounding left
          const int kk = (second ? k - p.k_blocks : left ? k - p.k_blocks / 2 : k) * kStageK;
          if constexpr (kAMn) {
            const int token = left ? kFewTokens + kk : kk;
            tma_load_pair(A, ta, bar, row, token);
            tma_load_pair(A + 8192, ta, bar, row + 64, token);
          } else {
            tma_load_pair(A, second ? &a1 : &a0, bar, kk, row);
          }
          if constexpr (!kBMn) {
            tma_load_pair(B, rank == 0 ? &b0 : &b1, bar, kk, n * (BN / 2));
          } else {
            const CUtensorMap* tb = second || left ? &b1 : &b0;
#pragma unroll
            for (int c = 0; c < BN / 128; ++c)
              tma_load_pair(B + c * 8192, tb, bar, n * BN + (int)rank * (BN / 2) + c * 64, kk);
          }
          if (++s == C::kStages) {
            s = 0;
            round ^= 1u;
          }
        }
      }
      // Copies still in flight after a wait that ran out are waited for, within the same limit: each stage's last
      // phase.
      if (*s_abort && rank == 0) {
        const long long t0 = clock64();
        for (int q = 0; q < C::kStages; ++q) {
          const uint32_t phase = q < s ? round : round ^ 1u;
          while (!mbar_try_wait(full + q, phase) && clock64() - t0 < p.wait_limit) {
          }
        }
      }
    }
  } else if (warp == kEpilogueWarps + 1) {
    // ---- products, for both CTAs ----
    if (rank == 0 && elect_one()) {
      const uint32_t base = smem_u32(smem);
      const uint64_t da = make_smem_desc(base, kAMn ? 8192u : 16u, 1024u);
      const uint64_t db = make_smem_desc(base + C::kA, kBMn ? 8192u : 16u, 1024u);
      constexpr uint32_t kStepA = kAMn ? 2048 : 32, kStepB = kBMn ? 2048 : 32;  // 16 elements of K
      int s = 0, acc = 0;
      uint32_t round = 0, acc_round = 0;
      while (!*s_abort && walk.next()) {
        mbar_wait_bounded_inline(acc_empty + acc, acc_round ^ 1u, s_abort, 2, p.wait_limit);
        tc_fence_after();
        for (int k = walk.k0; k < walk.k1; ++k) {
          if (!mbar_wait_bounded_inline(full + s, round, s_abort, 3, p.wait_limit)) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)((s * C::kStage) >> 4);
#pragma unroll
          for (int kk = 0; kk < kStageK / 16; ++kk)
            mma_ss_pair(tmem + acc * BN, da + off + (kk * kStepA >> 4), db + off + (kk * kStepB >> 4), p.idesc,
                        k > walk.k0 || kk > 0);
          mma_commit_pair(empty + s);
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
    // ---- results: warp w has the lanes of quarter w % 4, and a share of the columns ----
    // With one tile or two a pair, all warps do each; with more, eight warps do one tile while eight do the next, so
    // that one tile's loads and stores fill the time of the other's exponentials (2825 x 96 x 5456: 21.0 us, all
    // together 24.5; 1024 x 512 x 2048, fewer than two tiles a pair: 9.2 all together, 9.6 in turn).
    const int quarter = warp & 3, sides = p.alternate ? 2 : 4, side = (warp >> 2) % sides;
    const int turn = p.alternate ? warp >> 3 : -1;
    uint8_t* mine = smem + C::kOffOut + warp * 2048;
    int acc = 1;
    uint32_t acc_round = 1;
    const uint32_t even0 = cluster_addr(acc_empty, 0), even1 = cluster_addr(acc_empty + 1, 0);
    while (walk.next()) {
      acc ^= 1;
      if (acc == 0) acc_round ^= 1u;
      if (turn == (acc ^ 1)) continue;
      int m, n;
      tile_at(p, walk.tile, m, n);
      mbar_wait_bounded_inline(acc_full + acc, acc_round, s_abort, 4, p.wait_limit);
      if (__any_sync(0xffffffffu, *s_abort != 0)) break;  // (the same for all lanes)
      tc_fence_after();
      const uint32_t from = tmem + acc * BN + ((uint32_t)(quarter * 32) << 16);
      // after a warp's last load: the next product may have these columns while it is still busy with the values
      auto release = [&](bool last) {
        if (!last) return;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(acc == 0 ? even0 : even1);
      };
      const int in_tile = (int)rank * kTileRows + quarter * 32 + lane;
      if (walk.slot >= 0) {
        // [slot][BN / 4][256 rows] of four columns: lanes are rows, so a warp writes 512 bytes in a piece
        float4* to = reinterpret_cast<float4*>(p.partial) + (int64_t)walk.slot * (BN / 4) * 256 + in_tile;
#pragma unroll 1
        for (int c = side * (BN / sides); c < (side + 1) * (BN / sides); c += 32) {
          uint32_t r[32];
          tmem_ld32(from + c, r);
          tmem_ld_wait(r);
          release(c + 32 == (side + 1) * (BN / sides));
#pragma unroll
          for (int e = 0; e < 8; ++e)
            to[(c / 4 + e) * 256] = make_float4(__uint_as_float(r[4 * e]), __uint_as_float(r[4 * e + 1]),
                                                __uint_as_float(r[4 * e + 2]), __uint_as_float(r[4 * e + 3]));
        }
      } else if constexpr (kMode == kForward) {
        const int row = m * 256 + (int)rank * kTileRows + quarter * 32;
#pragma unroll 1
        for (int c = side * (BN / 2 / sides); c < (side + 1) * (BN / 2 / sides); c += 32) {
          float g[32], u[32];
          tmem_ld32(from + c, reinterpret_cast<uint32_t*>(g));
          tmem_ld32(from + BN / 2 + c, reinterpret_cast<uint32_t*>(u));
          tmem_ld_wait(g);
          tmem_ld_wait(u);
          release(c + 32 == (side + 1) * (BN / 2 / sides));
          const int col = n * (BN / 2) + c;
          if (p.keep[0] != nullptr) {
            write_out<T>(&o1, mine, g, lane, col, row, p.cols, p.rows);
            write_out<T>(&o2, mine, u, lane, col, row, p.cols, p.rows);
          }
          gate_product(p.activation, g, u, g);
          write_out<T>(&o0, mine, g, lane, col, row, p.cols, p.rows);
        }
      } else {
        const int half_m = p.m_tiles / 2;
        const bool second = kMode == kWeights && m >= half_m;
        const int row = (second ? m - half_m : m) * 256 + (int)rank * kTileRows + quarter * 32;
#pragma unroll 1
        for (int c = side * (BN / sides); c < (side + 1) * (BN / sides); c += 32) {
          float x[32];
          tmem_ld32(from + c, reinterpret_cast<uint32_t*>(x));
          tmem_ld_wait(x);
          release(c + 32 == (side + 1) * (BN / sides));
          write_out<T>(second ? &o1 : &o0, mine, x, lane, n * BN + c, row, p.cols, p.rows);
        }
      }
    }
    if (lane == 0) tma_store_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  // Products use both CTAs' memory until they have ended: after a wait that ran out nobody else has waited for them.
  if (warp == kEpilogueWarps + 1 && elect_one()) wait_drained(drained, p.wait_limit);
  __syncwarp();
  cluster_sync();  // the other CTA's arrivals and products here have ended
  if (warp == kEpilogueWarps + 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
  if (threadIdx.x == 0) report_abort(s_abort, p.status);
}

template <typename T, int kMode, int BN>
__global__ void __launch_bounds__(kGemmThreads, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1,
                const __grid_constant__ CUtensorMap o0, const __grid_constant__ CUtensorMap o1,
                const __grid_constant__ CUtensorMap o2, const GemmParams p) {
  gemm_tiles<T, kMode, BN>(a0, a1, b0, b1, o0, o1, o2, p, blockIdx.x >> 1, gridDim.x >> 1);
}

struct GemmMaps {
  CUtensorMap a0, a1, b0, b1, o0, o1, o2;
};

// dX and dW at once: the first `split` pairs make the one, the others the other.
template <typename T, int BN>
__global__ void __launch_bounds__(kGemmThreads, 1)
    gemm_both_kernel(const __grid_constant__ GemmMaps mi, const GemmParams pi,
                     const __grid_constant__ GemmMaps mw, const GemmParams pw, const int split) {
  const int pair = blockIdx.x >> 1;
  if (pair < split)
    gemm_tiles<T, kInput, BN>(mi.a0, mi.a1, mi.b0, mi.b1, mi.o0, mi.o1, mi.o2, pi, pair, split);
  else
    gemm_tiles<T, kWeights, BN>(mw.a0, mw.a1, mw.b0, mw.b1, mw.o0, mw.o1, mw.o2, pw, pair - split,
                                (gridDim.x >> 1) - split);
}

// ---- few tokens -----------------------------------------------------------------------------------------------------
//
// With a handful of tokens the call is one pass over the weights, and a 256-row tile of tokens would be all padding.
// Here the weights are the rows of the tile and the tokens its columns: D = [Wg; Wu] X^T, 2 F rows (F features of gate,
// then the same of up) by N columns (the tokens, rounded up to 16).  A CTA has F features at a time, F as small as
// shares the hidden size out evenly; the MMA takes 128 rows all the same, and those past 2 F are whatever lies behind
// in shared memory and are never read.  Gate and up of a feature are in different lanes, so they meet in shared memory,
// where the order turns to tokens by features for the store.  Where there are so few features that most SMs would have
// none, a cluster of CTAs shares out K for each tile, and each adds a part of the results from the others' shared
// memory. Bound by HBM: 1 x 5120 x 13824 bf16 45 to 47 us = 6.0 to 6.3 TB/s, by L2 where the weights are there already.
struct FewParams {
  void* out;
  void* keep[2];
  int64_t ld_out;
  int32_t tokens, hidden;
  int32_t features, columns;  // of a tile: F, N
  int32_t tiles, k_blocks, stages, stage_bytes, ld_turn;
  int32_t splits;  // CTAs of a cluster that share out K; each then has one tile at most
  int32_t activation;
  uint32_t idesc;
  int32_t* status;
  long long wait_limit;
};

constexpr int kFewThreads = 192;  // loads, products, four warps of results
constexpr int kFewSmem = 224 * 1024;

template <typename T, int kDeep>
__global__ void __launch_bounds__(kFewThreads, 1)
    few_kernel(const __grid_constant__ CUtensorMap mg, const __grid_constant__ CUtensorMap mu,
               const __grid_constant__ CUtensorMap mx, const FewParams p) {
  using namespace ptx;
  extern __shared__ uint8_t dynamic[];
  uint8_t* smem = dynamic + ((1024 - (smem_u32(dynamic) & 1023)) & 1023);
  __shared__ uint64_t full[16], empty[16], acc_full[2], acc_empty[2], drained;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  volatile int* s_abort = &abort_word;
  // behind the stages: room for the last stage's rows past 2 F, then the results on their turn
  float* turn = reinterpret_cast<float*>(smem + p.stages * p.stage_bytes + 16384);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + a, 1);
      mbar_init(acc_empty + a, 4);
    }
    mbar_init(&drained, 1);
    *s_abort = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_slot, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  enter_grid();  // (after tensor memory is ours, as above)
  const int F = p.features, N = p.columns;
  const int rank = (int)cluster_rank(), first_tile = blockIdx.x / p.splits, step = gridDim.x / p.splits;
  const int k0 = p.k_blocks * rank / p.splits, k1 = p.k_blocks * (rank + 1) / p.splits;

  if (warp == 0) {
    if (elect_one()) {
      int s = 0;
      uint32_t round = 0;
      const int block = (2 * F + N) * 128;
      for (int tile = first_tile; tile < p.tiles && !*s_abort; tile += step) {
        for (int k = k0; k < k1; k += kDeep) {
          if (!mbar_try_wait(empty + s, round ^ 1u)) {
            mbar_wait_bounded_inline(empty + s, round ^ 1u, s_abort, 11, p.wait_limit);
            if (*s_abort) break;
          }
          uint8_t* at = smem + s * p.stage_bytes;
          const int n = min(kDeep, k1 - k);
          mbar_expect_tx(full + s, n * block);
#pragma unroll
          for (int q = 0; q < kDeep; ++q)
            if (q < n) tma_load_2d(at + q * block, &mg, full + s, (k + q) * kStageK, tile * F);
#pragma unroll
          for (int q = 0; q < kDeep; ++q)
            if (q < n) tma_load_2d(at + q * block + F * 128, &mu, full + s, (k + q) * kStageK, tile * F);
#pragma unroll
          for (int q = 0; q < kDeep; ++q)
            if (q < n) tma_load_2d(at + q * block + 2 * F * 128, &mx, full + s, (k + q) * kStageK, 0);
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
      const uint64_t da = make_smem_desc(smem_u32(smem), 16u, 1024u);
      const uint64_t db = make_smem_desc(smem_u32(smem) + 2 * F * 128, 16u, 1024u);
      const int block = (2 * F + N) * 128;
      int s = 0, acc = 0;
      uint32_t round = 0, acc_round = 0;
      for (int tile = first_tile; tile < p.tiles && !*s_abort; tile += step) {
        mbar_wait_bounded_inline(acc_empty + acc, acc_round ^ 1u, s_abort, 12, p.wait_limit);
        tc_fence_after();
        for (int k = k0; k < k1; k += kDeep) {
          if (!mbar_wait_bounded_inline(full + s, round, s_abort, 13, p.wait_limit)) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)((s * p.stage_bytes) >> 4);
#pragma unroll
          for (int q = 0; q < kDeep; ++q)
            if (q < k1 - k) {
#pragma unroll
              for (int kk = 0; kk < kStageK / 16; ++kk)
                mma_ss(tmem + acc * kFewTokens, da + off + (q * block >> 4) + kk * 2, db + off + (q * block >> 4) + kk * 2,
                       p.idesc, k + q > k0 || kk > 0);
            }
          mma_commit(empty + s);
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
      wait_drained(&drained, p.wait_limit);  // (as above)
    }
  } else {
    const int quarter = warp & 3, in_tile = quarter * 32 + lane;
    const int ld = p.ld_turn;  // of `turn`, a row for each lane: odd, so that its columns do not meet in a bank
    int acc = 0;
    uint32_t acc_round = 0;
    // No way out before the last tile: the four warps meet at barrier 1 twice a tile, so all of them have to come, also
    // after a wait that ran out, when one may see the flag before another does.  Waits return at once then.
    for (int tile = first_tile; tile < p.tiles; tile += step) {
      mbar_wait_bounded_inline(acc_full + acc, acc_round, s_abort, 14, p.wait_limit);
      tc_fence_after();
      if (quarter * 32 < 2 * F) {
        for (int c = 0; c < N; c += 16) {
          uint32_t r[16];
          tmem_ld16(tmem + acc * kFewTokens + c + ((uint32_t)(quarter * 32) << 16), r);
          tmem_ld_wait(r);
          if (in_tile < 2 * F) {
#pragma unroll
            for (int i = 0; i < 16; ++i) turn[in_tile * ld + c + i] = __uint_as_float(r[i]);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_empty + acc);
      asm volatile("bar.sync 1, 128;" ::: "memory");
      // eight features of a token a thread
      const int per_row = F / 8;
      for (int i = threadIdx.x - 64; p.splits == 1 && i < p.tokens * per_row; i += 128) {
        const int token = i / per_row, f = (i - token * per_row) * 8, col = tile * F + f;
        if (col >= p.hidden) continue;
        float g[8], u[8], h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          g[e] = turn[(f + e) * ld + token];
          u[e] = turn[(F + f + e) * ld + token];
        }
        gate_product(p.activation, g, u, h);
        const int64_t at = token * p.ld_out + col;
        Vec<T, 8> v;
        v.set(h);
        store_vec(reinterpret_cast<T*>(p.out) + at, v);
        if (p.keep[0] != nullptr) {
          v.set(g);
          store_vec(reinterpret_cast<T*>(p.keep[0]) + at, v);
          v.set(u);
          store_vec(reinterpret_cast<T*>(p.keep[1]) + at, v);
        }
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      acc ^= 1;
      if (acc == 0) acc_round ^= 1u;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (p.splits > 1) {
    cluster_sync();  // the sums of all pieces of K are there
    // two features of a token a thread; each piece's four sums are under way together
    const uint32_t mine = smem_u32(turn);
    for (int i = rank * kFewThreads + threadIdx.x; i < p.tokens * (F / 2); i += p.splits * kFewThreads) {
      const int token = i / (F / 2), f = (i - token * (F / 2)) * 2, col = first_tile * F + f;
      if (col >= p.hidden) continue;
      float g[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f}, h[2];
#pragma unroll 2
      for (int r = 0; r < p.splits; ++r) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[e] = ld_cluster(mine + ((f + (e & 1) + (e < 2 ? 0 : F)) * p.ld_turn + token) * 4, r);
        g[0] += x[0];
        g[1] += x[1];
        u[0] += x[2];
        u[1] += x[3];
      }
      gate_product(p.activation, g, u, h);
      const int64_t at = token * p.ld_out + col;
      *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(p.out) + at) = pack2<T>(h[0], h[1]);
      if (p.keep[0] != nullptr) {
        *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(p.keep[0]) + at) = pack2<T>(g[0], g[1]);
        *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(p.keep[1]) + at) = pack2<T>(u[0], u[1]);
      }
    }
    cluster_sync();  // nobody leaves while others read here
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
  if (threadIdx.x == 0) report_abort(s_abort, p.status);
}

// Adds the pieces of a tile, in the order of K, and finishes it as gemm_kernel would have.  A thread has one row and
// eight columns (for the forward call of both projections).
template <typename T, int kMode, int BN>
__device__ __forceinline__ void join_tile(const GemmParams p, int cta) {
  const float* partial = p.partial;
  constexpr int kCols = kMode == kForward ? BN / 2 : BN;  // result columns of a tile
  const int rest = cta / (kCols / 8), c = (cta % (kCols / 8)) * 8;
  const int blocks = p.k_blocks * (kMode == kInput ? 2 : 1), lo = rest * blocks, hi = lo + blocks;
  // pairs with blocks lo .. hi - 1; the first may have begun in the tile before, and has this one in its second slot
  // then
  int q = (int)((int64_t)lo * p.shares / ((int64_t)(p.m_tiles * p.n_tiles - p.whole) * blocks));
  while (q > 0 && Walk::share_begin(p, blocks, q) > lo) --q;
  while (Walk::share_begin(p, blocks, q + 1) <= lo) ++q;
  const bool halves = kMode == kInput && p.two_parts;  // rows 128 and on belong to those 128 before
  if (halves ? threadIdx.x >= kFewTokens
             : Walk::share_begin(p, blocks, q) <= lo && Walk::share_begin(p, blocks, q + 1) >= hi)
    return;  // one pair had it all
  int m, n;
  tile_at(p, p.whole + rest, m, n);
  float v[8], u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = u[i] = 0.0f;
  const int first = 2 * q + (Walk::share_begin(p, blocks, q) < lo ? 1 : 0);
  int pieces = 1;
  while (q + pieces < p.shares && Walk::share_begin(p, blocks, q + pieces) < hi) ++pieces;
#pragma unroll 4
  for (int i = 0; i < pieces; ++i) {
    const float4* from = reinterpret_cast<const float4*>(partial) +
                         (int64_t)(i == 0 ? first : 2 * (q + i)) * (BN / 4) * 256 + threadIdx.x;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 x = from[(c / 4 + h) * 256];
      v[4 * h] += x.x;
      v[4 * h + 1] += x.y;
      v[4 * h + 2] += x.z;
      v[4 * h + 3] += x.w;
      if (halves) {  // what the roundings left, of either sign, times an infinite weight is not to be added
        const float4 y = from[(c / 4 + h) * 256 + kFewTokens];
        v[4 * h] += isfinite(y.x) ? y.x : 0.0f;
        v[4 * h + 1] += isfinite(y.y) ? y.y : 0.0f;
        v[4 * h + 2] += isfinite(y.z) ? y.z : 0.0f;
        v[4 * h + 3] += isfinite(y.w) ? y.w : 0.0f;
      }
      if (kMode == kForward) {
        const float4 y = from[((c + BN / 2) / 4 + h) * 256];
        u[4 * h] += y.x;
        u[4 * h + 1] += y.y;
        u[4 * h + 2] += y.z;
        u[4 * h + 3] += y.w;
      }
    }
  }
  const int half_m = p.m_tiles / 2;
  const bool second = kMode == kWeights && m >= half_m;
  const int64_t row = (int64_t)(second ? m - half_m : m) * 256 + threadIdx.x;
  const int col = n * kCols + c;
  if (row >= p.rows || col >= p.cols) return;
  const int64_t at = row * p.ld_out + col;
  Vec<T, 8> o;
  if constexpr (kMode == kForward) {
    if (p.keep[0] != nullptr) {
      o.set(v);
      store_vec(reinterpret_cast<T*>(p.keep[0]) + at, o);
      o.set(u);
      store_vec(reinterpret_cast<T*>(p.keep[1]) + at, o);
    }
    gate_product(p.activation, v, u, v);
  }
  o.set(v);
  store_vec(reinterpret_cast<T*>(second ? p.out[1] : p.out[0]) + at, o);
}

template <typename T, int kMode, int BN>
__global__ void __launch_bounds__(256) gemm_join_kernel(const GemmParams p) {
  enter_grid();
  join_tile<T, kMode, BN>(p, blockIdx.x);
}
// ... of dX by the first `split` CTAs, of dW by the others
template <typename T, int BN>
__global__ void __launch_bounds__(256)
    gemm_join_both_kernel(const GemmParams pi, const GemmParams pw, const int split) {
  enter_grid();
  if (blockIdx.x < split)
    join_tile<T, kInput, BN>(pi, blockIdx.x);
  else
    join_tile<T, kWeights, BN>(pw, blockIdx.x - split);
}

// dG = dH * up * a'(gate), dU = dH * a(gate), eight elements a thread.  A CTA has 2048 elements of one row, or of
// everything where rows follow one another without gaps: a division a CTA, not one a thread (37800 x 13824: 1241 us
// with that).
template <typename T>
__global__ void __launch_bounds__(256) gate_grad_kernel(const T* dh, const T* gate, const T* up, T* dg, T* du,
                                                        int64_t ld, int64_t ld_out, int64_t row_length,
                                                        int ctas_per_row, int activation) {
  enter_grid(dh, gate, up);
  const int row = blockIdx.x / ctas_per_row;
  const int64_t col = ((int64_t)(blockIdx.x - row * ctas_per_row) * 256 + threadIdx.x) * 8;
  if (col >= row_length) return;
  const int64_t at = row * ld + col, to = row * ld_out + col;
  const Vec<T, 8> h = load_once<T, 8>(dh + at), g = load_once<T, 8>(gate + at), u = load_once<T, 8>(up + at);
  float fg[8], fu[8];
  with_activation(activation, [&](auto k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a, slope;
      activate<decltype(k)::value>(g[e], a, slope);
      fg[e] = h[e] * u[e] * slope;
      fu[e] = h[e] * a;
    }
  });
  Vec<T, 8> og, ou;
  og.set(fg);
  ou.set(fu);
  store_vec<T, 8>(dg + to, og);
  store_vec<T, 8>(du + to, ou);
}

// ... in two parts: rows 0 .. tokens - 1 rounded, then zeros up to row 128, then what the roundings leave.  The last is
// multiplied by a copy of X without infinities and NaN, made here by the CTAs behind row 128: the rounded part times X
// has them already, and what is left, of either sign or zero, would make NaN of infinities.
template <typename T>
__global__ void __launch_bounds__(256) gate_grad_parts_kernel(const T* dh, const T* gate, const T* up, T* dg, T* du,
                                                              int64_t ld, int64_t ld_out, int hidden, int tokens,
                                                              int activation, const T* x, int64_t ld_x, T* finite_x,
                                                              int dim) {
  enter_grid(dh, gate, up, x);
  const int row = blockIdx.y, col = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (row >= kFewTokens) {
    if (col >= dim) return;
    const int64_t token = row - kFewTokens;
    Vec<T, 8> v = load_vec<T, 8>(x + token * ld_x + col);
    float keep[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) keep[e] = isfinite(v[e]) ? v[e] : 0.0f;
    v.set(keep);
    store_vec(finite_x + token * dim + col, v);
    return;
  }
  if (col >= hidden) return;
  const int64_t to = row * ld_out + col, rest = to + kFewTokens * ld_out;
  Vec<T, 8> og, ou;
  if (row >= tokens) {
    og.clear();
    store_vec(dg + to, og);
    store_vec(du + to, og);
    return;
  }
  const int64_t at = row * ld + col;
  const Vec<T, 8> h = load_once<T, 8>(dh + at), g = load_once<T, 8>(gate + at), u = load_once<T, 8>(up + at);
  float fg[8], fu[8];
  with_activation(activation, [&](auto k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a, slope;
      activate<decltype(k)::value>(g[e], a, slope);
      fg[e] = h[e] * u[e] * slope;
      fu[e] = h[e] * a;
    }
  });
  og.set(fg);
  ou.set(fu);
  store_vec(dg + to, og);
  store_vec(du + to, ou);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // an infinity leaves nothing
    fg[e] = isfinite(og[e]) ? fg[e] - og[e] : 0.0f;
    fu[e] = isfinite(ou[e]) ? fu[e] - ou[e] : 0.0f;
  }
  og.set(fg);
  ou.set(fu);
  store_vec(dg + rest, og);
  store_vec(du + rest, ou);
}

__global__ void __launch_bounds__(256) zero_rows_kernel(uint16_t* a, uint16_t* b, int rows, int cols, int64_t ld) {
  enter_grid();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)rows * cols; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cols, at = r * ld + (i - r * cols);
    a[at] = 0;
    b[at] = 0;
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------

constexpr int kPairs = kSms / 2;
constexpr long long kWaitLimit = 200000000LL;  // of a wait in a kernel: about 0.1 s of SM clocks
constexpr int64_t kPartialBytes = (int64_t)2 * kPairs * 256 * 256 * 4;

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Instruction descriptor: bits 7 and 10 say that A and B are bf16, not fp16.
static uint32_t instruction(int dtype, int M, int N, int a_mn_major, int b_mn_major) {
  const uint32_t d = ptx::make_idesc_bf16(M, N, a_mn_major, b_mn_major);
  return dtype == SPARSP_BF16 ? d : d & ~((1u << 7) | (1u << 10));
}

// [rows][cols] of 16-bit elements in boxes of 64 columns x box_rows rows, and for results of 32 x 32
static int make_map(CUtensorMap* out, int dtype, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  return make_matrix_tmap(out, base, dtype == SPARSP_BF16, rows, cols, ld, 64, box_rows);
}
static int make_out_map(CUtensorMap* out, int dtype, const void* base, int64_t rows, int64_t cols, int64_t ld) {
  return make_matrix_tmap(out, base, dtype == SPARSP_BF16, rows, cols, ld, 32, 32);
}

constexpr int BN = 256;
using Bf = __nv_bfloat16;
using Hf = __half;

static int join_ctas(const GemmParams& p, int mode) {
  return (p.m_tiles * p.n_tiles - p.whole) * ((mode == kForward ? BN / 2 : BN) / 8);
}

// What a product takes on some pairs of SMs, in clocks, and whether its last round is shared out by blocks of K for
// that.
//
// 512 a block of K and 2500 a unit for what no block hides.  Sharing costs 8000 for the launch that adds the sums, 1200
// for each piece of a tile, which are added one after the other, and 90 for each piece there is, which is written and
// read: fitted to 361 sizes of all three products, each timed whole and in 2, 3, 4, 6 and as many pieces as there are
// pairs; by these figures 0.3 % is lost on average against the best of them, 5 % at most against whole tiles.  (us,
// whole and in pieces; tiles of the last round x blocks: 6 x 128 42.3, two 29.1, four 22.5, twelve 29.0; 6 x 32 behind
// a round of 74 tiles 29.2, two 34.9; 20 x 32 16.3, two 18.1; 20 x 128 45.2, three 33.7; 37 x 64 26.8, two 29.4; 37 x
// 256 99, two 72.)
//
// Where there are not two pairs for a tile, all pairs can have equal runs, most of which touch two tiles.  They read
// different rows and columns at one time, so it takes long tiles and few of them: 24000 beside the blocks, and at most
// seven tiles for ten pairs (40 x 256 102, 85 shared; 48 x 256 118, 110; 48 x 128 54, 58; 50 x 160 64, 70; 56 x 256
// 127, 131; 64 x 512 254, 348).
struct Clocks {
  int64_t product, join;
  int shares;  // pairs that the last round is shared out to, 0: none
  int64_t all() const { return product + join; }
};
// share_all: every tile has to be shared (there are fewer than pairs).
static Clocks gemm_clocks(int tiles, int blocks, int pairs, bool share_all) {
  const int rounds = tiles / pairs, rest = tiles % pairs;
  const int64_t unit = 512LL * blocks + 2500;
  Clocks best = {(rounds + (rest > 0)) * unit, 0, 0};
  if (rest == 0) return best;
  if (share_all) best.product = INT64_MAX;
  auto shorter = [&](int64_t k, int64_t more, int64_t join, int shares) {
    const Clocks c = {rounds * unit + 512 * k + 2500 + more, join, shares};
    if (c.all() < best.all()) best = c;
  };
  const int fewest = share_all ? 1 : 2, most = std::max(fewest, std::min(pairs / rest, blocks / 4));
  if (pairs / rest >= fewest) {
    // the least of 512 blocks / pieces + (1200 + 90 rest) pieces, from either side
    const int near = (int)std::sqrt(512.0 * blocks / (1200 + 90 * rest));
    for (int pieces : {near, near + 1}) {
      pieces = std::min(std::max(pieces, fewest), most);
      shorter(ceil_div(blocks, pieces), 90LL * rest * pieces, 8000 + 1200LL * pieces, rest * pieces);
    }
  }
  const int all = (int)std::min<int64_t>(pairs, (int64_t)rest * blocks / 4);
  if (pairs / rest < 2 && all > rest && 10 * rest <= 7 * pairs)
    shorter(ceil_div((int64_t)rest * blocks, all), 12000, 12000, all);
  return best;
}
static void share_out(GemmParams* p, int pairs, int shares) {
  const int tiles = p->m_tiles * p->n_tiles;
  p->whole = shares > 0 ? tiles / pairs * pairs : tiles;
  p->shares = shares;
  p->alternate = tiles >= 3 * pairs;
}

// What every product needs beside its sizes.
static int prepare_gemm(GemmParams* p, int mode, const sparsp_ffn& f, char* ws) {
  if ((int64_t)p->m_tiles * p->n_tiles > (1 << 30)) {
    set_error("%d x %d tiles are too many", p->m_tiles, p->n_tiles);
    return SPARSP_ERR_UNSUPPORTED;
  }
  const Clocks c = gemm_clocks(p->m_tiles * p->n_tiles, p->k_blocks * (mode == kInput ? 2 : 1), kPairs,
                               mode == kInput && p->two_parts);
  share_out(p, kPairs, c.shares);
  p->band = 8;
  p->partial = reinterpret_cast<float*>(ws + kStatusWords * 4);
  p->status = reinterpret_cast<int32_t*>(ws);
  p->wait_limit = kWaitLimit;
  p->activation = f.activation;
  p->idesc = instruction(f.dtype, 256, BN, mode == kWeights, mode != kForward);
  return SPARSP_OK;
}

template <int kMode>
static int launch_gemm(const GemmParams& p, const GemmMaps& m, int dtype, cudaStream_t st) {
  using C = GemmCfg<BN>;
  auto kern = dtype == SPARSP_BF16 ? gemm_kernel<Bf, kMode, BN> : gemm_kernel<Hf, kMode, BN>;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, C::kDynamic));
  const unsigned grid = 2u * (unsigned)std::min(std::max(p.whole, p.shares), kPairs);
  SPARSP_CUDA_OK(launch_clusters(kern, dim3(grid), 2, kGemmThreads, C::kDynamic, st, m.a0, m.a1, m.b0, m.b1, m.o0, m.o1,
                                 m.o2, p));
  if (const int ctas = join_ctas(p, kMode)) {
    auto join = dtype == SPARSP_BF16 ? gemm_join_kernel<Bf, kMode, BN> : gemm_join_kernel<Hf, kMode, BN>;
    SPARSP_CUDA_OK(launch_kernel(join, dim3((unsigned)ctas), 256, 0, st, p));
  }
  return SPARSP_OK;
}

// dX and dW together.  Alone, each of two small products leaves pairs of SMs without a tile in its last round; together
// they share the pairs out so that both end at the same time.  What is shared out by blocks of K stays so for either
// product alone, so that it gives the same bits.  Returns the pairs of dX, or 0 where the two are better apart, with
// 10000 clocks for another launch and its wait: in two parts dX needs a pair for each of its tiles and more, which may
// leave dW too few (64 x 18432 x 256, 72 of 74: together 305 us, apart 31; x 16384, 64: 46 and 29; x 14336, 56: 29 and
// 28; x 12288: 21 and 27).
static int plan_both(GemmParams* pi, GemmParams* pw) {
  const int ti = pi->m_tiles * pi->n_tiles, tw = pw->m_tiles * pw->n_tiles;
  const int bi = 2 * pi->k_blocks, bw = pw->k_blocks;
  const bool all = pi->two_parts;
  const int fewest = all ? ti + 1 : 1;
  int low = fewest, high = kPairs - 1;  // the fewest pairs with which dX is no later than dW
  while (low < high) {
    const int mid = (low + high) / 2;
    if (gemm_clocks(ti, bi, mid, all).product <= gemm_clocks(tw, bw, kPairs - mid, false).product)
      high = mid;
    else
      low = mid + 1;
  }
  int64_t best = gemm_clocks(ti, bi, kPairs, all).all() + gemm_clocks(tw, bw, kPairs, false).all() + 10000;
  int pairs = 0;
  for (int s = std::max(fewest, low - 1); s <= low; ++s) {
    const Clocks i = gemm_clocks(ti, bi, s, all), w = gemm_clocks(tw, bw, kPairs - s, false);
    const int64_t t = std::max(i.product, w.product) + std::max(i.join, w.join);
    if (t >= best) continue;
    best = t;
    pairs = s;
    share_out(pi, s, i.shares);
    share_out(pw, kPairs - s, w.shares);
  }
  if (pairs > 0) pw->partial += (int64_t)2 * pi->shares * 256 * BN;
  return pairs;
}

static int launch_both(const GemmParams& pi, const GemmMaps& mi, const GemmParams& pw, const GemmMaps& mw, int pairs,
                       int dtype, cudaStream_t st) {
  using C = GemmCfg<BN>;
  auto kern = dtype == SPARSP_BF16 ? gemm_both_kernel<Bf, BN> : gemm_both_kernel<Hf, BN>;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, C::kDynamic));
  SPARSP_CUDA_OK(launch_clusters(kern, dim3(2 * kPairs), 2, kGemmThreads, C::kDynamic, st, mi, pi, mw, pw, pairs));
  const int ji = join_ctas(pi, kInput), jw = join_ctas(pw, kWeights);
  if (ji + jw > 0) {
    auto join = dtype == SPARSP_BF16 ? gemm_join_both_kernel<Bf, BN> : gemm_join_both_kernel<Hf, BN>;
    SPARSP_CUDA_OK(launch_kernel(join, dim3((unsigned)(ji + jw)), 256, 0, st, pi, pw, ji));
  }
  return SPARSP_OK;
}

// dG and dU have rows of whole 128-byte lines: a tile's rows of 128 bytes then lie in one line each, not in two (1003 x
// 1160 x 2504, backward: 41 us without).
static int64_t hidden_pitch(const sparsp_ffn& f) { return align_up(f.hidden, 64); }
// Two parts need the halves of every tile of dX to meet, in pieces of K that are added; rows of so many tiles that
// pairs have a whole one each are left out of it.  What they cost (backward us, two parts and one: 5120 x 13824, 1
// token 143 and 144, 64 147 and 141, 128 170 and 151; 1920 x 7680, 128 tokens 58 and 55; 1160 x 2504 22 and 21; 4096 x
// 1024 21 and 18) buys the error of fp32 operands, 1.4 times less; from 129 tokens on dX would take twice the tiles
// and dW twice the blocks.
static bool two_parts(const sparsp_ffn& f) { return f.tokens <= kFewTokens && ceil_div(f.dim, BN) <= kPairs - 2; }
static int64_t hidden_rows(const sparsp_ffn& f) { return two_parts(f) ? kFewTokens + f.tokens : f.tokens; }
static int64_t hidden_bytes(const sparsp_ffn& f, int64_t rows) { return align_up(rows * hidden_pitch(f) * 2, 256); }

// Never less for more tokens, so that a workspace for the most tokens serves every call with fewer: always room for two
// parts of kFewTokens rows.
int64_t ffn_workspace_bytes(const sparsp_ffn& f, bool backward) {
  if (!backward && f.tokens <= kFewTokens) return kStatusWords * 4;
  const int64_t rows = std::max<int64_t>(f.tokens, 2 * kFewTokens);
  const int64_t finite_x = (int64_t)kFewTokens * std::min(f.dim, kPairs * BN) * 2;
  return kStatusWords * 4 + kPartialBytes + (backward ? 2 * hidden_bytes(f, rows) + finite_x : 0);
}

static int launch_few(const sparsp_ffn& f, const void* X, const void* Wg, const void* Wu, void* H, void* gate,
                      void* up, char* ws, cudaStream_t st) {
  FewParams p = {};
  p.columns = (int32_t)align_up(f.tokens, 16);
  p.k_blocks = ceil_div(f.dim, kStageK);
  // CTAs that share out K, where there are few tiles, in pieces of eight blocks at least (100 x 5120 x 512: alone 17.8
  // us, two 12.6, four 10.1; 2 x 824 x 1144, pieces of six: alone 4.5, two 5.3).  Clusters of four find room on 128
  // SMs, of two on all; of eight there is not room for enough at once.
  auto splits = [&](int F) {
    const int tiles = ceil_div(f.hidden, F);
    if (tiles * 4 <= 128 && p.k_blocks >= 32) return 4;
    return tiles * 2 <= kSms && p.k_blocks >= 16 ? 2 : 1;
  };
  // features at a time: what a CTA loads, 2 F rows of weights and N of tokens a block of K in each round
  auto cost = [&](int F) {
    return (int64_t)ceil_div(ceil_div(f.hidden, F), kSms) * (2 * F + p.columns) * ceil_div(p.k_blocks, splits(F));
  };
  p.features = 64;
  for (int F = 32; F >= 16; F /= 2)
    if (cost(F) < cost(p.features)) p.features = F;
  p.splits = splits(p.features);
  p.tiles = ceil_div(f.hidden, p.features);
  p.ld_turn = p.columns + 1;
  const int turn = (int)align_up(2 * p.features * p.ld_turn * 4, 128), room = kFewSmem - 16384 - turn - 1024;
  const int block = (2 * p.features + p.columns) * 128;
  // blocks of K a stage, as many as leave four stages (16 x 5120 x 13824: 44.5 us with four, 51.1 with one)
  int deep = 4;
  while (deep > 1 && room / (deep * block) < 4) deep /= 2;
  p.stage_bytes = deep * block;
  p.stages = std::min(16, room / p.stage_bytes);
  p.out = H;
  p.keep[0] = gate;
  p.keep[1] = up;
  p.ld_out = f.stride_h;
  p.tokens = (int32_t)f.tokens;
  p.hidden = f.hidden;
  p.activation = f.activation;
  p.idesc = instruction(f.dtype, 128, p.columns, 0, 0);
  p.status = reinterpret_cast<int32_t*>(ws);
  p.wait_limit = kWaitLimit;
  CUtensorMap mg, mu, mx;
  int rc;
  if ((rc = make_map(&mg, f.dtype, Wg, f.hidden, f.dim, f.stride_w, p.features)) != SPARSP_OK) return rc;
  if ((rc = make_map(&mu, f.dtype, Wu, f.hidden, f.dim, f.stride_w, p.features)) != SPARSP_OK) return rc;
  if ((rc = make_map(&mx, f.dtype, X, f.tokens, f.dim, f.stride_x, p.columns)) != SPARSP_OK) return rc;
  const bool bf = f.dtype == SPARSP_BF16;
  auto kern = deep == 4   ? (bf ? few_kernel<__nv_bfloat16, 4> : few_kernel<__half, 4>)
              : deep == 2 ? (bf ? few_kernel<__nv_bfloat16, 2> : few_kernel<__half, 2>)
                          : (bf ? few_kernel<__nv_bfloat16, 1> : few_kernel<__half, 1>);
  const int smem = p.stages * p.stage_bytes + 16384 + turn + 1024;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, smem));
  SPARSP_CUDA_OK(launch_clusters(kern, dim3((unsigned)(std::min(p.tiles, kSms) * p.splits)), p.splits, kFewThreads, smem,
                                 st, mg, mu, mx, p));
  return SPARSP_OK;
}

int launch_ffn_fwd(const sparsp_ffn& f, const void* X, const void* Wg, const void* Wu, void* H, void* gate, void* up,
                   char* ws, cudaStream_t st) {
  if (f.tokens <= kFewTokens) return launch_few(f, X, Wg, Wu, H, gate, up, ws, st);
  GemmMaps m;
  int rc;
  if ((rc = make_map(&m.a0, f.dtype, X, f.tokens, f.dim, f.stride_x, kTileRows)) != SPARSP_OK) return rc;
  if ((rc = make_map(&m.b0, f.dtype, Wg, f.hidden, f.dim, f.stride_w, BN / 2)) != SPARSP_OK) return rc;
  if ((rc = make_map(&m.b1, f.dtype, Wu, f.hidden, f.dim, f.stride_w, BN / 2)) != SPARSP_OK) return rc;
  m.a1 = m.a0;
  if ((rc = make_out_map(&m.o0, f.dtype, H, f.tokens, f.hidden, f.stride_h)) != SPARSP_OK) return rc;
  m.o1 = m.o2 = m.o0;
  if (gate != nullptr) {
    if ((rc = make_out_map(&m.o1, f.dtype, gate, f.tokens, f.hidden, f.stride_h)) != SPARSP_OK) return rc;
    if ((rc = make_out_map(&m.o2, f.dtype, up, f.tokens, f.hidden, f.stride_h)) != SPARSP_OK) return rc;
  }
  GemmParams p = {};
  p.out[0] = H;
  p.keep[0] = gate;
  p.keep[1] = up;
  p.ld_out = f.stride_h;
  p.rows = (int32_t)f.tokens;
  p.cols = f.hidden;
  p.m_tiles = ceil_div(f.tokens, 256);
  p.n_tiles = ceil_div(f.hidden, BN / 2);
  p.k_blocks = ceil_div(f.dim, kStageK);
  if ((rc = prepare_gemm(&p, kForward, f, ws)) != SPARSP_OK) return rc;
  return launch_gemm<kForward>(p, m, f.dtype, st);
}

int launch_ffn_bwd(const sparsp_ffn& f, const void* dH, const void* X, const void* Wg, const void* Wu,
                   const void* gate, const void* up, void* dX, void* dWg, void* dWu, char* ws, cudaStream_t st) {
  if (f.tokens == 0) {
    if (dWg != nullptr)
      SPARSP_CUDA_OK(launch_kernel(zero_rows_kernel, dim3(2 * kSms), 256, 0, st, (uint16_t*)dWg, (uint16_t*)dWu,
                                   f.hidden, f.dim, f.stride_w));
    return SPARSP_OK;
  }
  if (dX == nullptr && dWg == nullptr) return SPARSP_OK;
  char* dg = ws + kStatusWords * 4 + kPartialBytes;
  char* du = dg + hidden_bytes(f, hidden_rows(f));
  char* finite_x = du + hidden_bytes(f, hidden_rows(f));
  const bool gaps = f.stride_h != f.hidden || hidden_pitch(f) != f.hidden;
  const int64_t row_length = gaps ? f.hidden : f.tokens * f.hidden, rows = gaps ? f.tokens : 1;
  const int64_t ctas_per_row = (row_length + 2047) / 2048;
  if (ctas_per_row * rows > 0x7fffffffLL) {
    set_error("tokens * hidden is too large");
    return SPARSP_ERR_UNSUPPORTED;
  }
  const dim3 grid((unsigned)(ctas_per_row * rows));
  auto grad = [&](auto* element) {
    using T = std::remove_pointer_t<decltype(element)>;
    return launch_kernel(gate_grad_kernel<T>, grid, 256, 0, st, (const T*)dH, (const T*)gate, (const T*)up, (T*)dg,
                         (T*)du, f.stride_h, hidden_pitch(f), row_length, (int)ctas_per_row, f.activation);
  };
  auto grad_parts = [&](auto* element) {
    using T = std::remove_pointer_t<decltype(element)>;
    const int widest = dWg != nullptr ? std::max(f.hidden, f.dim) : f.hidden;
    const int rows = kFewTokens + (dWg != nullptr ? (int)f.tokens : 0);
    return launch_kernel(gate_grad_parts_kernel<T>, dim3((unsigned)ceil_div(widest, 2048), (unsigned)rows), 256, 0, st,
                         (const T*)dH, (const T*)gate, (const T*)up, (T*)dg, (T*)du, f.stride_h, hidden_pitch(f),
                         f.hidden, (int)f.tokens, f.activation, (const T*)X, f.stride_x, (T*)finite_x, f.dim);
  };
  if (two_parts(f))
    SPARSP_CUDA_OK(f.dtype == SPARSP_BF16 ? grad_parts((Bf*)nullptr) : grad_parts((Hf*)nullptr));
  else
    SPARSP_CUDA_OK(f.dtype == SPARSP_BF16 ? grad((Bf*)nullptr) : grad((Hf*)nullptr));
  GemmMaps mi, mw;
  GemmParams pi = {}, pw = {};
  int rc;
  pi.m_tiles = ceil_div(f.tokens, 256);
  pw.m_tiles = 2 * ceil_div(f.hidden, 256);
  pi.n_tiles = pw.n_tiles = ceil_div(f.dim, BN);
  pi.k_blocks = ceil_div(f.hidden, kStageK);
  pw.k_blocks = ceil_div(f.tokens, kStageK) * (two_parts(f) ? 2 : 1);
  pi.two_parts = pw.two_parts = two_parts(f);
  if ((rc = prepare_gemm(&pi, kInput, f, ws)) != SPARSP_OK) return rc;
  if ((rc = prepare_gemm(&pw, kWeights, f, ws)) != SPARSP_OK) return rc;
  // both at once up to four rounds of tiles (1003 x 1160 x 2504 36 us, one after the other 46; 2048 x 1024 x 4096, 3.5
  // rounds, 65 and 81); with more, both ways are alike within what runs differ by (2048 x 2048 x 4096, 6.9 rounds:
  // 114-122 and 115-118 us), and apart they read less at a time
  const bool small = (int64_t)pi.m_tiles * pi.n_tiles + (int64_t)pw.m_tiles * pw.n_tiles <= 4 * kPairs;
  const int pairs = small ? plan_both(&pi, &pw) : 0;  // 0: apart
  if (dX != nullptr) {
    if ((rc = make_map(&mi.a0, f.dtype, dg, hidden_rows(f), f.hidden, hidden_pitch(f), kTileRows)) != SPARSP_OK) return rc;
    if ((rc = make_map(&mi.a1, f.dtype, du, hidden_rows(f), f.hidden, hidden_pitch(f), kTileRows)) != SPARSP_OK) return rc;
    if ((rc = make_map(&mi.b0, f.dtype, Wg, f.hidden, f.dim, f.stride_w, kStageK)) != SPARSP_OK) return rc;
    if ((rc = make_map(&mi.b1, f.dtype, Wu, f.hidden, f.dim, f.stride_w, kStageK)) != SPARSP_OK) return rc;
    if ((rc = make_out_map(&mi.o0, f.dtype, dX, f.tokens, f.dim, f.stride_x)) != SPARSP_OK) return rc;
    mi.o1 = mi.o2 = mi.o0;
    pi.out[0] = dX;
    pi.ld_out = f.stride_x;
    pi.rows = (int32_t)f.tokens;
    pi.cols = f.dim;
  }
  if (dWg != nullptr) {
    if ((rc = make_map(&mw.a0, f.dtype, dg, hidden_rows(f), f.hidden, hidden_pitch(f), kStageK)) != SPARSP_OK) return rc;
    if ((rc = make_map(&mw.a1, f.dtype, du, hidden_rows(f), f.hidden, hidden_pitch(f), kStageK)) != SPARSP_OK) return rc;
    if ((rc = make_map(&mw.b0, f.dtype, X, f.tokens, f.dim, f.stride_x, kStageK)) != SPARSP_OK) return rc;
    mw.b1 = mw.b0;
    if (two_parts(f) && (rc = make_map(&mw.b1, f.dtype, finite_x, f.tokens, f.dim, f.dim, kStageK)) != SPARSP_OK) return rc;
    if ((rc = make_out_map(&mw.o0, f.dtype, dWg, f.hidden, f.dim, f.stride_w)) != SPARSP_OK) return rc;
    if ((rc = make_out_map(&mw.o1, f.dtype, dWu, f.hidden, f.dim, f.stride_w)) != SPARSP_OK) return rc;
    mw.o2 = mw.o0;
    pw.out[0] = dWg;
    pw.out[1] = dWu;
    pw.ld_out = f.stride_w;
    pw.rows = f.hidden;
    pw.cols = f.dim;
  }
  if (pairs > 0 && dX != nullptr && dWg != nullptr) return launch_both(pi, mi, pw, mw, pairs, f.dtype, st);
  if (dX != nullptr && (rc = launch_gemm<kInput>(pi, mi, f.dtype, st)) != SPARSP_OK) return rc;
  if (dWg != nullptr && (rc = launch_gemm<kWeights>(pw, mw, f.dtype, st)) != SPARSP_OK) return rc;
  return SPARSP_OK;
}

}  // namespace sparsp
