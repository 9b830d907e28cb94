// Rotary positions: the table of (cos, sin) and the rotation of Q and K.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

// One entry a thread.  The angle is coordinate * frequency in fp64: in fp32 the product alone would be 0.004 radians
// off at position 100000.  Tables are made once per geometry.
__global__ void __launch_bounds__(256) rotary_table_kernel(const double* __restrict__ inv_freq, double amplitude,
                                                           float2* __restrict__ table, int pt, int ph, int pw,
                                                           int64_t nt, int64_t nh, int64_t total) {
  enter_grid(inv_freq);
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= total) return;
  int64_t at = e;
  int pairs = pt, first = 0;
  if (at >= nt) {
    at -= nt;
    pairs = ph;
    first = pt;
    if (at >= nh) {
      at -= nh;
      pairs = pw;
      first = pt + ph;
    }
  }
  const int64_t p = at / pairs;
  double s, c;
  sincos((double)p * inv_freq[first + (int)(at - p * pairs)], &s, &c);
  table[e] = make_float2((float)(amplitude * c), (float)(amplitude * s));
}

int launch_rotary_table(const sparsp_rotary& r, const double* inv_freq, double amplitude, float* table,
                        cudaStream_t st) {
  const int64_t nt = (int64_t)r.pairs_t * r.len_t, nh = (int64_t)r.pairs_h * r.len_h;
  const int64_t total = nt + nh + (int64_t)r.pairs_w * r.len_w;
  if (total == 0) return SPARSP_OK;
  SPARSP_CUDA_OK(launch_kernel(rotary_table_kernel, dim3((unsigned)((total + 255) / 256)), 256, 0, st, inv_freq,
                               amplitude, reinterpret_cast<float2*>(table), r.pairs_t, r.pairs_h, r.pairs_w, nt, nh,
                               total));
  return SPARSP_OK;
}

struct RotaryParams {
  const void* x[2];
  void* y[2];
  const float2* table;
  const int32_t* positions;
  int32_t* status;
  int64_t positions_stride_batch, sB, sH, sT;
  int32_t origin[3], len[3], pairs_of[3];
  int64_t table_of[3];  // first entry of each coordinate's part
  int32_t n_tensors, tokens, all_tokens, n_video, hw, w;
  int32_t heads, heads_per_cta, head_groups, head_lanes, tokens_per_cta;
  int32_t rot_begin, pairs, n_rotated, units;  // units of a row, the first n_rotated of them rotated
  int32_t inverse;
};

constexpr int kRotaryThreads = 256;
// Heads whose loads a thread has in flight at once (48 heads x 17776 tokens x 64 fp16, token-major: 75.5 us, with two
// 79.2, with eight, which leave fewer warps, 76.4; 40 heads x 75600 x 128: 491, 492, 502).
constexpr int kRotaryHeads = 4;

// A thread has one token and one unit of its row (16 bytes of interleaved pairs; two 16-byte vectors half the rotated
// part apart; 16 bytes to be copied), finds the (cos, sin) of its pairs once and goes over the heads of Q and K with
// them: the angles depend on the token alone, so the table costs little.  A token's units are consecutive lanes, so a
// head's row is read and written whole; where heads lie closer together than tokens, a few heads of a token come next
// to each other, so that a warp reads on in memory (48 heads x 17776 tokens x 64 fp16, token-major: 84 us without).
// Bound by HBM: 40 heads x 75600 x 128 bf16, Q and K, 491 us = 6.3 TB/s; with positions of permuted tokens 494. E:
// elements of a vector, 1 where the rotated part or the pairs do not begin and end on 16 bytes; then by the number of loads
// and stores, one an element (16 heads x 17776 x 72 bf16, halves of 36 pairs, 56 us; neighbours, on 16 bytes, 32).
template <typename T, int E, bool kHalf>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const RotaryParams p) {
  const int32_t* positions = p.positions;
  enter_grid(positions);
  constexpr int kPairs = kHalf ? E : (E > 1 ? E / 2 : 1);  // pairs of a unit
  constexpr int kLoads = kHalf ? 2 : 1;
  constexpr int V = kHalf ? E : (E > 1 ? E : 2);  // elements of a load
  constexpr int VA = kHalf || E > 1 ? V : 1;      // ... that are sure to be aligned together
  const int row_in_cta = threadIdx.x / p.units;
  const int u = threadIdx.x - row_in_cta * p.units;
  const int in_cta = row_in_cta / p.head_lanes, head_lane = row_in_cta - in_cta * p.head_lanes;
  const int tile = blockIdx.x / p.head_groups;
  const int64_t token = (int64_t)tile * p.tokens_per_cta + in_cta;
  if (in_cta >= p.tokens_per_cta || token >= p.all_tokens) return;
  const int batch = (int)token / p.tokens, n = (int)token - batch * p.tokens;

  bool turn = u < p.n_rotated;
  if (!turn && p.x[0] == p.y[0] && (p.n_tensors == 1 || p.x[1] == p.y[1])) return;
  int at[3];
  if (positions != nullptr) {
    const int32_t* mine = positions + batch * p.positions_stride_batch + 3LL * n;
    at[0] = mine[0];
    at[1] = mine[1];
    at[2] = mine[2];
    if (at[0] < 0) turn = false;
  } else {
    const int t = n / p.hw, r = n - t * p.hw, h = r / p.w;
    at[0] = t + p.origin[0];
    at[1] = h + p.origin[1];
    at[2] = r - h * p.w + p.origin[2];
    if (n >= p.n_video) turn = false;
  }
  if (positions != nullptr && turn) {
#pragma unroll
    for (int a = 0; a < 3; ++a)
      if (p.pairs_of[a] > 0 && (at[a] < 0 || at[a] >= p.len[a])) {
        turn = false;
        if (atomicCAS(p.status, 0, SPARSP_ERR_INVALID_ARG) == 0) {
          p.status[1] = a;
          p.status[2] = n;
          p.status[3] = at[a];
        }
      }
  }
  float2 cs[kPairs];
  if (turn) {
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      int i = u * kPairs + k, a = 0;
      if (i >= p.pairs_of[0]) {
        i -= p.pairs_of[0];
        a = 1;
        if (i >= p.pairs_of[1]) {
          i -= p.pairs_of[1];
          a = 2;
        }
      }
      const int where = a == 0 ? at[0] : a == 1 ? at[1] : at[2];
      cs[k] = p.table[p.table_of[a] + (int64_t)where * p.pairs_of[a] + i];
      if (p.inverse) cs[k].y = -cs[k].y;
    }
  }
  // first elements of the unit's loads; a copied unit has E elements and no second load
  const bool copied = u >= p.n_rotated;
  int e0, e1 = 0;
  if (copied) {
    e0 = (u - p.n_rotated) * E;
    if (e0 >= p.rot_begin) e0 += 2 * p.pairs;
  } else if (kHalf) {
    e0 = p.rot_begin + u * E;
    e1 = e0 + p.pairs;
  } else {
    e0 = p.rot_begin + u * 2 * kPairs;
  }
  const int h0 = (blockIdx.x % p.head_groups) * p.heads_per_cta, h1 = min(h0 + p.heads_per_cta, p.heads);
  const int64_t row = batch * p.sB + n * p.sT;
  for (int which = 0; which < p.n_tensors; ++which) {
    const T* x = reinterpret_cast<const T*>(p.x[which]) + row;
    T* y = reinterpret_cast<T*>(p.y[which]) + row;
    for (int h = h0 + head_lane; h < h1; h += kRotaryHeads * p.head_lanes) {
      Vec<T, VA> v[kRotaryHeads][kLoads][V / VA];
#pragma unroll
      for (int k = 0; k < kRotaryHeads; ++k)
        if (h + k * p.head_lanes < h1) {
          const T* mine = x + (h + k * p.head_lanes) * p.sH;
#pragma unroll
          for (int l = 0; l < kLoads; ++l) {
            if (l == 1 && copied) continue;
#pragma unroll
            for (int j = 0; j < V / VA; ++j)
              if (j == 0 || !copied) v[k][l][j] = load_once<T, VA>(mine + (l == 0 ? e0 : e1) + j * VA);
          }
        }
#pragma unroll
      for (int k = 0; k < kRotaryHeads; ++k)
        if (h + k * p.head_lanes < h1) {
          if (turn) {
            float z[kLoads][V];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
              // the pair's two elements: load and place in it
              constexpr int lb = kHalf ? 1 : 0;
              const int pa = kHalf ? i : 2 * i, pb = kHalf ? i : 2 * i + 1;
              const float a = v[k][0][pa / VA][pa % VA], b = v[k][lb][pb / VA][pb % VA];
              z[0][pa] = a * cs[i].x - b * cs[i].y;
              z[lb][pb] = a * cs[i].y + b * cs[i].x;
            }
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
#pragma unroll
              for (int j = 0; j < V / VA; ++j) v[k][l][j].set(z[l] + j * VA);
          }
          T* mine = y + (h + k * p.head_lanes) * p.sH;
#pragma unroll
          for (int l = 0; l < kLoads; ++l) {
            if (l == 1 && copied) continue;
#pragma unroll
            for (int j = 0; j < V / VA; ++j)
              if (j == 0 || !copied) store_vec<T, VA>(mine + (l == 0 ? e0 : e1) + j * VA, v[k][l][j]);
          }
        }
    }
  }
}

template <typename T, int E, bool kHalf>
static cudaError_t launch_rotary_t(RotaryParams p, int head_dim, cudaStream_t st) {
  constexpr int kPairs = kHalf ? E : (E > 1 ? E / 2 : 1);
  p.n_rotated = p.pairs / kPairs;
  p.units = p.n_rotated + (head_dim - 2 * p.pairs) / E;
  p.head_lanes = p.sH < p.sT ? std::min(p.heads, std::max(1, 32 / p.units)) : 1;
  p.tokens_per_cta = kRotaryThreads / (p.units * p.head_lanes);
  const int64_t tiles = ((int64_t)p.all_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta;
  // all heads to a CTA, unless there are too few tokens for eight CTAs an SM that way (40 heads x 5120 tokens x 128:
  // 36.5 us, with four CTAs 39.4, with sixteen 37.7)
  int64_t per = p.heads;
  while (per > p.head_lanes && tiles * ((p.heads + per - 1) / per) < 8 * kSms) per = (per + 1) / 2;
  p.heads_per_cta = (int)per;
  p.head_groups = (int)((p.heads + per - 1) / per);
  return launch_kernel(rotary_kernel<T, E, kHalf>, dim3((unsigned)(tiles * p.head_groups)), kRotaryThreads, 0, st, p);
}

int launch_rotary(const sparsp_shape& s, const sparsp_rotary& r, const float* table, const int32_t* positions,
                  int64_t positions_stride_batch, const int32_t* origin, const void* Q, const void* K, void* Qo,
                  void* Ko, int inverse, int32_t* status, cudaStream_t st) {
  RotaryParams p = {};
  p.x[0] = Q;
  p.x[1] = K;
  p.y[0] = Qo;
  p.y[1] = Ko;
  p.n_tensors = K != nullptr ? 2 : 1;
  p.table = reinterpret_cast<const float2*>(table);
  p.positions = positions;
  p.positions_stride_batch = positions_stride_batch;
  p.status = status;
  p.sB = s.stride_batch;
  p.sH = s.stride_head;
  p.sT = s.stride_token;
  const int32_t pairs[3] = {r.pairs_t, r.pairs_h, r.pairs_w}, len[3] = {r.len_t, r.len_h, r.len_w};
  int64_t entries = 0;
  for (int a = 0; a < 3; ++a) {
    p.origin[a] = origin[a];
    p.len[a] = len[a];
    p.pairs_of[a] = pairs[a];
    p.table_of[a] = entries;
    entries += (int64_t)pairs[a] * (pairs[a] > 0 ? len[a] : 0);
  }
  p.hw = s.grid_h * s.grid_w;
  p.w = s.grid_w;
  p.n_video = s.grid_t * p.hw;
  p.tokens = p.n_video + s.n_text;
  p.all_tokens = p.tokens * s.batch;
  p.heads = s.heads;
  p.rot_begin = r.rot_begin;
  p.pairs = r.pairs_t + r.pairs_h + r.pairs_w;
  p.inverse = inverse;
  const int full = 16 / element_bytes(r.dtype);
  const bool half = r.pairing == SPARSP_PAIRS_HALF;
  const bool whole = r.rot_begin % full == 0 && (half ? p.pairs : 2 * p.pairs) % full == 0;
  cudaError_t e = cudaSuccess;
  SPARSP_WITH_TYPE(r.dtype, T, {
    constexpr int E = 16 / sizeof(T);
    e = half ? (whole ? launch_rotary_t<T, E, true>(p, s.head_dim, st) : launch_rotary_t<T, 1, true>(p, s.head_dim, st))
             : (whole ? launch_rotary_t<T, E, false>(p, s.head_dim, st)
                      : launch_rotary_t<T, 1, false>(p, s.head_dim, st));
  });
  SPARSP_CUDA_OK(e);
  return SPARSP_OK;
}

}  // namespace sparsp
