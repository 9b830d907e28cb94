// The residual step between two blocks of a layer: r = x + gate * u, u = norm_y(y) or y, n = norm_r(r), and its backward
// pass with the reduction of the gate's and the weights' gradients.
//
// A row is worked on by a team: 4 to 32 lanes of a warp, or a CTA.  Teams have consecutive rows, so that the weights
// of a group, read again for each row, are in L1.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

struct StepParams {
  const void *x, *y;     // backward: r, y
  const void *dn, *dr;   // backward
  const void *gate, *wy, *by, *wr, *br;
  void *r, *n;           // backward: dx, dy
  float *stats_y, *stats_r;
  float *partial, *partial_y;  // backward: [teams][2][4][dim], of a team's first group and its last, and [teams][2][dim]
  void *dgate, *dwy, *dby, *dwr, *dbr;
  int64_t rows, rows_per_group, stride_x, stride_y, stride_n;
  int32_t dim, teams, lanes, norm_y, norm_r;
  float eps, inv_dim;
};

__host__ __device__ inline int64_t first_row(int64_t team, int64_t teams, int64_t rows) {
  return team * (rows / teams) + (team < rows % teams ? team : rows % teams);
}
// the team that has a row
__host__ __device__ inline int64_t team_of(int64_t row, int64_t teams, int64_t rows) {
  const int64_t each = rows / teams, more = rows % teams;
  return row < more * (each + 1) ? row / (each + 1) : more + (row - more * (each + 1)) / each;
}

// Sums over a team, the same in every lane.  kWarps: the team is a CTA; its warps meet at one barrier a call, by turns
// of `room`.
template <bool kWarps, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int lanes, float (*room)[32][2], int& turn) {
  const int most = kWarps ? 16 : lanes / 2;
#pragma unroll
  for (int d = 16; d > 0; d /= 2)
    if (kWarps || d <= most) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    }
  if constexpr (kWarps) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float (*mine)[2] = room[turn];
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) mine[warp][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    for (int w = 0; w < warps; ++w) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += mine[w][i];
    }
  }
}

// E values of a weight of type T or fp32 at `at`; fill where there is no weight
template <typename T, int E>
__device__ __forceinline__ void weights(const void* w, bool fp32, int64_t at, float fill, float (&out)[E]) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = fill;
  } else if (fp32) {
#pragma unroll
    for (int q = 0; q < E / 4; ++q) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + at) + q);
      out[4 * q] = v.x;
      out[4 * q + 1] = v.y;
      out[4 * q + 2] = v.z;
      out[4 * q + 3] = v.w;
    }
  } else {
    const Vec<T, E> v = load_vec<T, E>(static_cast<const T*>(w) + at);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = v[e];
  }
}

// Which group a row is in, for rows that come in order.
struct Group {
  int64_t index, end;
  __device__ __forceinline__ Group(int64_t row, int64_t per) : index(row / per), end((index + 1) * per) {}
  __device__ __forceinline__ bool advance(int64_t row, int64_t per) {
    if (row < end) return false;
    ++index;  // (one at a time is enough: rows come one by one)
    end += per;
    return true;
  }
};

template <typename T, int V, bool kWarps, bool kFp32Weights>
__global__ void __launch_bounds__(kWarps ? 512 : 128) step_kernel(StepParams p) {
  enter_grid(p.x, p.y, p.gate);
  constexpr int E = 16 / sizeof(T);
  __shared__ float room[2][32][2];
  int turn = 0;
  const int lanes = kWarps ? blockDim.x : p.lanes;
  const int team = kWarps ? blockIdx.x : (blockIdx.x * blockDim.x + threadIdx.x) / lanes;
  const int me = kWarps ? threadIdx.x : threadIdx.x & (lanes - 1);
  const bool there = team < p.teams;  // (every lane stays for the sums)
  const int64_t lo = there ? first_row(team, p.teams, p.rows) : 0, hi = there ? first_row(team + 1, p.teams, p.rows) : 0;
  // teams of one warp go through the same number of rows, those past the last of a team doing nothing
  const int64_t turns = kWarps ? hi - lo : (p.rows + p.teams - 1) / p.teams;
  const T *x = static_cast<const T*>(p.x), *y = static_cast<const T*>(p.y);
  Vec<T, E> nx[V], ny[V];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      if (row < hi && col < p.dim) {
        nx[v] = load_once<T, E>(x + row * p.stride_x + col);
        ny[v] = load_once<T, E>(y + row * p.stride_y + col);
      } else {
        nx[v].clear();
        ny[v].clear();
      }
    }
  };
  fetch(lo);
  Group group(lo, p.rows_per_group);
  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row = lo + i;
    const bool live = row < hi;
    if (live) group.advance(row, p.rows_per_group);
    float r[V * E], u[V * E];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        r[v * E + e] = nx[v][e];
        u[v * E + e] = ny[v][e];
      }
    fetch(row + 1);
    // mean and 1 / deviation of values of which those past the last column are 0
    auto statistics = [&](const float (&v)[V * E], int kind, float& mean, float& rstd) {
      mean = 0.0f;
      if (kind == SPARSP_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < V * E; ++k) s[0] += v[k];
        team_sum<kWarps>(s, lanes, room, turn);
        mean = s[0] * p.inv_dim;
      }
      float q[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < V; ++k)
        if ((k * lanes + me) * E < p.dim) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float d = v[k * E + e] - mean;
            q[0] = fmaf(d, d, q[0]);
          }
        }
      team_sum<kWarps>(q, lanes, room, turn);
      rstd = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
    };
    float mean = 0.0f, rstd = 1.0f;
    if (p.norm_y != SPARSP_NORM_NONE) {
      statistics(u, p.norm_y, mean, rstd);
      if (p.stats_y != nullptr && live && me == 0) reinterpret_cast<float2*>(p.stats_y)[row] = make_float2(mean, rstd);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      if (col >= p.dim) continue;
      float g[E];
      if (p.norm_y != SPARSP_NORM_NONE) {
        float w[E], b[E];
        weights<T, E>(p.wy, kFp32Weights, col, 1.0f, w);
        weights<T, E>(p.by, kFp32Weights, col, 0.0f, b);
#pragma unroll
        for (int e = 0; e < E; ++e) u[v * E + e] = fmaf((u[v * E + e] - mean) * rstd, w[e], b[e]);
      }
      weights<T, E>(p.gate, kFp32Weights, group.index * p.dim + col, 1.0f, g);
#pragma unroll
      for (int e = 0; e < E; ++e) r[v * E + e] = fmaf(g[e], u[v * E + e], r[v * E + e]);
      if (live) {
        Vec<T, E> out;
        out.set(r + v * E);
        store_vec(static_cast<T*>(p.r) + row * p.stride_x + col, out);
      }
    }
    if (p.norm_r == SPARSP_NORM_NONE) continue;
    statistics(r, p.norm_r, mean, rstd);
    if (!live) continue;
    if (p.stats_r != nullptr && me == 0) reinterpret_cast<float2*>(p.stats_r)[row] = make_float2(mean, rstd);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      if (col >= p.dim) continue;
      float w[E], b[E];
      weights<T, E>(p.wr, kFp32Weights, group.index * p.dim + col, 1.0f, w);
      weights<T, E>(p.br, kFp32Weights, group.index * p.dim + col, 0.0f, b);
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = fmaf((r[v * E + e] - mean) * rstd, w[e], b[e]);
      Vec<T, E> out;
      out.set(w);
      store_vec(static_cast<T*>(p.n) + row * p.stride_n + col, out);
    }
  }
}

// Backward.  With a = dn wr and rh = (r - mean) rstd:  t = dr + rstd (a - sum a / dim - rh sum(a rh) / dim) = dx;
// b = t gate wy and yh = (y - mean_y) rstd_y:  dy = rstd_y (b - sum b / dim - yh sum(b yh) / dim), or t gate where y has no
// norm.  (An rms norm has mean 0 and no sum a.)  Column sums over the rows of a group, in registers: dn rh, dn, t yh (or
// t y), t; from these come all gradients of weights.
template <typename T, int V, bool kWarps, bool kFp32Weights>
__global__ void __launch_bounds__(kWarps ? 512 : 128) step_back_kernel(StepParams p) {
  enter_grid(p.x, p.y, p.dn, p.dr, p.gate, p.stats_y, p.stats_r);
  constexpr int E = 16 / sizeof(T);
  __shared__ float room[2][32][2];
  int turn = 0;
  const int lanes = kWarps ? blockDim.x : p.lanes;
  const int team = kWarps ? blockIdx.x : (blockIdx.x * blockDim.x + threadIdx.x) / lanes;
  const int me = kWarps ? threadIdx.x : threadIdx.x & (lanes - 1);
  const bool there = team < p.teams;
  const int64_t lo = there ? first_row(team, p.teams, p.rows) : 0, hi = there ? first_row(team + 1, p.teams, p.rows) : 0;
  const int64_t turns = kWarps ? hi - lo : (p.rows + p.teams - 1) / p.teams;
  const bool norm_y = p.norm_y != SPARSP_NORM_NONE, norm_r = p.norm_r != SPARSP_NORM_NONE;
  float sums[4][V * E];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int k = 0; k < V * E; ++k) sums[q][k] = 0.0f;
  Group group(lo, p.rows_per_group);
  bool first_flush = true;

  auto flush = [&] {
    // a group that this team has all of is finished here
    const bool whole = (group.index * p.rows_per_group >= lo) && (group.end <= hi || hi == p.rows);
    float* to = p.partial + (2 * team + (group.index * p.rows_per_group > lo)) * 4 * (int64_t)p.dim;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      if (col >= p.dim) continue;
      const int64_t at = group.index * p.dim + col;
      float g[E], w[E], b[E];
      if (norm_y) {
        weights<T, E>(p.gate, kFp32Weights, at, 1.0f, g);
        weights<T, E>(p.wy, kFp32Weights, col, 1.0f, w);
        weights<T, E>(p.by, kFp32Weights, col, 0.0f, b);
      }
      auto put = [&](void* out, int e, float x) {
        if (out == nullptr) return;
        if (kFp32Weights)
          static_cast<float*>(out)[at + e] = x;
        else
          static_cast<T*>(out)[at + e] = from_float<T>(x);
      };
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = v * E + e;
        if (norm_y) {
          float* py = p.partial_y + team * 2 * (int64_t)p.dim + col + e;
          py[0] = (first_flush ? 0.0f : py[0]) + g[e] * sums[2][k];
          py[p.dim] = (first_flush ? 0.0f : py[p.dim]) + g[e] * sums[3][k];
        }
        if (whole) {
          put(p.dwr, e, sums[0][k]);
          put(p.dbr, e, sums[1][k]);
          put(p.dgate, e, norm_y ? fmaf(w[e], sums[2][k], b[e] * sums[3][k]) : sums[2][k]);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) to[q * (int64_t)p.dim + col + e] = sums[q][k];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[q][k] = 0.0f;
      }
    }
    first_flush = false;
  };

  for (int64_t i = 0; i < turns; ++i) {
    const int64_t row = lo + i;
    const bool live = row < hi;
    if (live && row >= group.end) {
      flush();
      group.advance(row, p.rows_per_group);
    }
    float2 sr = make_float2(0.0f, 0.0f), sy = make_float2(0.0f, 1.0f);
    if (live && norm_r) sr = reinterpret_cast<const float2*>(p.stats_r)[row];
    if (live && norm_y) sy = reinterpret_cast<const float2*>(p.stats_y)[row];
    float t[V * E], yh[V * E], a[V * E], rh[V * E];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      const bool in = live && col < p.dim;
      Vec<T, E> vy, vr, vn, vd;
      vy.clear();
      vr.clear();
      vn.clear();
      vd.clear();
      if (in) {
        vy = load_once<T, E>(static_cast<const T*>(p.y) + row * p.stride_y + col);
        if (p.dr != nullptr) vd = load_once<T, E>(static_cast<const T*>(p.dr) + row * p.stride_x + col);
        if (norm_r) {
          vr = load_once<T, E>(static_cast<const T*>(p.x) + row * p.stride_x + col);
          vn = load_once<T, E>(static_cast<const T*>(p.dn) + row * p.stride_n + col);
        }
      }
      float w[E];
      if (in && norm_r) weights<T, E>(p.wr, kFp32Weights, group.index * p.dim + col, 1.0f, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = v * E + e;
        t[k] = vd[e];
        yh[k] = in ? (vy[e] - sy.x) * sy.y : 0.0f;
        if (norm_r) {
          const float dn = vn[e];
          rh[k] = in ? (vr[e] - sr.x) * sr.y : 0.0f;
          a[k] = in ? dn * w[e] : 0.0f;
          s[0] += a[k];
          s[1] = fmaf(a[k], rh[k], s[1]);
          sums[0][k] = fmaf(dn, rh[k], sums[0][k]);
          sums[1][k] += dn;
        }
      }
    }
    if (norm_r) {
      team_sum<kWarps>(s, lanes, room, turn);
      const float m0 = p.norm_r == SPARSP_NORM_LAYER ? s[0] * p.inv_dim : 0.0f, m1 = s[1] * p.inv_dim;
#pragma unroll
      for (int k = 0; k < V * E; ++k) t[k] = fmaf(sr.y, a[k] - m0 - rh[k] * m1, t[k]);
    }
    s[0] = s[1] = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      const bool in = live && col < p.dim;
      if (!in) continue;
      if (p.r != nullptr) {
        Vec<T, E> out;
        out.set(t + v * E);
        store_vec(static_cast<T*>(p.r) + row * p.stride_x + col, out);
      }
      float g[E], w[E];
      weights<T, E>(p.gate, kFp32Weights, group.index * p.dim + col, 1.0f, g);
      if (norm_y) weights<T, E>(p.wy, kFp32Weights, col, 1.0f, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = v * E + e;
        sums[2][k] = fmaf(t[k], yh[k], sums[2][k]);
        sums[3][k] += t[k];
        t[k] *= g[e];
        if (norm_y) {
          t[k] *= w[e];
          s[0] += t[k];
          s[1] = fmaf(t[k], yh[k], s[1]);
        }
      }
    }
    float m0 = 0.0f, m1 = 0.0f;
    if (norm_y) {
      team_sum<kWarps>(s, lanes, room, turn);
      if (p.norm_y == SPARSP_NORM_LAYER) m0 = s[0] * p.inv_dim;
      m1 = s[1] * p.inv_dim;
    }
    if (p.n == nullptr) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + me) * E;
      if (!live || col >= p.dim) continue;
      if (norm_y) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int k = v * E + e;
          t[k] = sy.y * (t[k] - m0 - yh[k] * m1);
        }
      }
      Vec<T, E> out;
      out.set(t + v * E);
      store_vec(static_cast<T*>(p.n) + row * p.stride_y + col, out);
    }
  }
  if (lo < hi) flush();
}

// Adds what the teams left: blockIdx.y < `found`: the group of that number (or, of more groups than teams, the one that
// begins in that team and goes on in others), behind them dwy and dby.  A CTA has 32 columns and 16 teams at a time.
template <typename T, bool kFp32Weights>
__global__ void __launch_bounds__(512) step_columns_kernel(StepParams p, int found, bool by_team) {
  enter_grid(p.partial, p.partial_y);
  __shared__ float room[16][4][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const bool last = (int)blockIdx.y >= found;
  int64_t group = blockIdx.y, t0 = 0, t1 = p.teams;
  if (!last) {
    if (by_team) group = (first_row((int64_t)blockIdx.y + 1, p.teams, p.rows) - 1) / p.rows_per_group;
    t0 = team_of(group * p.rows_per_group, p.teams, p.rows);
    t1 = team_of(min((group + 1) * p.rows_per_group, p.rows) - 1, p.teams, p.rows) + 1;
    if (t1 - t0 < 2 || (by_team && t0 != blockIdx.y)) return;  // (finished by its team, or found by another)
  }
  const int sums = last ? 2 : 4;
  const float* from = last ? p.partial_y : p.partial;
  // the group is the last of its first team, and the first of the others
  const int64_t behind = !last && group * p.rows_per_group > first_row(t0, p.teams, p.rows) ? 1 : 0;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (col < p.dim)
    for (int64_t t = t0 + part; t < t1; t += 16) {
      const int64_t slot = last ? t : 2 * t + (t == t0 ? behind : 0);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < sums) s[q] += from[(slot * sums + q) * p.dim + col];
    }
#pragma unroll
  for (int q = 0; q < 4; ++q) room[part][q][lane] = s[q];
  __syncthreads();
  if (part > 0 || col >= p.dim) return;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    for (int i = 1; i < 16; ++i) s[q] += room[i][q][lane];
  auto put = [&](void* out, int64_t at, float x) {
    if (out == nullptr) return;
    if (kFp32Weights)
      static_cast<float*>(out)[at] = x;
    else
      static_cast<T*>(out)[at] = from_float<T>(x);
  };
  if (last) {
    put(p.dwy, col, s[0]);
    put(p.dby, col, s[1]);
    return;
  }
  const int64_t at = group * p.dim + col;
  auto weight = [&](const void* w, float fill) {
    return w == nullptr ? fill : kFp32Weights ? static_cast<const float*>(w)[col] : to_float<T>(static_cast<const T*>(w)[col]);
  };
  put(p.dwr, at, s[0]);
  put(p.dbr, at, s[1]);
  put(p.dgate, at, p.norm_y == SPARSP_NORM_NONE ? s[2] : fmaf(weight(p.wy, 1.0f), s[2], weight(p.by, 0.0f) * s[3]));
}

// gradients of no rows
template <typename W>
__global__ void __launch_bounds__(256) step_zero_kernel(W* a, W* b, int64_t n) {
  enter_grid();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    if (a != nullptr) a[i] = from_float<W>(0.0f);
    if (b != nullptr) b[i] = from_float<W>(0.0f);
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------

static int64_t per_group(const sparsp_gated_norm& n) {
  return n.rows_per_group > 0 ? n.rows_per_group : std::max<int64_t>(n.rows, 1);
}
int64_t step_groups(const sparsp_gated_norm& n) { return (n.rows + per_group(n) - 1) / per_group(n); }

// How rows are shared out: 16-byte pieces a thread, threads of a CTA, lanes of a team, and teams.
struct StepPlan {
  int pieces, threads, lanes, ctas;
  int64_t teams;
};
static StepPlan plan_step(const sparsp_gated_norm& n, bool backward) {
  StepPlan s;
  const int each = 16 / element_bytes(n.dtype), vectors = n.dim / each;
  const int most = backward ? (n.dtype == SPARSP_FP32 ? 4 : 2) : (n.dtype == SPARSP_FP32 ? 8 : 5);
  int64_t per_cta;
  if (vectors <= 32 * most) {  // a warp, or lanes of one
    s.pieces = vectors > 32 ? (vectors + 31) / 32 : 1;
    s.threads = 128;
    s.lanes = 32;
    while (s.pieces == 1 && s.lanes > 4 && s.lanes / 2 >= vectors) s.lanes /= 2;
    per_cta = s.threads / s.lanes;
  } else {
    s.pieces = 1;
    int best = 1 << 30;
    for (int v = 1; v <= most; ++v) {
      const int threads = (vectors + 32 * v - 1) / (32 * v) * 32;
      if (threads <= 512 && threads * v <= best) {
        best = threads * v;
        s.pieces = v;
        s.threads = threads;
      }
    }
    s.lanes = s.threads;
    per_cta = 1;
  }
  const int fit = std::max(1, (backward || s.pieces > 2 ? 512 : 1024) / s.threads);  // CTAs of a multiprocessor
  s.teams = std::max<int64_t>(1, std::min<int64_t>(n.rows, (int64_t)kSms * fit * per_cta));
  s.ctas = (int)((s.teams + per_cta - 1) / per_cta);
  return s;
}

int64_t step_workspace_bytes(const sparsp_gated_norm& n) {
  const StepPlan s = plan_step(n, true);
  return 256 + s.teams * 10 * n.dim * 4;
}

static StepParams step_params(const sparsp_gated_norm& n, const StepPlan& s) {
  StepParams p = {};
  p.rows = n.rows;
  p.rows_per_group = per_group(n);
  p.stride_x = n.stride_x;
  p.stride_y = n.stride_y;
  p.stride_n = n.stride_n;
  p.dim = n.dim;
  p.teams = (int32_t)s.teams;
  p.lanes = s.lanes;
  p.norm_y = n.norm_y;
  p.norm_r = n.norm_r;
  p.eps = n.eps;
  p.inv_dim = 1.0f / n.dim;
  return p;
}

template <typename T, bool kFp32, int V>
static int launch_step(const StepPlan& s, const StepParams& p, bool backward, cudaStream_t st) {
  const bool cta = s.lanes > 32 || s.threads == s.lanes;
  auto kern = backward ? (cta ? step_back_kernel<T, V, true, kFp32> : step_back_kernel<T, V, false, kFp32>)
                       : (cta ? step_kernel<T, V, true, kFp32> : step_kernel<T, V, false, kFp32>);
  SPARSP_CUDA_OK(launch_kernel(kern, dim3((unsigned)s.ctas), s.threads, 0, st, p));
  return SPARSP_OK;
}
template <typename T, bool kFp32>
static int launch_pieces(const StepPlan& s, const StepParams& p, bool backward, cudaStream_t st) {
  switch (s.pieces) {
    case 1: return launch_step<T, kFp32, 1>(s, p, backward, st);
    case 2: return launch_step<T, kFp32, 2>(s, p, backward, st);
    case 3: return launch_step<T, kFp32, 3>(s, p, backward, st);
    case 4: return launch_step<T, kFp32, 4>(s, p, backward, st);
    case 5: return launch_step<T, kFp32, 5>(s, p, backward, st);
    case 6: return launch_step<T, kFp32, 6>(s, p, backward, st);
    case 7: return launch_step<T, kFp32, 7>(s, p, backward, st);
    default: return launch_step<T, kFp32, 8>(s, p, backward, st);
  }
}
template <typename T>
static int launch_weights(const sparsp_gated_norm& n, const StepPlan& s, const StepParams& p, bool backward,
                          cudaStream_t st) {
  if constexpr (!std::is_same<T, float>::value)
    if (n.weight_dtype != SPARSP_FP32) return launch_pieces<T, false>(s, p, backward, st);
  return launch_pieces<T, true>(s, p, backward, st);
}

int launch_gated_norm_fwd(const sparsp_gated_norm& n, const void* X, const void* Y, const void* gate, const void* wy,
                          const void* by, const void* wr, const void* br, void* R, void* N, float* stats_y,
                          float* stats_r, cudaStream_t st) {
  const StepPlan s = plan_step(n, false);
  StepParams p = step_params(n, s);
  p.x = X;
  p.y = Y;
  p.gate = gate;
  p.wy = wy;
  p.by = by;
  p.wr = wr;
  p.br = br;
  p.r = R;
  p.n = N;
  p.stats_y = stats_y;
  p.stats_r = stats_r;
  SPARSP_WITH_TYPE(n.dtype, T, { return launch_weights<T>(n, s, p, false, st); });
}

int launch_gated_norm_bwd(const sparsp_gated_norm& n, const void* dN, const void* dR, const void* R, const void* Y,
                          const void* gate, const void* wy, const void* by, const void* wr, const float* stats_y,
                          const float* stats_r, void* dX, void* dY, void* dgate, void* dwy, void* dby, void* dwr,
                          void* dbr, char* ws, cudaStream_t st) {
  const bool fp32 = n.weight_dtype == SPARSP_FP32;
  if (n.rows == 0) {
    if (dwy != nullptr || dby != nullptr)
      SPARSP_WITH_TYPE(n.weight_dtype, W, SPARSP_CUDA_OK(launch_kernel(step_zero_kernel<W>, dim3(8), 256, 0, st, (W*)dwy,
                                                                       (W*)dby, (int64_t)n.dim)));
    return SPARSP_OK;
  }
  const StepPlan s = plan_step(n, true);
  StepParams p = step_params(n, s);
  p.x = R;
  p.y = Y;
  p.dn = dN;
  p.dr = dR;
  p.gate = gate;
  p.wy = wy;
  p.by = by;
  p.wr = wr;
  p.stats_y = const_cast<float*>(stats_y);
  p.stats_r = const_cast<float*>(stats_r);
  p.r = dX;
  p.n = dY;
  p.dgate = dgate;
  p.dwy = dwy;
  p.dby = dby;
  p.dwr = dwr;
  p.dbr = dbr;
  p.partial_y = reinterpret_cast<float*>(ws + 256);
  p.partial = p.partial_y + s.teams * 2 * n.dim;
  int rc = SPARSP_OK;
  SPARSP_WITH_TYPE(n.dtype, T, rc = launch_weights<T>(n, s, p, true, st));
  if (rc != SPARSP_OK) return rc;
  const int64_t groups = step_groups(n);
  const bool by_team = groups > s.teams;
  const bool wanted = dgate != nullptr || dwr != nullptr || dbr != nullptr;
  const int found = wanted ? (int)std::min(groups, s.teams) : 0, last = dwy != nullptr || dby != nullptr;
  if (found + last == 0) return SPARSP_OK;
  const dim3 grid((unsigned)((n.dim + 31) / 32), (unsigned)(found + last));
  SPARSP_WITH_TYPE(n.dtype, T, {
    auto kern = fp32 ? step_columns_kernel<T, true> : step_columns_kernel<T, false>;
    SPARSP_CUDA_OK(launch_kernel(kern, grid, 512, 0, st, p, found, by_team));
  });
  return SPARSP_OK;
}

}  // namespace sparsp
