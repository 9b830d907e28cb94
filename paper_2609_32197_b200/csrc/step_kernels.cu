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
  int32_t dim, teams, lanes, stages, norm_y, norm_r;
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

// E values of a weight as they lie in memory, of type W, from its own 16-byte pieces.
template <typename W, int E>
struct Weights {
  static constexpr int kParts = E * (int)sizeof(W) / 16, kEach = E / kParts;
  Vec<W, kEach> part[kParts];
  __device__ __forceinline__ float operator[](int i) const { return part[i / kEach][i % kEach]; }
  // from global memory at `at`; `fill` where there is no weight
  __device__ __forceinline__ void load(const void* w, int64_t at, float fill) {
    if (w == nullptr) {
      float x[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = fill;
#pragma unroll
      for (int i = 0; i < kParts; ++i) part[i].set(x);
    } else {
#pragma unroll
      for (int i = 0; i < kParts; ++i) part[i] = load_vec<W, kEach>(static_cast<const W*>(w) + at + i * kEach);
    }
  }
};

// A thread's own 16-byte places in shared memory: nobody else's, so that nothing has to be waited for but its own copies.
// Place k is at k * threads + this thread.
struct Places {
  uint4* base;
  __device__ __forceinline__ Places() {
    extern __shared__ uint4 dynamic[];
    base = dynamic + threadIdx.x;
  }
  __device__ __forceinline__ uint4* at(int k) const { return base + k * (int)blockDim.x; }
  template <typename T, int E>
  __device__ __forceinline__ Vec<T, E> get(int k) const {
    return load_vec<T, E>(reinterpret_cast<const T*>(at(k)));
  }
  template <typename W, int E>
  __device__ __forceinline__ Weights<W, E> weights(int k) const {
    Weights<W, E> w;
#pragma unroll
    for (int i = 0; i < Weights<W, E>::kParts; ++i) w.part[i] = get<W, Weights<W, E>::kEach>(k + i);
    return w;
  }
  template <typename W, int E>
  __device__ __forceinline__ void put(int k, const Weights<W, E>& w) const {
#pragma unroll
    for (int i = 0; i < Weights<W, E>::kParts; ++i) store_vec(reinterpret_cast<W*>(at(k + i)), w.part[i]);
  }
  __device__ __forceinline__ void copy(int k, const void* from) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(at(k))), "l"(from)
                 : "memory");
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // until all but the last `behind` groups of this thread's copies have arrived
  static __device__ __forceinline__ void wait(int behind) {
    if (behind >= 3)
      asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (behind == 2)
      asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (behind == 1)
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    else
      asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
};

// Rows on their way into shared memory: `stages` rows of N tensors, V pieces each.
template <typename T, int V, int N>
struct Ring {
  Places places;
  int stages, slot, lanes, me, dim;
  const T* from[N];
  int64_t ld[N];
  __device__ __forceinline__ void fetch(int64_t row, int64_t hi) const {
    if (row < hi) {
#pragma unroll
      for (int q = 0; q < N; ++q)
        if (from[q] != nullptr) {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int col = (v * lanes + me) * (16 / (int)sizeof(T));
            if (col < dim) places.copy((slot * N + q) * V + v, from[q] + row * ld[q] + col);
          }
        }
    }
    places.commit();
  }
  __device__ __forceinline__ void start(int64_t lo, int64_t hi) {
    for (slot = 0; slot < stages; ++slot) fetch(lo + slot, hi);
    slot = 0;
  }
  __device__ __forceinline__ Vec<T, 16 / sizeof(T)> get(int q, int v) const {
    return places.get<T, 16 / sizeof(T)>((slot * N + q) * V + v);
  }
  // the row in use is done with: the one `stages` behind it takes its place
  __device__ __forceinline__ void next(int64_t row, int64_t hi) {
    fetch(row + stages, hi);
    if (++slot == stages) slot = 0;
  }
};

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

// What a thread is: of which team, and with which rows.  Teams of less than a CTA go through the same number of rows,
// those past the last of a team doing nothing, for their lanes meet in the sums.
template <bool kWarps>
struct Member {
  int lanes, team, me;
  int64_t lo, hi, turns;
  __device__ __forceinline__ Member(const StepParams& p) {
    lanes = kWarps ? blockDim.x : p.lanes;
    team = kWarps ? blockIdx.x : (blockIdx.x * blockDim.x + threadIdx.x) / lanes;
    me = kWarps ? threadIdx.x : threadIdx.x & (lanes - 1);
    const bool there = team < p.teams;
    lo = there ? first_row(team, p.teams, p.rows) : 0;
    hi = there ? first_row(team + 1, p.teams, p.rows) : 0;
    turns = kWarps ? hi - lo : (p.rows + p.teams - 1) / p.teams;
  }
};

template <typename T, typename W, int V, bool kWarps, bool kNormY>
__global__ void __launch_bounds__(kWarps ? 512 : 128, kWarps ? 2 : 8) step_kernel(StepParams p) {
  enter_grid(p.x, p.y, p.gate, p.wy, p.by, p.wr, p.br);
  constexpr int E = 16 / sizeof(T);
  __shared__ float room[2][32][2];
  int turn = 0;
  const Member<kWarps> m(p);
  Ring<T, V, 2> ring = {{}, p.stages, 0, m.lanes, m.me, p.dim, {static_cast<const T*>(p.x), static_cast<const T*>(p.y)},
                        {p.stride_x, p.stride_y}};
  ring.start(m.lo, m.hi);
  Group group(m.lo, p.rows_per_group);
  auto column = [&](int v) { return (v * m.lanes + m.me) * E; };
  // mean and 1 / deviation of values of which those past the last column are 0
  auto statistics = [&](const float (&x)[V * E], int kind, float& mean, float& rstd) {
    mean = 0.0f;
    if (kind == SPARSP_NORM_LAYER) {
      float s[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < V * E; ++k) s[0] += x[k];
      team_sum<kWarps>(s, m.lanes, room, turn);
      mean = s[0] * p.inv_dim;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (column(v) < p.dim) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = x[v * E + e] - mean;
          q[0] = fmaf(d, d, q[0]);
        }
      }
    team_sum<kWarps>(q, m.lanes, room, turn);
    rstd = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
  };
  for (int64_t i = 0; i < m.turns; ++i) {
    const int64_t row = m.lo + i;
    const bool live = row < m.hi;
    if (live) group.advance(row, p.rows_per_group);
    Places::wait(p.stages - 1);
    float r[V * E], mean = 0.0f, rstd = 1.0f;
    if constexpr (kNormY) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Vec<T, E> y;
        y.clear();
        if (live && column(v) < p.dim) y = ring.get(1, v);
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = y[e];
      }
      statistics(r, p.norm_y, mean, rstd);
      if (p.stats_y != nullptr && live && m.me == 0) reinterpret_cast<float2*>(p.stats_y)[row] = make_float2(mean, rstd);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (!live || col >= p.dim) {
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = 0.0f;
        continue;
      }
      const Vec<T, E> x = ring.get(0, v);
      Weights<W, E> g;
      g.load(p.gate, group.index * p.dim + col, 1.0f);
      if constexpr (kNormY) {
        Weights<W, E> w, b;
        w.load(p.wy, col, 1.0f);
        b.load(p.by, col, 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = fmaf(g[e], fmaf((r[v * E + e] - mean) * rstd, w[e], b[e]), x[e]);
      } else {
        const Vec<T, E> y = ring.get(1, v);
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = fmaf(g[e], y[e], x[e]);
      }
      Vec<T, E> out;
      out.set(r + v * E);
      store_vec(static_cast<T*>(p.r) + row * p.stride_x + col, out);
    }
    ring.next(row, m.hi);
    if (p.norm_r == SPARSP_NORM_NONE) continue;
    statistics(r, p.norm_r, mean, rstd);
    if (!live) continue;
    if (p.stats_r != nullptr && m.me == 0) reinterpret_cast<float2*>(p.stats_r)[row] = make_float2(mean, rstd);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (col >= p.dim) continue;
      Weights<W, E> w, b;
      w.load(p.wr, group.index * p.dim + col, 1.0f);
      b.load(p.br, group.index * p.dim + col, 0.0f);
      float n[E];
#pragma unroll
      for (int e = 0; e < E; ++e) n[e] = fmaf((r[v * E + e] - mean) * rstd, w[e], b[e]);
      Vec<T, E> out;
      out.set(n);
      store_vec(static_cast<T*>(p.n) + row * p.stride_n + col, out);
    }
  }
}

// Backward.  With a = dn wr and rh = (r - mean) rstd:  t = dr + rstd (a - sum a / dim - rh sum(a rh) / dim) = dx;
// b = t gate wy and yh = (y - mean_y) rstd_y:  dy = rstd_y (b - sum b / dim - yh sum(b yh) / dim), or t gate where y has no
// norm.  (An rms norm has mean 0 and no sum a.)  Column sums over the rows of a group, in registers: dn rh, dn, t yh (or
// t y), t; from these come all gradients of weights.  There are no registers for more: rows and weights stay in shared
// memory and are read again for each step.
template <typename T, typename W, int V, bool kWarps, bool kNormY>
__global__ void __launch_bounds__(kWarps ? 512 : 128) step_back_kernel(StepParams p) {
  enter_grid(p.x, p.y, p.dn, p.dr, p.gate, p.wy, p.wr, p.stats_y, p.stats_r);
  constexpr int E = 16 / sizeof(T), kSums = kNormY ? 4 : 3, kPart = Weights<W, E>::kParts;
  __shared__ float room[2][32][2];
  int turn = 0;
  const Member<kWarps> m(p);
  const bool norm_r = p.norm_r != SPARSP_NORM_NONE;
  enum { kDn, kR, kDr, kY };
  Ring<T, V, 4> ring = {{}, p.stages, 0, m.lanes, m.me, p.dim,
                        {static_cast<const T*>(p.dn), static_cast<const T*>(p.x), static_cast<const T*>(p.dr),
                         static_cast<const T*>(p.y)},
                        {p.stride_n, p.stride_x, p.stride_x, p.stride_y}};
  ring.start(m.lo, m.hi);
  const Places places;
  const int wr_at = p.stages * 4 * V, gate_at = wr_at + V * kPart, wy_at = gate_at + V * kPart;
  auto column = [&](int v) { return (v * m.lanes + m.me) * E; };
  Group group(m.lo, p.rows_per_group);
  auto hold_weights = [&] {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (col >= p.dim) continue;
      const int64_t at = group.index * p.dim + col;
      Weights<W, E> w;
      w.load(p.wr, at, 1.0f);
      places.put(wr_at + v * kPart, w);
      w.load(p.gate, at, 1.0f);
      places.put(gate_at + v * kPart, w);
      if (kNormY) {
        w.load(p.wy, col, 1.0f);
        places.put(wy_at + v * kPart, w);
      }
    }
  };
  if (m.lo < m.hi) hold_weights();

  float sums[kSums][V * E];
#pragma unroll
  for (int q = 0; q < kSums; ++q)
#pragma unroll
    for (int k = 0; k < V * E; ++k) sums[q][k] = 0.0f;
  bool first_flush = true;
  auto flush = [&] {
    // a group that this team has all of is finished here
    const bool whole = (group.index * p.rows_per_group >= m.lo) && (group.end <= m.hi || m.hi == p.rows);
    float* to = p.partial + (2 * (int64_t)m.team + (group.index * p.rows_per_group > m.lo)) * 4 * p.dim;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (col >= p.dim) continue;
      const int64_t at = group.index * p.dim + col;
      Weights<W, E> g, w, b;
      if (kNormY) {
        g = places.weights<W, E>(gate_at + v * kPart);
        w = places.weights<W, E>(wy_at + v * kPart);
        b.load(p.by, col, 0.0f);
      }
      auto put = [&](void* out, int e, float x) {
        if (out != nullptr) static_cast<W*>(out)[at + e] = from_float<W>(x);
      };
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int k = v * E + e;
        const float alone = kNormY ? sums[kSums - 1][k] : 0.0f;
        if (kNormY) {
          float* py = p.partial_y + (int64_t)m.team * 2 * p.dim + col + e;
          py[0] = (first_flush ? 0.0f : py[0]) + g[e] * sums[2][k];
          py[p.dim] = (first_flush ? 0.0f : py[p.dim]) + g[e] * alone;
        }
        if (whole) {
          put(p.dwr, e, sums[0][k]);
          put(p.dbr, e, sums[1][k]);
          put(p.dgate, e, kNormY ? fmaf(w[e], sums[2][k], b[e] * alone) : sums[2][k]);
        } else {
#pragma unroll
          for (int q = 0; q < kSums; ++q) to[q * (int64_t)p.dim + col + e] = sums[q][k];
        }
#pragma unroll
        for (int q = 0; q < kSums; ++q) sums[q][k] = 0.0f;
      }
    }
    first_flush = false;
  };

  // the kept statistics of a row, asked for a row ahead
  auto kept = [&](const float* from, bool norm, int64_t row) {
    return norm && row < m.hi ? reinterpret_cast<const float2*>(from)[row] : make_float2(0.0f, 1.0f);
  };
  float2 next_r = kept(p.stats_r, norm_r, m.lo), next_y = kept(p.stats_y, kNormY, m.lo);
  for (int64_t i = 0; i < m.turns; ++i) {
    const int64_t row = m.lo + i;
    const bool live = row < m.hi;
    if (live && row >= group.end) {
      flush();
      group.advance(row, p.rows_per_group);
      hold_weights();
    }
    const float2 sr = next_r, sy = next_y;
    next_r = kept(p.stats_r, norm_r, row + 1);
    next_y = kept(p.stats_y, kNormY, row + 1);
    Places::wait(p.stages - 1);
    float s[2] = {0.0f, 0.0f}, k0 = 0.0f, k1 = 0.0f;
    if (norm_r) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!live || column(v) >= p.dim) continue;
        const Vec<T, E> dn = ring.get(kDn, v), r = ring.get(kR, v);
        const Weights<W, E> w = places.weights<W, E>(wr_at + v * kPart);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int k = v * E + e;
          const float d = dn[e], a = d * w[e], rh = (r[e] - sr.x) * sr.y;
          s[0] += a;
          s[1] = fmaf(a, rh, s[1]);
          sums[0][k] = fmaf(d, rh, sums[0][k]);
          sums[1][k] += d;
        }
      }
      team_sum<kWarps>(s, m.lanes, room, turn);
      k0 = p.norm_r == SPARSP_NORM_LAYER ? s[0] * p.inv_dim : 0.0f;
      k1 = s[1] * p.inv_dim;
    }
    s[0] = s[1] = 0.0f;
    float b[V * E];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (!live || col >= p.dim) continue;
      float t[E];
      if (p.dr != nullptr) {
        const Vec<T, E> dr = ring.get(kDr, v);
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = dr[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = 0.0f;
      }
      if (norm_r) {
        const Vec<T, E> dn = ring.get(kDn, v), r = ring.get(kR, v);
        const Weights<W, E> w = places.weights<W, E>(wr_at + v * kPart);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float rh = (r[e] - sr.x) * sr.y;
          t[e] = fmaf(sr.y, fmaf(dn[e], w[e], -fmaf(rh, k1, k0)), t[e]);
        }
      }
      if (p.r != nullptr) {
        Vec<T, E> out;
        out.set(t);
        store_vec(static_cast<T*>(p.r) + row * p.stride_x + col, out);
      }
      const Vec<T, E> y = ring.get(kY, v);
      const Weights<W, E> g = places.weights<W, E>(gate_at + v * kPart);
      if constexpr (kNormY) {
        const Weights<W, E> w = places.weights<W, E>(wy_at + v * kPart);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int k = v * E + e;
          const float yh = (y[e] - sy.x) * sy.y;
          sums[2][k] = fmaf(t[e], yh, sums[2][k]);
          sums[kSums - 1][k] += t[e];
          b[k] = t[e] * g[e] * w[e];
          s[0] += b[k];
          s[1] = fmaf(b[k], yh, s[1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sums[2][v * E + e] = fmaf(t[e], y[e], sums[2][v * E + e]);
          t[e] *= g[e];
        }
        if (p.n != nullptr) {
          Vec<T, E> out;
          out.set(t);
          store_vec(static_cast<T*>(p.n) + row * p.stride_y + col, out);
        }
      }
    }
    if constexpr (kNormY) {
      team_sum<kWarps>(s, m.lanes, room, turn);
      k0 = p.norm_y == SPARSP_NORM_LAYER ? s[0] * p.inv_dim : 0.0f;
      k1 = s[1] * p.inv_dim;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = column(v);
        if (!live || col >= p.dim || p.n == nullptr) continue;
        const Vec<T, E> y = ring.get(kY, v);
        float d[E];
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = sy.y * (b[v * E + e] - fmaf((y[e] - sy.x) * sy.y, k1, k0));
        Vec<T, E> out;
        out.set(d);
        store_vec(static_cast<T*>(p.n) + row * p.stride_y + col, out);
      }
    }
    ring.next(row, m.hi);
  }
  if (m.lo < m.hi) flush();
}

// Adds what the teams left: blockIdx.y < `found`: the group of that number (or, of more groups than teams, the one that
// begins in that team and goes on in others), behind them dwy and dby.  A CTA has 32 columns and 16 teams at a time.
template <typename W>
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
        if (q < (last ? 2 : p.norm_y != SPARSP_NORM_NONE ? 4 : 3)) s[q] += from[(slot * sums + q) * p.dim + col];
    }
#pragma unroll
  for (int q = 0; q < 4; ++q) room[part][q][lane] = s[q];
  __syncthreads();
  if (part > 0 || col >= p.dim) return;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    for (int i = 1; i < 16; ++i) s[q] += room[i][q][lane];
  auto put = [&](void* out, int64_t at, float x) {
    if (out != nullptr) static_cast<W*>(out)[at] = from_float<W>(x);
  };
  if (last) {
    put(p.dwy, col, s[0]);
    put(p.dby, col, s[1]);
    return;
  }
  const int64_t at = group * p.dim + col;
  auto weight = [&](const void* w, float fill) {
    return w == nullptr ? fill : to_float<W>(static_cast<const W*>(w)[col]);
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

// How rows are shared out: 16-byte pieces a thread (16 values at most), threads of a CTA, lanes of a team, teams; rows in
// shared memory.
struct StepPlan {
  int pieces, threads, lanes, ctas, stages, smem;
  bool by_warps;
  int64_t teams;
};
constexpr int kStepSmem = 226 * 1024;  // of a multiprocessor, without what CTAs reserve

static StepPlan plan_step(const sparsp_gated_norm& n, bool backward) {
  StepPlan s;
  const int each = 16 / element_bytes(n.dtype), vectors = n.dim / each, most = 16 / each;
  int64_t per_cta = 1;
  s.by_warps = vectors <= 32 * most;
  s.pieces = 1;
  if (s.by_warps) {  // a warp, or lanes of one
    s.pieces = (vectors + 31) / 32;
    s.threads = 128;
    s.lanes = 32;
    while (s.lanes > 4 && s.lanes / 2 >= vectors) s.lanes /= 2;
    per_cta = s.threads / s.lanes;
  } else {
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
  }
  const int threads_fit = backward ? 512 : 1024;  // by registers
  int fit = std::max(1, threads_fit / s.threads);
  const int piece = s.threads * 16, stage = piece * s.pieces * (backward ? 4 : 2);
  const int held = backward ? s.pieces * 3 * piece * std::max(1, element_bytes(n.weight_dtype) / element_bytes(n.dtype)) : 0;
  auto stages = [&](int ctas) { return (kStepSmem / ctas - 1536 - held) / stage; };
  while (fit > 1 && stages(fit) < 2) --fit;
  s.stages = std::max(1, std::min(backward ? 3 : 2, stages(fit)));
  s.smem = s.stages * stage + held;
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
  p.stages = s.stages;
  p.norm_y = n.norm_y;
  p.norm_r = n.norm_r;
  p.eps = n.eps;
  p.inv_dim = 1.0f / n.dim;
  return p;
}

template <typename T, typename W, int V, bool kWarps, bool kNormY>
static int launch_kind(const StepPlan& s, const StepParams& p, bool backward, cudaStream_t st) {
  auto kern = backward ? step_back_kernel<T, W, V, kWarps, kNormY> : step_kernel<T, W, V, kWarps, kNormY>;
  SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, s.smem));
  SPARSP_CUDA_OK(launch_kernel(kern, dim3((unsigned)s.ctas), s.threads, (size_t)s.smem, st, p));
  return SPARSP_OK;
}
template <typename T, typename W, int V>
static int launch_pieces(const StepPlan& s, const StepParams& p, bool backward, cudaStream_t st) {
  if constexpr (V * 16 / (int)sizeof(T) <= 16) {
    if (s.pieces > V) return launch_pieces<T, W, V + 1>(s, p, backward, st);
    const bool norm_y = p.norm_y != SPARSP_NORM_NONE;
    if (s.by_warps)
      return norm_y ? launch_kind<T, W, V, false, true>(s, p, backward, st) : launch_kind<T, W, V, false, false>(s, p, backward, st);
    return norm_y ? launch_kind<T, W, V, true, true>(s, p, backward, st) : launch_kind<T, W, V, true, false>(s, p, backward, st);
  } else {
    return SPARSP_ERR_UNSUPPORTED;  // (plan_step has no more pieces)
  }
}
template <typename T>
static int launch_weights(const sparsp_gated_norm& n, const StepPlan& s, const StepParams& p, bool backward,
                          cudaStream_t st) {
  return n.weight_dtype == SPARSP_FP32 ? launch_pieces<T, float, 1>(s, p, backward, st)
                                       : launch_pieces<T, T, 1>(s, p, backward, st);
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
  SPARSP_WITH_TYPE(n.weight_dtype, W, SPARSP_CUDA_OK(launch_kernel(step_columns_kernel<W>, grid, 512, 0, st, p, found, by_team)));
  return SPARSP_OK;
}

}  // namespace sparsp
