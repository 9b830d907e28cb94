// The residual step between two blocks of a layer: r = x + gate * u, u = norm_y(y) or y, n = norm_r(r), and its backward
// pass with the reduction of the gate's and the weights' gradients.
//
// A norm takes the difference to the mean before it scales: that of nearby values is exact, while v rstd - mean rstd, an
// operation less, is off by |mean| / deviation roundings (dweight of rows with a mean of 1000 deviations 2e-5 of itself, 1.5e-7 so).
// These operations go by pairs of values (75600 x 5120 bf16 backward, in a graph, 714 us, one by one 808).
//
// A row is worked on by a team: 4 to 32 lanes of a warp up to 512 values, otherwise a CTA.  Teams have rows of one group for
// as long as they can, so that its weights are read once for many.  The rows ahead are on their way into shared memory, each thread
// copying the 16-byte pieces that it will itself use, so that nobody waits for anybody else's copies; a thread's
// pieces lie a CTA's width apart (one behind the other, copies took twice as long: backward 75600 x 5120 1302 us, 922).
//
// Bound by HBM, forward: 75600 x 5120 bf16 500 to 538 us = 5.8 to 6.2 TB/s (weights from L1 for each row 728; with a norm of y, which
// reads them so, 970).  Backward the sums of columns take the registers that more warps would need, and a row's sums along it
// are waited for: 75600 x 5120 742 to 807 us = 5.8 to 6.3 TB/s, with norms on both sides 1220.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

struct StepParams {
  const void *x, *y;     // backward: r, y
  const void *dn, *dr;   // backward
  const void *gate, *wy, *by, *wr, *br;
  void *r, *n;           // backward: dx, dy
  float *stats_y, *stats_r;
  float* joined;               // backward: [found and last][parts][4][dim], see step_columns_kernel
  float *partial, *partial_y;  // backward: [teams][2][4][dim], of a team's first group and its last, and [teams][2][dim]
  void *dgate, *dwy, *dby, *dwr, *dbr;
  int64_t rows, rows_per_group, stride_x, stride_y, stride_n;
  int32_t dim, teams, lanes, stages, by_turns, norm_y, norm_r;
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
// of `room`, whose places of warps that are not there are 0.
template <bool kWarps, int N, int kPlaces>
__device__ __forceinline__ void team_sum(float (&v)[N], int lanes, float (*room)[4][kPlaces], int& turn) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2)
    if (kWarps || d < lanes) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    }
  if constexpr (kWarps) {
    const int warp = threadIdx.x >> 5;
    float (*at)[kPlaces] = room[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[i][warp] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float4* w = reinterpret_cast<const float4*>(at[i]);
      float s[kPlaces / 4];
#pragma unroll
      for (int k = 0; k < kPlaces / 4; ++k) s[k] = (w[k].x + w[k].y) + (w[k].z + w[k].w);
      v[i] = s[0];
#pragma unroll
      for (int k = 1; k < kPlaces / 4; ++k) v[i] += s[k];
    }
  }
}
// places of a kernel of so many threads at most, four at a time
__host__ __device__ constexpr int room_places(int threads) { return (threads / 32 + 3) / 4 * 4; }
template <int kPlaces>
__device__ __forceinline__ void clear_room(float (*room)[4][kPlaces]) {
  for (int i = threadIdx.x; i < 8 * kPlaces; i += blockDim.x) (&room[0][0][0])[i] = 0.0f;
  __syncthreads();
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

// E values to `at`, rounded to W
template <typename W, int E>
__device__ __forceinline__ void store_pieces(void* out, int64_t at, const float (&x)[E]) {
  Weights<W, E> w;
#pragma unroll
  for (int i = 0; i < Weights<W, E>::kParts; ++i) {
    w.part[i].set(x + i * Weights<W, E>::kEach);
    store_vec(static_cast<W*>(out) + at + i * Weights<W, E>::kEach, w.part[i]);
  }
}

// A thread's own 16-byte places in shared memory, each a CTA's width behind the last: nobody else's, so that nothing has to
// be waited for but its own copies; lanes' places of one number lie next to each other, in different banks.
struct Places {
  uint8_t* base;
  int pitch;
  __device__ __forceinline__ Places() {
    extern __shared__ uint4 dynamic[];
    base = reinterpret_cast<uint8_t*>(dynamic) + threadIdx.x * 16;
    pitch = blockDim.x * 16;
  }
  template <typename W, int E>
  __device__ __forceinline__ Weights<W, E> weights(int k) const {
    Weights<W, E> w;
#pragma unroll
    for (int i = 0; i < Weights<W, E>::kParts; ++i)
      w.part[i] = load_vec<W, Weights<W, E>::kEach>(reinterpret_cast<const W*>(base + (k + i) * pitch));
    return w;
  }
  template <typename W, int E>
  __device__ __forceinline__ void put(int k, const Weights<W, E>& w) const {
#pragma unroll
    for (int i = 0; i < Weights<W, E>::kParts; ++i) store_vec(reinterpret_cast<W*>(base + (k + i) * pitch), w.part[i]);
  }
};

// Rows on their way into shared memory, behind `first` places: `stages` rows of N tensors, V pieces each.  Tensor number
// q is left out where it is NULL.
template <typename T, int V, int N>
struct Ring {
  static constexpr int E = 16 / sizeof(T), kRow = N * V;
  const uint8_t* from[N];  // this thread's first piece of the next row to ask for
  int64_t step[N];
  uint8_t *begin, *end, *slot;
  int across, left, stages, pitch;  // bytes from a piece to the next; rows still to be asked for
  bool in[V];
  __device__ __forceinline__ Ring(const Places& places, int first, int stages, const void* const (&tensors)[N],
                                  const int64_t (&ld)[N], int64_t row, int64_t apart, int rows, int lanes, int me,
                                  int dim)
      : across(lanes * 16), left(rows), stages(stages) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      step[q] = ld[q] * (int)sizeof(T);
      from[q] = tensors[q] == nullptr ? nullptr : static_cast<const uint8_t*>(tensors[q]) + row * step[q] + me * 16;
      step[q] *= apart;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) in[v] = (v * lanes + me) * E < dim;
    pitch = places.pitch;
    begin = slot = places.base + first * pitch;
    end = begin + stages * kRow * pitch;
    for (int i = 0; i < stages; ++i) next();
  }
  // piece v of tensor q of the row in use, or of the one behind it
  __device__ __forceinline__ Vec<T, E> get(int q, int v, int behind = 0) const {
    const uint8_t* at = slot;
    if (behind > 0) at = slot + kRow * pitch == end ? begin : slot + kRow * pitch;
    return load_vec<T, E>(reinterpret_cast<const T*>(at + (q * V + v) * pitch));
  }
  // the row in use is done with: the one `stages` behind it takes its place
  __device__ __forceinline__ void next() {
    if (left > 0) {
      --left;
      const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
#pragma unroll
      for (int q = 0; q < N; ++q)
        if (from[q] != nullptr) {
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (in[v])
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + (q * V + v) * pitch), "l"(from[q] + v * across)
                           : "memory");
          from[q] += step[q];
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    slot = slot + kRow * pitch == end ? begin : slot + kRow * pitch;
  }
  // until the rows in use, one or two, have arrived
  __device__ __forceinline__ void wait(int rows = 1) const {
    const int behind = stages - rows;
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

// Which group a row is in, for rows that come in order.
struct Group {
  int64_t index, end;
  __device__ __forceinline__ Group(int64_t row, int64_t per) : index(row / per), end((index + 1) * per) {}
  __device__ __forceinline__ void next(int64_t per) {
    ++index;
    end += per;
  }
  __device__ __forceinline__ bool advance(int64_t row, int64_t per) {
    if (row < end) return false;
    index = row / per;
    end = (index + 1) * per;
    return true;
  }
};

// What a thread is: of which team, and with which rows.  Teams of less than a CTA go through the same number of rows,
// those past the last of a team doing nothing, for their lanes meet in the sums.  kTurns: rows may go by turns.  Backward they
// do not, and are known not to: the registers of a distance between rows are missing there (15554 x 1928 fp32 with two norms
// 157 us, 202 with it; 50000 x 8192 bf16 with two 1339 and 1988).
template <bool kWarps, bool kTurns>
struct Member {
  int lanes, team, me, rows, turns;
  int64_t lo, apart;  // first row; from one of its rows to the next
  __device__ __forceinline__ Member(const StepParams& p) {
    const bool by_turns = kTurns && p.by_turns;
    apart = by_turns ? p.teams : 1;
    lanes = kWarps ? blockDim.x : p.lanes;
    team = kWarps ? blockIdx.x : (blockIdx.x * blockDim.x + threadIdx.x) / lanes;
    me = kWarps ? threadIdx.x : threadIdx.x & (lanes - 1);
    const bool there = team < p.teams;
    lo = !there ? 0 : by_turns ? team : first_row(team, p.teams, p.rows);
    rows = !there ? 0 : (int)(by_turns ? (p.rows - team + p.teams - 1) / p.teams : first_row(team + 1, p.teams, p.rows) - lo);
    turns = kWarps ? rows : (int)((p.rows + p.teams - 1) / p.teams);
  }
};

// kNormY: y has a norm.  Without it, registers hold the weights of a group; with it there are too many.
template <typename T, typename W, int V, int kThreads, bool kNormY>
__global__ void __launch_bounds__(kThreads, 640 / kThreads) step_kernel(StepParams p) {
  constexpr bool kWarps = kThreads > 128;  // teams of 128 threads or fewer in a CTA of their own have room for 320
  enter_grid(p.x, p.y, p.gate, p.wy, p.by, p.wr, p.br);
  constexpr int E = 16 / sizeof(T);
  __shared__ __align__(16) float room[2][4][room_places(kThreads)];
  int turn = 0;
  if (kWarps) clear_room(room);
  const Member<kWarps, true> m(p);
  const Places places;
  Ring<T, V, 2> ring(places, 0, p.stages, {p.x, p.y}, {p.stride_x, p.stride_y}, m.lo, m.apart, m.rows, m.lanes, m.me, p.dim);
  Group group(m.lo, p.rows_per_group);
  Weights<W, E> gate[V], wr[V], br[V];
  auto load_weights = [&] {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (ring.in[v]) {
        const int64_t at = group.index * p.dim + (v * m.lanes + m.me) * E;
        gate[v].load(p.gate, at, 1.0f);
        wr[v].load(p.wr, at, 1.0f);
        br[v].load(p.br, at, 0.0f);
      }
  };
  if (!kNormY) load_weights();
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
      if (ring.in[v]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = x[v * E + e] - mean;
          q[0] = fmaf(d, d, q[0]);
        }
      }
    team_sum<kWarps>(q, m.lanes, room, turn);
    rstd = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
  };
  T* to_r = static_cast<T*>(p.r) + m.lo * p.stride_x + m.me * E;
  T* to_n = static_cast<T*>(p.n) + m.lo * p.stride_n + m.me * E;
  int64_t row = m.lo;
  for (int i = 0; i < m.turns; ++i, row += m.apart, to_r += m.apart * p.stride_x, to_n += m.apart * p.stride_n) {
    const bool live = i < m.rows;
    if (live && group.advance(row, p.rows_per_group) && !kNormY) load_weights();
    ring.wait();
    float r[V * E], mean = 0.0f, rstd = 1.0f;
    if constexpr (kNormY) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Vec<T, E> y;
        y.clear();
        if (live && ring.in[v]) y = ring.get(1, v);
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = y[e];
      }
      statistics(r, p.norm_y, mean, rstd);
      if (p.stats_y != nullptr && live && m.me == 0)
        reinterpret_cast<float2*>(p.stats_y)[row] = make_float2(mean, rstd);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!live || !ring.in[v]) {
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = 0.0f;
        continue;
      }
      const Vec<T, E> x = ring.get(0, v);
      if constexpr (kNormY) {
        const int col = (v * m.lanes + m.me) * E;
        Weights<W, E> g, w, b;
        g.load(p.gate, group.index * p.dim + col, 1.0f);
        w.load(p.wy, col, 1.0f);
        b.load(p.by, col, 0.0f);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          float* at = r + v * E + e;
          ((F2(at[0], at[1]) + F2(-mean)) * F2(rstd)).get(at[0], at[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i) at[i] = fmaf(g[e + i], fmaf(at[i], w[e + i], b[e + i]), x[e + i]);
        }
      } else {
        const Vec<T, E> y = ring.get(1, v);
#pragma unroll
        for (int e = 0; e < E; ++e) r[v * E + e] = fmaf(gate[v][e], y[e], x[e]);
      }
      Vec<T, E> out;
      out.set(r + v * E);
      store_vec(to_r + v * m.lanes * E, out);
    }
    ring.next();
    if (p.norm_r == SPARSP_NORM_NONE) continue;
    statistics(r, p.norm_r, mean, rstd);
    if (!live) continue;
    if (p.stats_r != nullptr && m.me == 0) reinterpret_cast<float2*>(p.stats_r)[row] = make_float2(mean, rstd);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!ring.in[v]) continue;
      if constexpr (kNormY) {
        const int64_t at = group.index * p.dim + (v * m.lanes + m.me) * E;
        wr[v].load(p.wr, at, 1.0f);
        br[v].load(p.br, at, 0.0f);
      }
      float n[E];
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        ((F2(r[v * E + e], r[v * E + e + 1]) + F2(-mean)) * F2(rstd)).get(n[e], n[e + 1]);
#pragma unroll
        for (int i = e; i < e + 2; ++i) n[i] = fmaf(n[i], wr[v][i], br[v][i]);
      }
      Vec<T, E> out;
      out.set(n);
      store_vec(to_n + v * m.lanes * E, out);
    }
  }
}

// Backward.  With a = dn wr and rh = (r - mean) rstd:  t = dr + rstd (a - sum a / dim - rh sum(a rh) / dim) = dx;
// b = t gate wy and yh = (y - mean_y) rstd_y:  dy = rstd_y (b - sum b / dim - yh sum(b yh) / dim), or t gate where y has no
// norm.  (An rms norm has mean 0 and no sum a.)  Column sums over the rows of a group, in registers: dn rh, dn, t yh (or
// t y), t; from these come all gradients of weights.  There are no registers for more: rows and weights stay in shared
// memory and are read again for each step.
template <typename T, typename W, int V, int kThreads, int R, bool kNormY>
__global__ void __launch_bounds__(kThreads, kThreads == 320 && R == 1 ? 2 : 1) step_back_kernel(StepParams p) {
  constexpr bool kWarps = kThreads > 128;  // teams of 128 threads or fewer in a CTA of their own have room for 320
  enter_grid(p.x, p.y, p.dn, p.dr, p.gate, p.wy, p.by, p.wr, p.stats_y, p.stats_r);
  constexpr int E = 16 / sizeof(T), kSums = kNormY ? 4 : 3, kPart = Weights<W, E>::kParts;
  __shared__ __align__(16) float room[2][4][room_places(kThreads)];
  int turn = 0;
  if (kWarps) clear_room(room);
  const Member<kWarps, false> m(p);
  const bool norm_r = p.norm_r != SPARSP_NORM_NONE;
  enum { kDn, kR, kDr, kY };
  const Places places;
  constexpr int kWrAt = 0, kGateAt = V * kPart, kWyAt = 2 * V * kPart;  // then rows
  Ring<T, V, 4> ring(places, (kNormY ? 3 : 2) * V * kPart, p.stages, {p.dn, p.x, p.dr, p.y},
                     {p.stride_n, p.stride_x, p.stride_x, p.stride_y}, m.lo, m.apart, m.rows, m.lanes, m.me, p.dim);
  const int64_t hi = m.lo + m.rows;
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
      places.put(kWrAt + v * kPart, w);
      w.load(p.gate, at, 1.0f);
      places.put(kGateAt + v * kPart, w);
      if (kNormY) {
        w.load(p.wy, col, 1.0f);
        places.put(kWyAt + v * kPart, w);
      }
    }
  };
  if (m.rows > 0) hold_weights();

  float sums[kSums][V * E];
#pragma unroll
  for (int q = 0; q < kSums; ++q)
#pragma unroll
    for (int k = 0; k < V * E; ++k) sums[q][k] = 0.0f;
  bool first_flush = true;
  auto flush = [&] {
    // a group that this team has all of is finished here
    const bool whole = (group.index * p.rows_per_group >= m.lo) && (group.end <= hi || hi == p.rows);
    float* to = p.partial + (2 * (int64_t)m.team + (group.index * p.rows_per_group > m.lo)) * 4 * p.dim;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = column(v);
      if (col >= p.dim) continue;
      const int64_t at = group.index * p.dim + col;
      Weights<W, E> g, w, b;
      if (kNormY) {
        g = places.weights<W, E>(kGateAt + v * kPart);
        w = places.weights<W, E>(kWyAt + v * kPart);
        b.load(p.by, col, 0.0f);
      }
      auto sum = [&](int q, float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = sums[q][v * E + e];
      };
      float x[E], y[E];
      if (kNormY) {
        float* py = p.partial_y + (int64_t)m.team * 2 * p.dim + col;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          Weights<float, E> held;
          if (!first_flush) held.load(py, q * (int64_t)p.dim, 0.0f);
          sum(q == 0 ? 2 : kSums - 1, x);
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = first_flush ? g[e] * x[e] : fmaf(g[e], x[e], held[e]);
          store_pieces<float, E>(py, q * (int64_t)p.dim, x);
        }
      }
      if (whole) {
        sum(0, x);
        if (p.dwr != nullptr) store_pieces<W, E>(p.dwr, at, x);
        sum(1, x);
        if (p.dbr != nullptr) store_pieces<W, E>(p.dbr, at, x);
        sum(2, x);
        if (kNormY) {
          sum(kSums - 1, y);
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = fmaf(w[e], x[e], b[e] * y[e]);
        }
        if (p.dgate != nullptr) store_pieces<W, E>(p.dgate, at, x);
      } else {
#pragma unroll
        for (int q = 0; q < kSums; ++q) {
          sum(q, x);
          store_pieces<float, E>(to, q * (int64_t)p.dim + col, x);
        }
      }
#pragma unroll
      for (int q = 0; q < kSums; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[q][v * E + e] = 0.0f;
    }
    first_flush = false;
  };

  // the kept statistics of rows, asked for a turn ahead
  auto kept = [&](const float* from, bool norm, int64_t row) {
    return norm && row < hi ? reinterpret_cast<const float2*>(from)[row] : make_float2(0.0f, 1.0f);
  };
  float2 next_r[R], next_y[R];
  auto ask = [&](int64_t row) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      next_r[q] = kept(p.stats_r, norm_r, row + q);
      next_y[q] = kept(p.stats_y, kNormY, row + q);
    }
  };
  ask(m.lo);
  T* to_x = static_cast<T*>(p.r) + m.lo * p.stride_x + m.me * E;
  T* to_y = static_cast<T*>(p.n) + m.lo * p.stride_y + m.me * E;
  // C rows of one group
  auto process = [&](auto count, const float2 (&sr)[R], const float2 (&sy)[R], bool live) {
    constexpr int C = decltype(count)::value;
    float k0[C], k1[C];
#pragma unroll
    for (int q = 0; q < C; ++q) k0[q] = k1[q] = 0.0f;
    float s[2 * C];
    auto along_rows = [&](int kind, const float2 (&kept)[R]) {
      team_sum<kWarps>(s, m.lanes, room, turn);
#pragma unroll
      for (int q = 0; q < C; ++q) {
        k1[q] = s[2 * q + 1] * p.inv_dim;
        k0[q] = kind == SPARSP_NORM_LAYER ? s[2 * q] * p.inv_dim : 0.0f;
        k1[q] *= kept[q].y;  // (of the difference to the mean)
        s[2 * q] = s[2 * q + 1] = 0.0f;
      }
    };
#pragma unroll
    for (int q = 0; q < 2 * C; ++q) s[q] = 0.0f;
    if (norm_r) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!live || !ring.in[v]) continue;
        const Weights<W, E> w = places.weights<W, E>(kWrAt + v * kPart);
#pragma unroll
        for (int q = 0; q < C; ++q) {
          const Vec<T, E> dn = ring.get(kDn, v, q), r = ring.get(kR, v, q);
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            float rh[2];
            ((F2(r[e], r[e + 1]) + F2(sr[q].x)) * F2(sr[q].y)).get(rh[0], rh[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int k = v * E + e + i;
              const float d = dn[e + i], a = d * w[e + i];
              s[2 * q] += a;
              s[2 * q + 1] = fmaf(a, rh[i], s[2 * q + 1]);
              sums[0][k] = fmaf(d, rh[i], sums[0][k]);
              sums[1][k] += d;
            }
          }
        }
      }
      along_rows(p.norm_r, sr);
    }
    float b[kNormY ? C : 1][V * E];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!live || !ring.in[v]) continue;
#pragma unroll
      for (int q = 0; q < C; ++q) {
        float t[E];
        if (p.dr != nullptr) {
          const Vec<T, E> dr = ring.get(kDr, v, q);
#pragma unroll
          for (int e = 0; e < E; ++e) t[e] = dr[e];
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) t[e] = 0.0f;
        }
        if (norm_r) {
          const Vec<T, E> dn = ring.get(kDn, v, q), r = ring.get(kR, v, q);
          const Weights<W, E> w = places.weights<W, E>(kWrAt + v * kPart);
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            float line[2];
            fma(F2(r[e], r[e + 1]) + F2(sr[q].x), F2(k1[q]), F2(k0[q])).get(line[0], line[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) t[e + i] = fmaf(sr[q].y, fmaf(dn[e + i], w[e + i], -line[i]), t[e + i]);
          }
        }
        if (p.r != nullptr) {
          Vec<T, E> out;
          out.set(t);
          store_vec(to_x + q * p.stride_x + v * m.lanes * E, out);
        }
        const Vec<T, E> y = ring.get(kY, v, q);
        const Weights<W, E> g = places.weights<W, E>(kGateAt + v * kPart);
        if constexpr (kNormY) {
          const Weights<W, E> wy = places.weights<W, E>(kWyAt + v * kPart);
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            float yh[2];
            ((F2(y[e], y[e + 1]) + F2(sy[q].x)) * F2(sy[q].y)).get(yh[0], yh[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int k = v * E + e + i;
              sums[2][k] = fmaf(t[e + i], yh[i], sums[2][k]);
              sums[kSums - 1][k] += t[e + i];
              b[q][k] = t[e + i] * g[e + i] * wy[e + i];
              s[2 * q] += b[q][k];
              s[2 * q + 1] = fmaf(b[q][k], yh[i], s[2 * q + 1]);
            }
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
            store_vec(to_y + q * p.stride_y + v * m.lanes * E, out);
          }
        }
      }
    }
    if constexpr (kNormY) {
      along_rows(p.norm_y, sy);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!live || !ring.in[v] || p.n == nullptr) continue;
#pragma unroll
        for (int q = 0; q < C; ++q) {
          const Vec<T, E> y = ring.get(kY, v, q);
          float d[E];
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            float line[2];
            fma(F2(y[e], y[e + 1]) + F2(sy[q].x), F2(k1[q]), F2(k0[q])).get(line[0], line[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) d[e + i] = sy[q].y * (b[q][v * E + e + i] - line[i]);
          }
          Vec<T, E> out;
          out.set(d);
          store_vec(to_y + q * p.stride_y + v * m.lanes * E, out);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < C; ++q) ring.next();
    to_x += C * p.stride_x;
    to_y += C * p.stride_y;
  };
  for (int i = 0; i < m.turns;) {
    const int64_t row = m.lo + i;
    const bool live = i < m.rows;
    if (live && row >= group.end) {
      flush();
      group.next(p.rows_per_group);  // (rows come one by one)
      hold_weights();
    }
    const bool two = R == 2 && row + 1 < hi && row + 1 < group.end;
    float2 sr[R], sy[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      sr[q] = make_float2(-next_r[q].x, next_r[q].y);
      sy[q] = make_float2(-next_y[q].x, next_y[q].y);
    }
    ask(row + (two ? 2 : 1));
    ring.wait(R);
    if (R == 2 && two)
      process(std::integral_constant<int, R>(), sr, sy, true);
    else
      process(std::integral_constant<int, 1>(), sr, sy, live);
    i += two ? 2 : 1;
  }
  if (m.rows > 0) flush();
}

// What the sums of 32 columns are of: blockIdx.y < `found`: the group of that number (or, of more groups than teams, the one
// that begins in that team and goes on in others), behind them dwy and dby.
struct Columns {
  int64_t group, t0, t1;  // teams that have rows of it
  bool last, none;        // none: finished by its team, or found by another
  __device__ __forceinline__ Columns(const StepParams& p, int found, bool by_team)
      : group(blockIdx.y), t0(0), t1(p.teams), last((int)blockIdx.y >= found), none(false) {
    if (last) return;
    if (by_team) group = (first_row((int64_t)blockIdx.y + 1, p.teams, p.rows) - 1) / p.rows_per_group;
    t0 = team_of(group * p.rows_per_group, p.teams, p.rows);
    t1 = team_of(min((group + 1) * p.rows_per_group, p.rows) - 1, p.teams, p.rows) + 1;
    none = t1 - t0 < 2 || (by_team && t0 != blockIdx.y);
  }
  template <typename W>
  __device__ __forceinline__ void finish(const StepParams& p, int col, const float (&s)[4]) const {
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
};

// Adds what the teams left.  A CTA has 32 columns and 16 teams at a time; where there are few columns and many teams,
// gridDim.z CTAs share the teams out, and step_join_kernel adds their sums (75600 x 64 bf16, all of the backward pass: 153 us
// with one CTA for 32 columns, 45 so).
template <typename W>
__global__ void __launch_bounds__(512) step_columns_kernel(StepParams p, int found, bool by_team) {
  enter_grid(p.partial, p.partial_y, p.wy, p.by);
  __shared__ float room[16][4][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const Columns c(p, found, by_team);
  if (c.none) return;
  const int sums = c.last ? 2 : 4;
  const float* from = c.last ? p.partial_y : p.partial;
  // the group is the last of its first team, and the first of the others
  const int64_t behind = !c.last && c.group * p.rows_per_group > first_row(c.t0, p.teams, p.rows) ? 1 : 0;
  const int64_t begin = c.t0 + first_row(blockIdx.z, gridDim.z, c.t1 - c.t0);
  const int64_t end = c.t0 + first_row(blockIdx.z + 1, gridDim.z, c.t1 - c.t0);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const int there = c.last ? 2 : p.norm_y != SPARSP_NORM_NONE ? 4 : 3;
  if (col < p.dim)
#pragma unroll 4
    for (int64_t t = begin + part; t < end; t += 16) {
      const int64_t slot = c.last ? t : 2 * t + (t == c.t0 ? behind : 0);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < there) s[q] += from[(slot * sums + q) * p.dim + col];
    }
#pragma unroll
  for (int q = 0; q < 4; ++q) room[part][q][lane] = s[q];
  __syncthreads();
  if (part > 0 || col >= p.dim) return;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    for (int i = 1; i < 16; ++i) s[q] += room[i][q][lane];
  if (gridDim.z == 1) {
    c.finish<W>(p, col, s);
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) p.joined[(((int64_t)blockIdx.y * gridDim.z + blockIdx.z) * 4 + q) * p.dim + col] = s[q];
}
template <typename W>
__global__ void __launch_bounds__(32) step_join_kernel(StepParams p, int found, bool by_team, int parts) {
  enter_grid(p.joined, p.wy, p.by);
  const int col = blockIdx.x * 32 + threadIdx.x;
  const Columns c(p, found, by_team);
  if (c.none || col >= p.dim) return;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int z = 0; z < parts; ++z)
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] += p.joined[(((int64_t)blockIdx.y * parts + z) * 4 + q) * p.dim + col];
  c.finish<W>(p, col, s);
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
  const int64_t all = std::max<int64_t>(n.rows, 1);  // (any number that is not less is one group)
  return n.rows_per_group > 0 ? std::min(n.rows_per_group, all) : all;
}
int64_t step_groups(const sparsp_gated_norm& n) { return (n.rows + per_group(n) - 1) / per_group(n); }

// How rows are shared out: 16-byte pieces a thread (16 values at most), threads of a CTA, lanes of a team, teams; rows in
// shared memory.
struct StepPlan {
  int pieces, threads, lanes, ctas, stages, smem;
  bool by_warps, two_rows;
  int64_t teams;
};
constexpr int kStepSmem = 228 * 1024;  // of a multiprocessor; each CTA has 1 KB more than it asks for

static StepPlan plan_step(const sparsp_gated_norm& n, bool backward) {
  StepPlan s;
  const int each = 16 / element_bytes(n.dtype), vectors = n.dim / each;
  int64_t per_cta = 1;
  s.by_warps = n.dim <= 32 * 16;
  // Values of a thread, and threads that registers then hold: of a CTA, of a multiprocessor.  Backward, 8 values leave room
  // for twice the warps (15554 x 1928 fp32 with two norms 168 us, 216 with 16); where only one CTA fits, 16, and two rows
  // at a time whose sums are waited for together (75600 x 5120 bf16 843, 962 with 8 and one row, 922 with 16 and one;
  // 714 now).
  // Two rows take 157 to 168 registers: 384 threads, two CTAs up to 192 (40000 x 2816 bf16 240 us, 279 with one, 335 with 8 values
  // and one row, with a norm of y 344, 502 and 867; x 4096 with one 313, with two of which one has to wait 421).  A
  // norm of y over more than 4 values of lanes of a warp takes 158 to 224: two CTAs of 128 (75600 x 512 bf16 115 us, 155 with
  // four, x 256 85 and 90).
  s.two_rows = backward && each == 8 && n.dim > 320 * 8 && n.dim <= 320 * 16;
  const int values = backward && !s.by_warps && !s.two_rows && n.dim <= 640 * 8 ? 8 : 16, most = values / each;
  const int most_threads = values == 8 ? 640 : 512;
  s.pieces = 1;
  if (s.by_warps) {  // a warp, or lanes of one
    s.pieces = (vectors + 31) / 32;
    s.threads = 128;
    s.lanes = 32;
    while (s.lanes > 4 && s.lanes / 2 >= vectors) s.lanes /= 2;
    per_cta = s.threads / s.lanes;
  } else {
    int best = 1 << 30;
    for (int v = s.two_rows ? most : 1; v <= most; ++v) {
      const int threads = (vectors + 32 * v - 1) / (32 * v) * 32;
      if (threads <= most_threads && threads * v <= best) {
        best = threads * v;
        s.pieces = v;
        s.threads = threads;
      }
    }
    s.lanes = s.threads;
  }
  // CTAs of a multiprocessor by what registers hold
  const bool many_sums = s.by_warps && n.norm_y != SPARSP_NORM_NONE && s.pieces * each > 4;
  const int all_threads = !backward || values == 8 ? 640 : s.two_rows ? 384 : many_sums ? 256 : 512;
  int fit = std::max(1, all_threads / s.threads);
  const int row = s.pieces * (backward ? 4 : 2);
  const int per_weight = std::max(1, element_bytes(n.weight_dtype) / element_bytes(n.dtype));
  const int held = backward ? s.pieces * per_weight * (n.norm_y != SPARSP_NORM_NONE ? 3 : 2) : 0;
  auto fits = [&](int places, int ctas) { return (places * s.threads * 16 + 1024 + 256) * ctas <= kStepSmem; };
  auto stages = [&](int ctas) {
    int k = s.two_rows ? 4 : backward ? 3 : 2;  // (forward 75600 x 5120 bf16 532 us, 550 with three)
    while (k > 0 && !fits(k * row + held, ctas)) --k;
    return k;
  };
  while (fit > 1 && stages(fit) < 2) --fit;
  s.stages = std::max(1, stages(fit));
  s.smem = (s.stages * row + held) * s.threads * 16;
  s.teams = std::max<int64_t>(1, std::min<int64_t>(n.rows, (int64_t)kSms * fit * per_cta));
  s.ctas = (int)((s.teams + per_cta - 1) / per_cta);
  return s;
}

constexpr int kMostJoined = 4 * kSms;  // sums of 32 columns that CTAs share out, times those CTAs

int64_t step_workspace_bytes(const sparsp_gated_norm& n) {
  const StepPlan s = plan_step(n, true);
  return 256 + (s.teams * 10 + kMostJoined * 4) * n.dim * 4;
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

template <typename T, typename W, int V, int kThreads, bool kBack, int R = 1>
static int launch_kind(const StepPlan& s, const StepParams& p, cudaStream_t st) {
  auto launch = [&](auto kern) {
    SPARSP_CUDA_OK(ensure_dynamic_smem((const void*)kern, s.smem));
    SPARSP_CUDA_OK(launch_kernel(kern, dim3((unsigned)s.ctas), s.threads, (size_t)s.smem, st, p));
    return (int)SPARSP_OK;
  };
  if constexpr (kBack)
    return p.norm_y != SPARSP_NORM_NONE ? launch(step_back_kernel<T, W, V, kThreads, R, true>)
                                        : launch(step_back_kernel<T, W, V, kThreads, R, false>);
  else
    return p.norm_y != SPARSP_NORM_NONE ? launch(step_kernel<T, W, V, kThreads, true>)
                                        : launch(step_kernel<T, W, V, kThreads, false>);
}
template <typename T, typename W, int V>
static int launch_pieces(const StepPlan& s, const StepParams& p, bool backward, cudaStream_t st) {
  constexpr int kValues = V * 16 / (int)sizeof(T);
  if constexpr (kValues <= 16) {
    if (s.pieces > V) return launch_pieces<T, W, V + 1>(s, p, backward, st);
    if (!backward) {
      if (s.by_warps) return launch_kind<T, W, V, 128, false>(s, p, st);
      return s.threads <= 320 ? launch_kind<T, W, V, 320, false>(s, p, st) : launch_kind<T, W, V, 512, false>(s, p, st);
    }
    if (s.by_warps) return launch_kind<T, W, V, 128, true>(s, p, st);
    if constexpr (kValues <= 8) {
      return s.threads <= 320 ? launch_kind<T, W, V, 320, true>(s, p, st) : launch_kind<T, W, V, 640, true>(s, p, st);
    } else {
      if constexpr (sizeof(T) == 2)
        if (s.two_rows) return launch_kind<T, W, V, 320, true, 2>(s, p, st);
      return launch_kind<T, W, V, 512, true>(s, p, st);
    }
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
  // Teams take rows by turns, so that those at work at one time lie near each other (75600 x 5120 bf16 525 us, 532 with rows
  // one behind the other), unless a team would meet new weights every few rows.
  p.by_turns = p.rows_per_group >= 16 * s.teams || p.rows_per_group >= n.rows;
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
  p.joined = p.partial + s.teams * 8 * n.dim;
  // CTAs for a sum: up to two for each SM in all, 32 teams for one at least (1: no second launch)
  const int columns = (n.dim + 31) / 32, sums = found + last;
  int parts = (int)std::min<int64_t>(2 * kSms / ((int64_t)columns * sums), s.teams / std::min(groups, s.teams) / 32);
  if (parts < 2) parts = 1;
  const dim3 grid((unsigned)columns, (unsigned)sums, (unsigned)parts);
  SPARSP_WITH_TYPE(n.weight_dtype, W, {
    SPARSP_CUDA_OK(launch_kernel(step_columns_kernel<W>, grid, 512, 0, st, p, found, by_team));
    if (parts > 1)
      SPARSP_CUDA_OK(launch_kernel(step_join_kernel<W>, dim3((unsigned)columns, (unsigned)sums), 32, 0, st, p, found, by_team,
                                   parts));
  });
  return SPARSP_OK;
}

}  // namespace sparsp
