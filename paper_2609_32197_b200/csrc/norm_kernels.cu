// Layer norm: forward, and backward with the reduction of the weights' gradients.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

// Rows are worked on by "workers": a warp each where a row is at most 1280 values, otherwise a CTA.  A worker has
// consecutive rows and holds the weights of the group it is in, so that they are read once per worker, not once per
// row.  It takes R rows at a time, which share each barrier; their values stay in registers from there to the store.
// The next 2R rows are on their way into shared memory: each thread copies the 16-byte pieces that it will itself
// use (cp.async), so nobody waits for anybody else's copies.  There are as many workers as fit the multiprocessors by
// their registers and their shared memory, so none waits for another to end.
//
// Rows of any length are read in 16-byte pieces.  Where a row is not a multiple of 16 bytes, every second, fourth or
// eighth row begins at the same place inside its first piece: these make a class, and a worker has rows of one class
// only, every P-th of its part, so that a thread's columns, and with them its weights and sums, do not change from row
// to row.  (Value by value, backward over 15554 x 1921 fp32 took 153 us, with single 4-byte copies 111.)
//
// Bound by HBM: 75600 x 5120 bf16 forward 245 to 264 us = 5.9 to 6.3 TB/s.  Backward, twice as much is read as written,
// by few warps, for the sums of the weights' gradients stay in registers: 380 to 423 us = 5.5 to 6.1 TB/s.

// Who works on a row, by its length: a warp up to 1280 values, otherwise a team, a CTA of as few warps as hold the row
// with 24, 32 or 40 values a thread.  Few warps with many registers are better than more with fewer: what a row costs
// beside its values (sums over the lanes, barriers, turns of the loop) is shared by more of them, the loads ahead need
// no warps, and a row that nearly fills its lanes wastes none (174000 x 1152 bf16 backward 195 us, 284 by three warps
// with 16 values a thread; 260000 x 768 215 and 260; 98000 x 2048 204 and 217; 75600 x 5120 383 to 402 and 393 to 412
// with 10 warps).  A warp takes several short rows at once: 4, 8 or 16 lanes have a row of up to 32, 64 or 128 values.
enum Worker { kWarp8, kWarp16, kWarp24, kWarp32, kWarp40, kTeam24, kTeam32, kTeam40, kWideTeam, kLongTeam };
struct WorkerKind {  // pairs: forward, backward
  int values;                    // of a thread
  int threads[2], registers[2];  // of a multiprocessor, and what that leaves a thread
  int rows[2];                   // at a time
  int ahead[2];                  // batches of so many rows in shared memory
};
// Rows at a time by what the registers hold: forward the row and two weights, backward two rows and three weights or
// sums.  Batches: one in use and two on their way, or two, the next but one of which follows the one in use to its place
// as soon as that is in registers.  With two, backward, another CTA fits a multiprocessor where rows are long (21700 x
// 4608 fp32 211 us, 261 with three); where nothing more fits, three are as good or better (300000 x 512 bf16 156 us,
// 165 with two; 75600 x 5120 forward 251 and 254).
constexpr WorkerKind kWorkers[] = {
    {8, {512, 512}, {128, 128}, {4, 2}, {3, 3}},   // kWarp8
    {16, {512, 512}, {128, 128}, {2, 1}, {3, 3}},  // kWarp16
    {24, {384, 384}, {168, 168}, {2, 1}, {3, 2}},  // kWarp24
    {32, {384, 256}, {168, 255}, {1, 1}, {3, 2}},  // kWarp32
    {40, {384, 256}, {168, 255}, {1, 1}, {3, 2}},  // kWarp40
    {24, {384, 384}, {168, 168}, {2, 1}, {3, 2}},  // kTeam24
    {32, {384, 256}, {168, 255}, {1, 1}, {3, 2}},  // kTeam32
    {40, {384, 256}, {168, 255}, {1, 1}, {3, 2}},  // kTeam40
    {32, {384, 384}, {168, 168}, {1, 1}, {3, 2}},  // kWideTeam: backward, one on a multiprocessor
    {32, {512, 512}, {128, 128}, {1, 1}, {3, 2}},  // kLongTeam
};

// Threads of a CTA whose warps are workers, where there are enough for every SM (260000 x 384 fp32 backward: 211 us,
// 239 in CTAs of 128)
__host__ __device__ constexpr int warp_threads(int kind) { return kind <= kWarp16 ? 256 : 128; }

// How a worker meets its rows.
//   kPlain    every row begins on 16 bytes and is a multiple of them
//   kShifted  rows in classes, pieces that a row shares with its neighbours
//   kSingle   value by value: tensors that do not begin on 16 bytes or whose rows move against one another, and rows
//             that shared memory does not hold
// Plain rows have a form of their own because nothing of theirs has to be masked (75600 x 5120 bf16 forward 246 us, 261
// in the other form, backward 387 and 406; 104000 x 1920 backward 210 and 240).
enum Form { kPlain, kShifted, kSingle };

// Backward, a thread's weights are in shared memory where there are no registers for them.
__host__ __device__ constexpr bool weights_shared(int form, int kind) {
  return form != kPlain || kind == kWarp40 || kind == kTeam40 || kind == kWideTeam;
}

struct NormParams {
  const void* x;
  const void* dy;
  const void* weight;
  const void* bias;
  const float* mean_in;
  const float* rstd_in;
  void* y;  // y or dx
  float* mean;
  float* rstd;
  float* partial;  // backward: [slots][2][dim]
  int64_t rows, rows_per_group, stride_x, stride_y;
  int32_t dim, weights_fp32, want_weights;
  int32_t parts, log_classes;  // workers: parts << log_classes
  int32_t ring_bytes, ring_half;  // of a worker; where dy's begins
  int32_t log_lanes;              // kWarp8: lanes of a row
  int32_t row_ctas;               // backward: the CTAs behind these add columns
  int32_t whole_groups;           // ... groups that a worker has all of are finished by it
  int32_t vector_weights;         // ... and their gradients stored four at a time
  void* dweight;
  void* dbias;
  float eps, inv_dim;
};

__host__ __device__ inline int64_t first_row(int64_t part, int64_t parts, int64_t rows) {
  return part * (rows / parts) + (part < rows % parts ? part : rows % parts);
}

// The rows of a worker: those of its class in its part.
template <bool kClasses>
struct Mine {
  int64_t lo, hi, per_group;
  int part, cls, log_of;
  __device__ __forceinline__ Mine(const NormParams& p, int worker)
      : per_group(p.rows_per_group), part(kClasses ? worker >> p.log_classes : worker),
        cls(kClasses ? worker & ((1 << p.log_classes) - 1) : 0), log_of(kClasses ? p.log_classes : 0) {
    lo = first_row(part, p.parts, p.rows);
    hi = first_row(part + 1, p.parts, p.rows);
  }
  __device__ __forceinline__ int log_classes() const { return kClasses ? log_of : 0; }
  // rows of the class below x; the class row with i such rows below it
  __device__ __forceinline__ int64_t below(int64_t x) const {
    return kClasses ? (x - cls + (1 << log_of) - 1) >> log_of : x;
  }
  __device__ __forceinline__ int64_t row(int64_t i) const { return kClasses ? cls + (i << log_of) : i; }
};

// ... in batches: at most R rows at a time, and none across two groups of weights.
template <typename M>
struct Batches {
  int64_t end;  // of the group's rows
  int left;     // of the group, yet to be fetched
  __device__ __forceinline__ Batches(const M& m) {
    end = min(m.hi, (m.lo / m.per_group + 1) * m.per_group);
    left = (int)(m.below(end) - m.below(m.lo));
    skip(m);
  }
  __device__ __forceinline__ void skip(const M& m) {
    while (left == 0 && end < m.hi) {
      const int64_t from = end;
      end = min(m.hi, end + m.per_group);
      left = (int)(m.below(end) - m.below(from));
    }
  }
  __device__ __forceinline__ int size(int R) const { return min(R, left); }
  __device__ __forceinline__ void take(const M& m, int n) {
    left -= n;
    if (left == 0) skip(m);
  }
};

// Sums N values over the worker's threads, in an order that depends on its size alone; every thread gets the sums.
// Inside a warp the values are halved with the lanes (after log2 N exchanges a lane carries one of them), so that N
// sums take little more than one.  A CTA's warps meet in `slot`, which the caller alternates so that one barrier a call
// is enough.
template <int N, bool kCta>
__device__ __forceinline__ void worker_sum(float (&v)[N], float (*slot)[N], int lanes) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = N / 2, o = 1; k > 0; k /= 2, o *= 2) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < k; ++i) {
      const float send = high ? v[i] : v[i + k], keep = high ? v[i + k] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
  float sum = v[0];  // of value `mine`
  int mine = 0;
#pragma unroll
  for (int k = N / 2, o = 1; k > 0; k /= 2, o *= 2) mine += lane & o ? k : 0;
#pragma unroll
  for (int o = N; o < 32; o *= 2)
    if (kCta || o < lanes) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if constexpr (kCta) {
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (lane < N) slot[warp][mine] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int w = lane / N; w < warps; w += 32 / N) sum += slot[w][lane % N];
#pragma unroll
    for (int o = N; o < 32; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, sum, i);
  } else {
    // lane whose bits say value i
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int from = 0;
#pragma unroll
      for (int k = N / 2, o = 1; k > 0; k /= 2, o *= 2) from |= i & k ? o : 0;
      v[i] = __shfl_sync(0xffffffffu, sum, from + (lane & -lanes));
    }
  }
}

// The rows ahead of a worker, of one tensor: in shared memory as above, or (kSingle) the next R rows in registers.
// A thread's place: among the lanes of its row, and among the threads of its worker.
struct Place {
  int lanes, t, threads, thread, at_once, sub;
  __device__ __forceinline__ Place(bool cta, bool several, int log_lanes) {
    threads = cta ? blockDim.x : 32;
    thread = cta ? threadIdx.x : (threadIdx.x & 31);
    lanes = several ? 1 << log_lanes : threads;
    t = several ? thread & (lanes - 1) : thread;
    at_once = several ? 32 >> log_lanes : 1;
    sub = several ? thread >> log_lanes : 0;
  }
};

template <typename T, int kForm, int NV, int R, int kAhead>
struct RowsAhead {
  static constexpr int E = kForm == kSingle ? 1 : 16 / sizeof(T);
  Vec<T, E> next[E > 1 ? 1 : R][E > 1 ? 1 : NV];
  const T* from;  // this thread's first piece of the next row to be fetched
  int64_t stride;
  char* ring;  // this thread's places, `threads` pieces from one to the next
  int lanes, t, dim, shift, threads;
  int at_once, sub;  // rows that a warp has at once, and which of them is this thread's

  __device__ __forceinline__ RowsAhead(const void* x, int64_t row, int64_t ld, int log_classes, char* place,
                                       const Place& me, int dim)
      : stride(ld << log_classes), lanes(me.lanes), t(me.t), dim(dim), threads(me.threads), at_once(me.at_once),
        sub(me.sub) {
    shift = kForm == kShifted ? (int)((row * ld) & (E - 1)) : 0;
    from = reinterpret_cast<const T*>(x) + row * ld - shift + t * E + sub * stride;
    ring = place + me.thread * (int)(E * sizeof(T));
    // what lies beyond the row is zero, once: nothing is ever fetched to there
    Vec<T, E> zero;
    zero.clear();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (E > 1) {
        if (column(v) >= dim)
          for (int k = 0; k < kAhead * R; ++k) store_vec(reinterpret_cast<T*>(at(k, v)), zero);
      } else {
#pragma unroll
        for (int k = 0; k < R; ++k) next[k][v] = zero;
      }
    }
  }
  // First column of the thread's piece v; below 0 where the row begins inside it.
  __device__ __forceinline__ int column(int v) const {
    return (v * lanes + t) * E - (kForm == kShifted ? shift : 0);
  }
  __device__ __forceinline__ bool whole(int v) const {
    return kForm == kShifted ? column(v) >= 0 && column(v) + E <= dim : column(v) < dim;
  }
  __device__ __forceinline__ char* at(int row, int v) const {
    return ring + (row * NV + v) * threads * (int)(E * sizeof(T));
  }
  __device__ __forceinline__ void fetch(int n, int batch) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (k * at_once + sub >= n) break;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (column(v) < dim) {
          const T* p = from + k * at_once * stride + v * lanes * E;
          if constexpr (E > 1)  // nothing past the row is read, zeros take its place
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                             (uint32_t)__cvta_generic_to_shared(at(batch * R + k, v))),
                         "l"(p), "r"(kForm == kPlain ? 16 : min(16, (dim - column(v)) * (int)sizeof(T)))
                         : "memory");
          else
            next[k][v] = load_once<T, E>(p);
        }
      }
    }
    from += n * stride;
  }
  // Row k of a batch as pairs, zeros outside the row.  Where the batch has no row k: of an earlier one, or anything.
  __device__ __forceinline__ void values(F2 (&out)[NV * E / 2], int k, int batch) const {
    float f[NV * E];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Vec<T, E> x;
      if constexpr (E > 1)
        x = load_vec<T, E>(reinterpret_cast<const T*>(at(batch * R + k, v)));
      else
        x = next[k][v];
#pragma unroll
      for (int i = 0; i < E; ++i) f[v * E + i] = x[i];
    }
    if (kForm == kShifted && shift > 0 && t == 0) {  // the end of the row before
#pragma unroll
      for (int i = 0; i < E - 1; ++i)
        if (i < shift) f[i] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < NV * E / 2; ++j) out[j] = F2(f[2 * j], f[2 * j + 1]);
  }
  // Makes zero what lies outside the row, again.
  __device__ __forceinline__ void mask(F2 (&x)[NV * E / 2]) const {
#pragma unroll
    for (int j = 0; j < NV * E / 2; ++j) {
      float a, b;
      x[j].get(a, b);
      const int c0 = column(2 * j / E) + 2 * j % E, c1 = column((2 * j + 1) / E) + (2 * j + 1) % E;
      x[j] = F2(c0 >= 0 && c0 < dim ? a : 0.0f, c1 >= 0 && c1 < dim ? b : 0.0f);
    }
  }
  __device__ __forceinline__ bool has_outside() const {
    bool any = false;
#pragma unroll
    for (int v = 0; v < NV; ++v) any = any || !whole(v);
    return any;
  }
  // Stores a row's results; `to` is the thread's first piece of it.
  __device__ __forceinline__ void store(T* to, const float (&y)[NV * E]) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (whole(v)) {
        Vec<T, E> o;
        o.set(y + v * E);
        store_vec(to + v * lanes * E, o);
      } else if (kForm == kShifted && column(v) < dim) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (column(v) + i >= 0 && column(v) + i < dim) to[v * lanes * E + i] = from_float<T>(y[v * E + i]);
      }
    }
  }
};
// One group of copies per batch of rows, an empty one past the end; at a batch's start all but the newest have to be
// there.
__device__ __forceinline__ void close_batch() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_batch() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// Where the batch after the next goes: to the one before this, or with two places to this one, which has been read.
template <int kAhead>
__device__ __forceinline__ int refilled(int at) {
  return kAhead == 2 ? at : at == 0 ? kAhead - 1 : at - 1;
}

// A thread's values of a row of weights, in 16-byte pieces where they lie so; zeros outside the row.  All loads are
// under way together.
template <typename W, int K, typename Rows>
__device__ __forceinline__ void load_row(const W* row, int dim, const Rows& rows, float (&f)[K]) {
  constexpr int E = Rows::E;
  if (E > 1 && rows.shift == 0 && dim % E == 0 && reinterpret_cast<uintptr_t>(row) % 16 == 0) {
    constexpr int N = 16 / sizeof(W);  // weights of a piece
#pragma unroll
    for (int j = 0; j < K; j += E > N ? N : E) {
      const int c = rows.column(j / E) + j % E;
      Vec<W, E == 1 ? 1 : N> x;
      x.clear();
      if (c < dim) x = load_vec<W, E == 1 ? 1 : N>(row + c);
#pragma unroll
      for (int i = 0; i < (E > N ? N : E); ++i) f[j + i] = x[i];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const int c = rows.column(j / E) + j % E;
    f[j] = c >= 0 && c < dim ? to_float<W>(row[c]) : 0.0f;
  }
}
// ... of group g
template <typename T, int K, typename Rows>
__device__ __forceinline__ void load_weights(const NormParams& p, const void* from, int64_t g, const Rows& rows,
                                             float missing, F2 (&out)[K / 2]) {
  float f[K];
  if (from == nullptr) {
#pragma unroll
    for (int j = 0; j < K; ++j) f[j] = missing;
  } else if (sizeof(T) == 4 || p.weights_fp32) {
    load_row(reinterpret_cast<const float*>(from) + g * p.dim, p.dim, rows, f);
  } else {
    load_row(reinterpret_cast<const T*>(from) + g * p.dim, p.dim, rows, f);
  }
#pragma unroll
  for (int j = 0; j < K / 2; ++j) out[j] = F2(f[2 * j], f[2 * j + 1]);
}

template <typename T, int kForm, int kKind>
__global__ void __launch_bounds__(kWorkers[kKind].threads[0], 1) norm_fwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  constexpr int E = kForm == kSingle ? 1 : 16 / sizeof(T), K = kWorkers[kKind].values, NV = K / E;
  constexpr int R = kWorkers[kKind].rows[0], kAhead = kWorkers[kKind].ahead[0];
  constexpr bool kCta = kKind >= kTeam24, kRing = E > 1;
  extern __shared__ __align__(16) char ring[];
  __shared__ float slots[4][32][R];
  const Place me(kCta, kKind == kWarp8, p.log_lanes);
  const int t = me.t, batch = R * me.at_once;
  const int worker = kCta ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (worker >= (kForm == kShifted ? p.parts << p.log_classes : p.parts)) return;
  const Mine<kForm == kShifted> m(p, worker);
  Batches<Mine<kForm == kShifted>> ahead(m);
  const int64_t r = m.row(m.below(m.lo));
  RowsAhead<T, kForm, NV, R, kAhead> rows(x, r, p.stride_x, m.log_classes(),
                                  ring + (kCta ? 0 : (threadIdx.x >> 5) * p.ring_bytes), me, p.dim);
  const bool ragged = rows.has_outside();
  const int64_t out_stride = p.stride_y << m.log_classes();
  T* out = reinterpret_cast<T*>(p.y) + r * p.stride_y - rows.shift + t * E + me.sub * out_stride;
  // n[0]: rows of the batch at work, n[1]: of the one after it
  int n[2];
  n[0] = ahead.size(batch);
  rows.fetch(n[0], 0);
  ahead.take(m, n[0]);
  n[1] = 0;
  if constexpr (kRing) {
    close_batch();
    n[1] = ahead.size(batch);
    rows.fetch(n[1], 1);
    close_batch();
    ahead.take(m, n[1]);
  }
  float* mean = p.mean == nullptr ? nullptr : p.mean + r;
  float* rstds = p.rstd + (p.mean == nullptr ? 0 : r);
  int phase = 0, at = 0;
  int64_t g = m.lo / m.per_group;
  for (int64_t a = m.lo, e; a < m.hi; a = e, ++g) {
    e = min(m.hi, (g + 1) * m.per_group);
    int left = (int)(m.below(e) - m.below(a));
    if (left == 0) continue;
    F2 w[K / 2], b[K / 2];
    load_weights<T, K>(p, p.weight, g, rows, 1.0f, w);
    load_weights<T, K>(p, p.bias, g, rows, 0.0f, b);
#pragma unroll 1
    while (left > 0) {
      if constexpr (kRing) wait_batch();
      F2 cur[R][K / 2];
      float sum[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        rows.values(cur[k], k, at);
        F2 s = cur[k][0];
#pragma unroll
        for (int j = 1; j < K / 2; ++j) s = s + cur[k][j];
        sum[k] = s.sum();
      }
      // the batch after the next: into the places that are free, or the registers that were just emptied
      const int more = ahead.size(batch);
      rows.fetch(more, refilled<kAhead>(at));
      if constexpr (kRing) close_batch();
      ahead.take(m, more);
      worker_sum<R, kCta>(sum, slots[phase], me.lanes);
      float sq[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        sum[k] *= p.inv_dim;
        const F2 minus(-sum[k]);
        F2 q(0.0f);
#pragma unroll
        for (int j = 0; j < K / 2; ++j) cur[k][j] = cur[k][j] + minus;
        if (ragged) rows.mask(cur[k]);  // what lies outside the row is no deviation
#pragma unroll
        for (int j = 0; j < K / 2; ++j) q = fma(cur[k][j], cur[k][j], q);
        sq[k] = q.sum();
      }
      worker_sum<R, kCta>(sq, slots[phase + 1], me.lanes);
      phase ^= 2;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k * me.at_once + me.sub >= n[0]) continue;
        const float rstd = rsqrtf(sq[k] * p.inv_dim + p.eps);
        const F2 scale(rstd);
        float y[K];
#pragma unroll
        for (int j = 0; j < K / 2; ++j) fma(cur[k][j] * scale, w[j], b[j]).get(y[2 * j], y[2 * j + 1]);
        rows.store(out + k * me.at_once * out_stride, y);
        if (mean != nullptr && t == 0) {
          mean[(k * me.at_once + me.sub) << m.log_classes()] = sum[k];
          rstds[(k * me.at_once + me.sub) << m.log_classes()] = rstd;
        }
      }
      out += n[0] * out_stride;
      if (mean != nullptr) {
        mean += (int64_t)n[0] << m.log_classes();
        rstds += (int64_t)n[0] << m.log_classes();
      }
      left -= n[0];
      if constexpr (kRing) {
        n[0] = n[1];
        n[1] = more;
        at = at == kAhead - 1 ? 0 : at + 1;
      } else {
        n[0] = more;
      }
    }
  }
}

__device__ __forceinline__ void store_weight(void* to, int64_t at, float v, bool fp32, bool fp16) {
  if (fp32)
    reinterpret_cast<float*>(to)[at] = v;
  else if (fp16)
    reinterpret_cast<__half*>(to)[at] = __float2half_rn(v);
  else
    reinterpret_cast<__nv_bfloat16*>(to)[at] = __float2bfloat16_rn(v);
}

// ... of four columns next to each other
template <typename T>
__device__ __forceinline__ void store_four_weights(void* to, int64_t at, const float* v, bool fp32) {
  if (to == nullptr) return;
  if constexpr (sizeof(T) == 2) {
    if (!fp32) {
      *reinterpret_cast<uint2*>(reinterpret_cast<T*>(to) + at) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
      return;
    }
  }
  *reinterpret_cast<float4*>(reinterpret_cast<float*>(to) + at) = make_float4(v[0], v[1], v[2], v[3]);
}

// Few rows: the gradients of 16 columns' weights of a group straight from x and dy, by CTAs of the launch that makes
// dx. Half a warp reads a row's columns; the sums of a thread's rows, then of the halves, then of the warps, in that
// order.
template <typename T>
__device__ __forceinline__ void add_columns(const NormParams& p, int cta, float* sums) {
  const int tiles = (p.dim + 15) / 16, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t g = cta / tiles, lo = g * p.rows_per_group, hi = min(lo + p.rows_per_group, p.rows);
  const int col = cta % tiles * 16 + (lane & 15);
  float sw = 0.0f, sb = 0.0f;
  if (col < p.dim) {
    const T* x = reinterpret_cast<const T*>(p.x) + col;
    const T* dy = reinterpret_cast<const T*>(p.dy) + col;
#pragma unroll 8
    for (int64_t row = lo + (threadIdx.x >> 4); row < hi; row += blockDim.x >> 4) {
      const float d = (float)dy[row * p.stride_y];
      sw = fmaf(d, ((float)x[row * p.stride_x] - p.mean_in[row]) * p.rstd_in[row], sw);
      sb += d;
    }
  }
  sw += __shfl_xor_sync(0xffffffffu, sw, 16);
  sb += __shfl_xor_sync(0xffffffffu, sb, 16);
  sums[threadIdx.x] = lane < 16 ? sw : sb;
  __syncthreads();
  void* to = lane < 16 ? p.dweight : p.dbias;
  if (warp > 0 || col >= p.dim || to == nullptr) return;
  float v = 0.0f;
  for (int i = lane; i < (int)blockDim.x; i += 32) v += sums[i];
  store_weight(to, g * p.dim + col, v, sizeof(T) == 4 || p.weights_fp32, std::is_same<T, __half>::value);
}

// ... in a launch of their own before dx is made, where dx takes the place of x or dy.
template <typename T>
__global__ void __launch_bounds__(512) norm_columns_kernel(const NormParams p) {
  enter_grid();
  __shared__ float sums[512];
  add_columns<T>(p, blockIdx.x, sums);
}

// The gradients of the weights are sums over rows: each worker keeps those of its rows in registers and writes them out
// where a group of its part ends.  Of P classes, class c of part i writes group g to slot (i + g) P + c, which no other
// (worker, group) has, as rows and with them groups ascend from part to part.  norm_weights_kernel adds a group's
// slots.
//
// Without classes and with as many groups as workers or more (whole_groups) most groups lie in one part, and its worker
// writes their gradients themselves.  Of those that lie across boundaries, part i writes the one that comes into it from
// before to slot 2 i and the one that goes on behind it to slot 2 i + 1, and norm_few_slots_kernel adds them.  A row of
// weights per row leaves nothing to add.  (75600 x 1920 bf16, a group a row: 412 us and 18 MB; with a slot and a CTA of
// norm_weights_kernel for each group 43 ms and 1.2 GB.)
template <typename T, int kForm, int kKind>
__global__ void __launch_bounds__(kWorkers[kKind].threads[1], 1) norm_bwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  constexpr int E = kForm == kSingle ? 1 : 16 / sizeof(T), K = kWorkers[kKind].values, NV = K / E;
  constexpr int R = kWorkers[kKind].rows[1], kAhead = kWorkers[kKind].ahead[1];
  constexpr bool kCta = kKind >= kTeam24, kRing = E > 1;
  extern __shared__ __align__(16) char ring[];
  if (blockIdx.x >= p.row_ctas) return add_columns<T>(p, blockIdx.x - p.row_ctas, reinterpret_cast<float*>(ring));
  __shared__ float slots[2][32][2 * R];
  const Place me(kCta, kKind == kWarp8, p.log_lanes);
  const int t = me.t, batch = R * me.at_once;
  const int worker = kCta ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (worker >= (kForm == kShifted ? p.parts << p.log_classes : p.parts)) return;
  const Mine<kForm == kShifted> m(p, worker);
  Batches<Mine<kForm == kShifted>> ahead(m);
  const int64_t r = m.row(m.below(m.lo));
  char* place = ring + (kCta ? 0 : (threadIdx.x >> 5) * p.ring_bytes);
  RowsAhead<T, kForm, NV, R, kAhead> xs(x, r, p.stride_x, m.log_classes(), place, me, p.dim);
  RowsAhead<T, kForm, NV, R, kAhead> ys(p.dy, r, p.stride_y, m.log_classes(), place + p.ring_half, me, p.dim);
  T* out = reinterpret_cast<T*>(p.y) + r * p.stride_x - xs.shift + t * E + me.sub * xs.stride;
  // a thread's weights, four from place to place of the threads: but for plain rows there are no registers for them
  float4* ws = reinterpret_cast<float4*>(place + p.ring_bytes - me.threads * K * 4) + me.thread;
  float mean[R], rstd[R];  // of the next batch, whose first row is row_ahead
  int64_t row_ahead = r;
  auto stats = [&](int n) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int row = k * me.at_once + me.sub;
      mean[k] = row < n ? p.mean_in[row_ahead + (row << m.log_classes())] : 0.0f;
      rstd[k] = row < n ? p.rstd_in[row_ahead + (row << m.log_classes())] : 0.0f;
    }
    row_ahead += n << m.log_classes();
  };
  int n[2];
  n[0] = ahead.size(batch);
  xs.fetch(n[0], 0);
  ys.fetch(n[0], 0);
  stats(n[0]);
  ahead.take(m, n[0]);
  n[1] = 0;
  if constexpr (kRing) {
    close_batch();
    n[1] = ahead.size(batch);
    xs.fetch(n[1], 1);
    ys.fetch(n[1], 1);
    close_batch();
    ahead.take(m, n[1]);
  }
  int phase = 0, at = 0;
  int64_t g = m.lo / m.per_group;
  for (int64_t a0 = m.lo, e; a0 < m.hi; a0 = e, ++g) {
    e = min(m.hi, (g + 1) * m.per_group);
    int left = (int)(m.below(e) - m.below(a0));
    F2 w[K / 2], dw[K / 2], db[K / 2];
    load_weights<T, K>(p, p.weight, g, xs, 1.0f, w);
    if constexpr (weights_shared(kForm, kKind)) {
#pragma unroll
      for (int j = 0; j < K / 4; ++j) {
        float4 four;
        w[2 * j].get(four.x, four.y);
        w[2 * j + 1].get(four.z, four.w);
        ws[j * me.threads] = four;
      }
    }
#pragma unroll
    for (int j = 0; j < K / 2; ++j) dw[j] = db[j] = F2(0.0f);
#pragma unroll 1
    while (left > 0) {
      if constexpr (kRing) wait_batch();
      F2 xh[R][K / 2], a[R][K / 2], scale[R];
      float sum[2 * R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        scale[k] = F2(rstd[k]);
        const F2 minus(-mean[k]);
        // outside the row there is no gradient: dy is 0 there
        xs.values(xh[k], k, at);
        ys.values(a[k], k, at);
        sum[2 * k] = sum[2 * k + 1] = 0.0f;
        if ((R > 1 || me.at_once > 1) && k * me.at_once + me.sub >= n[0]) continue;
        F2 s0(0.0f), s1(0.0f);
        float4 four;
#pragma unroll
        for (int j = 0; j < K / 2; ++j) {
          const F2 dy = a[k][j];
          if constexpr (weights_shared(kForm, kKind)) {
            if (j % 2 == 0) four = ws[j / 2 * me.threads];
            w[j] = j % 2 == 0 ? F2(four.x, four.y) : F2(four.z, four.w);
          }
          xh[k][j] = (xh[k][j] + minus) * scale[k];
          a[k][j] = dy * w[j];
          s0 = s0 + a[k][j];
          s1 = fma(a[k][j], xh[k][j], s1);
          dw[j] = fma(dy, xh[k][j], dw[j]);
          db[j] = db[j] + dy;
        }
        sum[2 * k] = s0.sum();
        sum[2 * k + 1] = s1.sum();
      }
      const int more = ahead.size(batch);
      xs.fetch(more, refilled<kAhead>(at));
      ys.fetch(more, refilled<kAhead>(at));
      if constexpr (kRing) close_batch();
      ahead.take(m, more);
      stats(kRing ? n[1] : more);
      worker_sum<2 * R, kCta>(sum, slots[phase], me.lanes);
      phase ^= 1;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k * me.at_once + me.sub >= n[0]) continue;
        const F2 c0(-sum[2 * k] * p.inv_dim), c1(-sum[2 * k + 1] * p.inv_dim);
        float dx[K];
#pragma unroll
        for (int j = 0; j < K / 2; ++j) (scale[k] * fma(xh[k][j], c1, a[k][j] + c0)).get(dx[2 * j], dx[2 * j + 1]);
        xs.store(out + k * me.at_once * xs.stride, dx);
      }
      out += n[0] * xs.stride;
      left -= n[0];
      if constexpr (kRing) {
        n[0] = n[1];
        n[1] = more;
        at = at == kAhead - 1 ? 0 : at + 1;
      } else {
        n[0] = more;
      }
    }
    if (p.want_weights) {
      // to the gradients themselves, or as fp32 to a slot
      const int64_t begin = g * m.per_group;
      const bool alone = p.whole_groups && begin >= m.lo && min(begin + m.per_group, p.rows) <= m.hi;
      const int64_t slot =
          p.whole_groups ? 2 * m.part + (begin >= m.lo) : ((m.part + g) << m.log_classes()) + m.cls;
      const bool fp32 = sizeof(T) == 4 || !alone || p.weights_fp32;
      char* to_w = reinterpret_cast<char*>(p.partial + slot * 2 * p.dim);
      char* to_b = to_w + p.dim * 4;
      if (alone) {
        const int64_t row = g * p.dim * (fp32 ? 4 : 2);
        to_w = p.dweight == nullptr ? nullptr : reinterpret_cast<char*>(p.dweight) + row;
        to_b = p.dbias == nullptr ? nullptr : reinterpret_cast<char*>(p.dbias) + row;
      }
      constexpr int S = E > 1 ? 4 : 2;  // sums that are stored together
#pragma unroll
      for (int j = 0; j < K; j += S) {
        float a[S], c[S];
#pragma unroll
        for (int i = 0; i < S; i += 2) {
          dw[(j + i) / 2].get(a[i], a[i + 1]);
          db[(j + i) / 2].get(c[i], c[i + 1]);
        }
        if constexpr (kKind == kWarp8) {
          for (int o = me.lanes; o < 32; o *= 2) {  // of the rows that the warp has at once
#pragma unroll
            for (int i = 0; i < S; ++i) {
              a[i] += __shfl_xor_sync(0xffffffffu, a[i], o);
              c[i] += __shfl_xor_sync(0xffffffffu, c[i], o);
            }
          }
        }
        if (me.sub != 0) continue;
        const int col = xs.column(j / E) + j % E;
        if (kForm == kPlain && (!alone || p.vector_weights)) {  // dim is a multiple of four, and so is the column
          if (col < p.dim) {
            store_four_weights<T>(to_w, col, a, fp32);
            store_four_weights<T>(to_b, col, c, fp32);
          }
        } else {
#pragma unroll
          for (int i = 0; i < S; ++i) {
            const int one = E > 1 ? col + i : xs.column(j + i);
            if (one < 0 || one >= p.dim) continue;
            if (to_w != nullptr) store_weight(to_w, one, a[i], fp32, std::is_same<T, __half>::value);
            if (to_b != nullptr) store_weight(to_b, one, c[i], fp32, std::is_same<T, __half>::value);
          }
        }
      }
    }
  }
}

// Parts with rows of a group: from the one that has the group's first row to the one that has its last.
struct GroupParts {
  int64_t first, last;
  __device__ __forceinline__ GroupParts(int64_t g, int64_t rows, int64_t rows_per_group, int64_t parts) {
    const int64_t lo = g * rows_per_group, hi = min(lo + rows_per_group, rows) - 1;
    const int64_t q = rows / parts, m = rows % parts;
    const int64_t cut = m * (q + 1);  // rows of the parts that have one more
    first = lo < cut ? lo / (q + 1) : m + (lo - cut) / q;
    last = hi < cut ? hi / (q + 1) : m + (hi - cut) / q;
  }
};

// Adds the slots of each group.  A CTA has kWeightColumns columns of one group; its threads take every 128th (32nd)
// slot each and meet in shared memory, so the order is the same whatever runs when.  32 columns read whole lines; with
// eight, narrow rows too have enough CTAs (70000 x 64 backward: 13.6 us, 21.3 with 32; 10000 x 8192: 112 us, 106 with
// 32).
template <int kWeightColumns>
__global__ void __launch_bounds__(1024) norm_weights_kernel(const float* partial, int64_t rows, int64_t rows_per_group,
                                                            int64_t parts, int log_classes, int dim,
                                                            void* dweight, void* dbias, int dtype) {
  enter_grid(partial);
  constexpr int kSlots = 1024 / kWeightColumns;
  __shared__ float s[2][kWeightColumns][33];
  const int tiles = (dim + kWeightColumns - 1) / kWeightColumns;
  const int64_t g = blockIdx.x / tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first = (blockIdx.x % tiles) * kWeightColumns, col = first + lane % kWeightColumns;
  float sw = 0.0f, sb = 0.0f;
  if (rows > 0) {
    const GroupParts of(g, rows, rows_per_group, parts);
    if (col < dim) {
      const int mine = threadIdx.x / kWeightColumns;
      const float* slot = partial + (((of.first + g) << log_classes) + mine) * 2 * dim + col;
#pragma unroll 4
      for (int left = (int)((of.last - of.first + 1) << log_classes) - mine; left > 0;
           left -= kSlots, slot += (int64_t)2 * kSlots * dim) {
        sw += slot[0];
        sb += slot[dim];
      }
    }
  }
#pragma unroll
  for (int o = kWeightColumns; o < 32; o *= 2) {
    sw += __shfl_xor_sync(0xffffffffu, sw, o);
    sb += __shfl_xor_sync(0xffffffffu, sb, o);
  }
  if (lane < kWeightColumns) {
    s[0][lane][warp] = sw;
    s[1][lane][warp] = sb;
  }
  __syncthreads();
  // a warp adds what the warps have of a column of dweight or dbias
  for (int i = warp; i < 2 * kWeightColumns; i += 32) {
    const int which = i / kWeightColumns, at_col = i % kWeightColumns, mine = first + at_col;
    float v = s[which][at_col][lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    void* to = which == 0 ? dweight : dbias;
    if (lane == 0 && mine < dim && to != nullptr) {
      const int64_t at = g * dim + mine;
      store_weight(to, at, v, dtype == SPARSP_FP32, dtype == SPARSP_FP16);
    }
  }
}

// ... where a group has few: a CTA has 256 columns of it, a thread one.  whole: of the groups that lie across boundaries of
// parts, a CTA for each boundary, which has work if that is its group's first.
__global__ void __launch_bounds__(256) norm_few_slots_kernel(const float* partial, int64_t rows, int64_t rows_per_group,
                                                             int64_t parts, int log_classes, int dim, bool whole,
                                                             void* dweight, void* dbias, int dtype) {
  enter_grid(partial);
  const int tiles = (dim + 255) / 256, col = (int)(blockIdx.x % tiles) * 256 + threadIdx.x;
  if (col >= dim) return;
  int64_t g = blockIdx.x / tiles;
  float sw = 0.0f, sb = 0.0f;
  const float* slot;
  int n, step;
  if (whole) {
    const int64_t part = g + 1, boundary = first_row(part, parts, rows);
    g = boundary / rows_per_group;
    const int64_t lo = g * rows_per_group;
    if (lo == boundary || first_row(part - 1, parts, rows) > lo) return;
    slot = partial + (2 * part - 1) * 2 * dim + col;
    sw = slot[0];
    sb = slot[dim];
    slot += 2 * dim;
    n = (int)(GroupParts(g, rows, rows_per_group, parts).last - part + 1);
    step = 4 * dim;
  } else {
    const GroupParts of(g, rows, rows_per_group, parts);
    slot = partial + ((of.first + g) << log_classes) * 2 * dim + col;
    n = (int)((of.last - of.first + 1) << log_classes);
    step = 2 * dim;
  }
#pragma unroll 4
  for (int i = 0; i < n; ++i, slot += step) {
    sw += slot[0];
    sb += slot[dim];
  }
  const bool fp32 = dtype == SPARSP_FP32, fp16 = dtype == SPARSP_FP16;
  if (dweight != nullptr) store_weight(dweight, g * dim + col, sw, fp32, fp16);
  if (dbias != nullptr) store_weight(dbias, g * dim + col, sb, fp32, fp16);
}

// ---- host side ------------------------------------------------------------------------------------------------------

int64_t norm_groups(const sparsp_norm& n) {
  return n.rows_per_group == 0 ? 1 : n.rows / n.rows_per_group + (n.rows % n.rows_per_group != 0);
}

// How the rows are shared out.
struct NormPlan {
  int form, kind, threads;                // threads of a CTA
  int ring_bytes, ring_half, smem_bytes;  // of a worker, where dy's begins, of a CTA
  int parts, log_classes, log_lanes;
  int resident;  // CTAs on a multiprocessor
  unsigned grid, column_ctas;  // rows', and behind them columns'
  bool whole_groups;           // backward
};

// By the values that a worker has to hold.  Teams: the least that holds them of those whose number of warps shares out
// a multiprocessor's 12 or 8 (forward 16 of kLongTeam), a whole multiprocessor's beyond 5120 (backward) or 7680.
static int worker_kind(int span, bool bwd) {
  if (span <= 1280)
    return span <= 256 ? kWarp8 : span <= 512 ? kWarp16 : span <= 768 ? kWarp24 : span <= 1024 ? kWarp32 : kWarp40;
  struct Team {
    int warps, kind;
  };
  static const Team both[] = {{2, kTeam24}, {2, kTeam32}, {3, kTeam24}, {2, kTeam40},
                              {4, kTeam24}, {4, kTeam32}, {4, kTeam40}};
  static const Team forward[] = {{6, kTeam32}, {6, kTeam40}, {8, kLongTeam}, {12, kTeam24}};
  // 17400 x 11000 bf16 backward: 234 us, 565 by kLongTeam, which has to put registers aside
  static const Team backward[] = {{8, kTeam32}, {8, kTeam40}, {12, kWideTeam}};
  const auto holds = [&](const Team& t) { return span <= t.warps * 32 * kWorkers[t.kind].values; };
  for (const Team& t : both)
    if (holds(t)) return t.kind;
  if (bwd) {
    for (const Team& t : backward)
      if (holds(t)) return t.kind;
  } else {
    for (const Team& t : forward)
      if (holds(t)) return t.kind;
  }
  return kLongTeam;
}

constexpr int kFewSlots = 24;
constexpr int kNormSmem = 224 * 1024;  // of a multiprocessor, for rings

// In classes a group has slots of every one of them: 16 bytes a column and class, written and read, beside 6 or 12 a
// column and row.  Groups of so few rows go value by value, without classes (17776 x 1921 fp32, four classes, groups of 2
// rows 187 us, 579 in classes; of 10 155 and 170; of 20 151 and 121; bf16, eight classes, of 20 150 and 230).
static bool short_groups(const sparsp_norm& n, int log_classes) {
  return n.rows_per_group > 0 && n.rows_per_group < (40 << log_classes) / (3 * element_bytes(n.dtype));
}

static NormPlan plan_norm(const sparsp_norm& n, bool pieces, bool bwd) {
  NormPlan p = {};
  const int bytes = element_bytes(n.dtype);
  p.form = kSingle;
  if (pieces) {
    const int E = 16 / bytes;
    if (n.rows > 1)
      while ((n.stride_x << p.log_classes) % E) ++p.log_classes;
    p.form = n.dim % E == 0 && p.log_classes == 0 ? kPlain : kShifted;
  }
  for (bool long_team = false;;) {
    const int E = p.form == kSingle ? 1 : 16 / bytes;
    const int units = (n.dim + (p.log_classes > 0 ? E - 1 : 0) + E - 1) / E, span = units * E;
    p.kind = long_team ? kLongTeam : worker_kind(span, bwd);
    p.log_lanes = 2;
    while (p.log_lanes < 5 && (8 << p.log_lanes) < span) ++p.log_lanes;
    const bool cta = p.kind >= kTeam24;
    const WorkerKind& kind = kWorkers[p.kind];
    const int per_thread = kind.values / E;
    p.threads = cta ? ((units + per_thread - 1) / per_thread + 31) / 32 * 32 : warp_threads(p.kind);
    int workers = cta ? 1 : p.threads / 32;  // of a CTA
    const int lanes = cta ? p.threads : 32;
    const int values = lanes * kind.values;
    p.ring_half = p.form == kSingle ? 0 : kind.ahead[bwd] * kind.rows[bwd] * values * bytes;
    p.ring_bytes = bwd ? 2 * p.ring_half + (weights_shared(p.form, p.kind) ? values * 4 : 0) : p.ring_half;
    p.smem_bytes = p.ring_bytes * workers;
    // rows of x and of dy that are too long, and a row that begins behind the first of 16384 places, do not fit
    if (p.form != kSingle && (p.smem_bytes > kNormSmem - 4096 || p.threads > kind.threads[bwd])) {
      if (p.kind == kWideTeam) {  // kLongTeam has room for 12288 in fp32 (362 us; value by value 436)
        long_team = true;
        continue;
      }
      long_team = false;
      p.form = kSingle;
      p.log_classes = 0;
      continue;
    }
    // each quarter of a multiprocessor has registers for so many warps of its own (100000 x 1536 bf16, CTAs of three
    // warps, of which six fit, not seven: forward 110 us, 130 with seven; backward 185 and 210)
    const int warps = 4 * (16384 / (32 * kind.registers[bwd]));
    p.resident = std::min({32, warps * 32 / p.threads, kNormSmem / (p.smem_bytes + 2048)});
    const int64_t rows = p.kind == kWarp8 ? (n.rows + (32 >> p.log_lanes) - 1) >> (5 - p.log_lanes) : n.rows;
    int64_t most = std::min<int64_t>(rows, (int64_t)kSms * p.resident * workers);
    // backward, a worker's sums are written and read again: four rows of its own at least, if every SM has a worker
    // (3023 x 752 fp32: 14.0 us, 17.3 with eight, 15.6 with one)
    if (bwd) most = std::min(most, std::max<int64_t>(kSms, rows / 4));
    p.parts = (int)std::max<int64_t>(1, most >> p.log_classes);
    const int all = p.parts << p.log_classes;
    p.whole_groups = bwd && norm_groups(n) >= all && p.log_classes == 0;
    // few warps go to as many SMs as there are (300 x 512 bf16 backward 6.8 us, 8.6 by eights; 64 x 256 5.2 and 5.8)
    while (workers > 1 && (all + workers - 1) / workers < kSms) workers /= 2;
    if (!cta) p.threads = 32 * workers;
    p.smem_bytes = p.ring_bytes * workers;
    p.grid = (unsigned)((all + workers - 1) / workers);
    return p;
  }
}

int64_t norm_workspace_bytes(const sparsp_norm& n) {
  int64_t slots = 0;
  for (const bool pieces : {true, false}) {
    const NormPlan p = plan_norm(n, pieces, true);
    int64_t groups = norm_groups(n);
    if (p.log_classes == 0 || short_groups(n, p.log_classes)) groups = std::min<int64_t>(groups, p.parts << p.log_classes);
    slots = std::max(slots, (p.parts + groups) << p.log_classes);
  }
  return kStatusWords * 4 + slots * 2 * n.dim * 4;
}

// Rows of all tensors have to begin at the same place of a 16-byte piece.
static bool in_pieces(const sparsp_norm& n, const void* a, const void* b, const void* c) {
  const int E = 16 / element_bytes(n.dtype);
  return (n.rows <= 1 || (n.stride_x - n.stride_y) % E == 0) && (uintptr_t)a % 16 == 0 && (uintptr_t)b % 16 == 0 &&
         (uintptr_t)c % 16 == 0;
}

static cudaError_t launch_kernel_of(void (*kern)(NormParams), const NormParams& p, const NormPlan& plan,
                                    cudaStream_t st) {
  const cudaError_t e = ensure_dynamic_smem((const void*)kern, plan.smem_bytes);
  return e != cudaSuccess ? e : launch_kernel(kern, dim3(plan.grid + plan.column_ctas), plan.threads, plan.smem_bytes, st, p);
}

template <typename T, int kForm, int kKind>
static cudaError_t launch_norm_t(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  return launch_kernel_of(bwd ? norm_bwd_kernel<T, kForm, kKind> : norm_fwd_kernel<T, kForm, kKind>, p, plan, st);
}

template <typename T, int kForm>
static cudaError_t launch_norm_f(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  switch (plan.kind) {
    case kWarp8: return launch_norm_t<T, kForm, kWarp8>(p, plan, bwd, st);
    case kTeam24: return launch_norm_t<T, kForm, kTeam24>(p, plan, bwd, st);
    case kTeam32: return launch_norm_t<T, kForm, kTeam32>(p, plan, bwd, st);
    case kTeam40: return launch_norm_t<T, kForm, kTeam40>(p, plan, bwd, st);
    case kWarp40: return launch_norm_t<T, kForm, kWarp40>(p, plan, bwd, st);
    case kWarp32: return launch_norm_t<T, kForm, kWarp32>(p, plan, bwd, st);
    case kWarp24: return launch_norm_t<T, kForm, kWarp24>(p, plan, bwd, st);
    case kWarp16: return launch_norm_t<T, kForm, kWarp16>(p, plan, bwd, st);
    case kWideTeam: return launch_kernel_of(norm_bwd_kernel<T, kForm, kWideTeam>, p, plan, st);
    default: return launch_norm_t<T, kForm, kLongTeam>(p, plan, bwd, st);
  }
}

static cudaError_t launch_norm(int dtype, const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  SPARSP_WITH_TYPE(dtype, T, {
    e = plan.form == kPlain     ? launch_norm_f<T, kPlain>(p, plan, bwd, st)
        : plan.form == kShifted ? launch_norm_f<T, kShifted>(p, plan, bwd, st)
                                : launch_norm_f<T, kSingle>(p, plan, bwd, st);
  });
  return e;
}

static NormParams norm_params(const sparsp_norm& n, const NormPlan& plan) {
  NormParams p = {};
  p.rows = n.rows;
  // (no more than there are, so that a sum of a row and a group stays far from 2^63)
  p.rows_per_group = std::max<int64_t>(n.rows_per_group == 0 ? n.rows : std::min(n.rows_per_group, n.rows), 1);
  p.stride_x = n.stride_x;
  p.stride_y = n.stride_y;
  p.dim = n.dim;
  p.weights_fp32 = n.weight_dtype == SPARSP_FP32;
  p.parts = plan.parts;
  p.log_classes = plan.log_classes;
  p.log_lanes = plan.log_lanes;
  p.ring_bytes = plan.ring_bytes;
  p.ring_half = plan.ring_half;
  p.whole_groups = plan.whole_groups;
  p.eps = n.eps;
  p.inv_dim = 1.0f / (float)n.dim;
  return p;
}

int launch_norm_fwd(const sparsp_norm& n, const void* X, const void* w, const void* b, void* Y, float* mean,
                    float* rstd, cudaStream_t st) {
  if (n.rows == 0) return SPARSP_OK;
  const NormPlan plan = plan_norm(n, in_pieces(n, X, Y, nullptr), false);
  NormParams p = norm_params(n, plan);
  p.x = X;
  p.weight = w;
  p.bias = b;
  p.y = Y;
  p.mean = mean;
  p.rstd = rstd;
  SPARSP_CUDA_OK(launch_norm(n.dtype, p, plan, false, st));
  return SPARSP_OK;
}

int launch_norm_bwd(const sparsp_norm& n, const void* dY, const void* X, const void* w, const float* mean,
                    const float* rstd, void* dX, void* dw, void* db, char* ws, cudaStream_t st) {
  NormPlan plan = plan_norm(n, in_pieces(n, X, dY, dX), true);
  if (plan.log_classes > 0 && short_groups(n, plan.log_classes) && norm_groups(n) >= plan.parts << plan.log_classes >> 2)
    plan = plan_norm(n, false, true);  // (with fewer groups than that the slots are few as well)
  NormParams p = norm_params(n, plan);
  p.want_weights = dw != nullptr || db != nullptr;
  // Few rows are added in the same launch (backward bf16 1 x 32: 2.1 us, 4.8 with sums of workers in a second launch;
  // 64 x 5120 3.6 and 10.8): up to 32 of a group a thread of add_columns, and up to ten rounds of CTAs; half of both
  // where a multiprocessor has one CTA at a time (500 x 8192 23 and 15 with 32; 2 groups of 250 x 8192, ten rounds, 29
  // and 20); up to 2^22 values, for x and dy are read twice (8 groups of 64 x 5120 15.2 and 17.3; of 250 x 5120 46 and
  // 33; 64 of 250 x 256 17.4 and 16.5; 150 of 400 x 256 51 and 26).
  const int64_t columns = norm_groups(n) * ((n.dim + 15) / 16);
  const int several = std::min(plan.resident, 2);
  const bool direct = p.want_weights && n.rows > 0 && n.rows * n.dim <= 1 << 22 &&
                      std::min(p.rows_per_group, n.rows) <= several * plan.threads &&
                      plan.grid + columns <= 5 * several * kSms * plan.resident;
  const unsigned column_ctas = (unsigned)columns;
  if (direct) p.want_weights = 0;
  p.row_ctas = (int32_t)plan.grid;
  if (n.rows > 0) {
    p.x = X;
    p.dy = dY;
    p.weight = w;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.y = dX;
    p.partial = reinterpret_cast<float*>(ws + kStatusWords * 4);
    p.dweight = dw;
    p.dbias = db;
    p.vector_weights = n.dim % 4 == 0 && (uintptr_t)dw % 16 == 0 && (uintptr_t)db % 16 == 0;
    if (direct && dX != X && dX != dY) {
      plan.column_ctas = column_ctas;
    } else if (direct) {
      SPARSP_WITH_TYPE(n.dtype, T, {
        SPARSP_CUDA_OK(launch_kernel(norm_columns_kernel<T>, dim3(column_ctas), plan.threads, 0, st, p));
      });
    }
    SPARSP_CUDA_OK(launch_norm(n.dtype, p, plan, true, st));
  }
  if (p.want_weights && norm_groups(n) > 0) {
    const int64_t groups = norm_groups(n), slots = (plan.parts + groups) << plan.log_classes;
    // few slots of a group: a thread adds a column of them (17776 x 1920 bf16, groups of 40 rows, two slots: 54 us, 296 by
    // CTAs; of 500, 12 slots, 49 and 65; of 1000, 25, 52 and 55; of 1500, 37, 56 and 51)
    if (n.rows > 0 && (plan.whole_groups || slots <= kFewSlots * groups)) {
      const int64_t items = plan.whole_groups ? (n.rows_per_group > 1 ? plan.parts - 1 : 0) : groups;
      if (items > 0)
        SPARSP_CUDA_OK(launch_kernel(norm_few_slots_kernel, dim3((unsigned)(items * ((n.dim + 255) / 256))), 256, 0, st,
                                     p.partial, n.rows, p.rows_per_group, (int64_t)plan.parts, plan.log_classes, n.dim,
                                     plan.whole_groups, dw, db, n.weight_dtype));
      return SPARSP_OK;
    }
    const bool wide = norm_groups(n) * ((n.dim + 31) / 32) >= 100;
    const int columns = wide ? 32 : 8;
    const unsigned grid = (unsigned)(norm_groups(n) * ((n.dim + columns - 1) / columns));
    SPARSP_CUDA_OK(launch_kernel(wide ? norm_weights_kernel<32> : norm_weights_kernel<8>, dim3(grid), 1024, 0, st,
                                 p.partial, n.rows, p.rows_per_group, (int64_t)plan.parts, plan.log_classes, n.dim, dw,
                                 db, n.weight_dtype));
  }
  return SPARSP_OK;
}

}  // namespace sparsp
