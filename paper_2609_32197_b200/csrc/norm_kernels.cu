// Layer norm: forward, and backward with the reduction of the weights' gradients.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

// Rows are worked on by "workers": a warp each where a row is at most 512 values, otherwise a CTA.  Worker i of n has the
// consecutive rows [i rows / n, (i + 1) rows / n) and holds the weights of the group it is in, so that they are read once
// per worker, not once per row.  It takes R rows at a time, which share each barrier; their values stay in registers from
// there to the store.  The 2R rows after them are on their way into shared memory: each thread copies the values that it
// will itself use (cp.async), so nobody waits for anybody else's copies.  There are as many workers as fit the
// multiprocessors by their registers and their shared memory, so none waits for another to end.
constexpr int kNormThreads = 256;  // of a CTA whose warps are workers
constexpr int kAhead = 3;          // batches of R rows in shared memory: one in use, two on their way

// Who works on a row, by its length: a warp with 8 values a thread (up to 256) or 16 (512), or a CTA with 16 values a
// thread and up to 320 threads (5120), of which a multiprocessor takes two or more, so that one computes while another
// waits at its barrier; beyond that up to 512 threads with 16 values (8192) or 32.
enum Worker { kWarp8, kWarp16, kTeam, kLongTeam, kLongestTeam };
__host__ __device__ constexpr int worker_values(int kind) { return kind == kWarp8 ? 8 : kind == kLongestTeam ? 32 : 16; }
__host__ __device__ constexpr int worker_threads(int kind) { return kind <= kWarp16 ? kNormThreads : kind == kTeam ? 320 : 512; }  // of a CTA, at most
__host__ __device__ constexpr int worker_ctas(int kind) { return kind <= kTeam ? 2 : 1; }  // such CTAs that fit a multiprocessor
__host__ __device__ constexpr int worker_registers(int kind) { return kind == kTeam ? 96 : 128; }
// Rows at a time, by what the registers hold: forward the row and two weights, backward two rows and three weights or
// sums.
__host__ __device__ constexpr int worker_rows(int kind, bool bwd) { return kind == kWarp8 ? (bwd ? 2 : 4) : kind == kLongestTeam || bwd ? 1 : 2; }

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
  int32_t dim, weights_fp32, n_workers, want_weights;
  int32_t ring_bytes;  // of a worker
  float eps, inv_dim;
};

__host__ __device__ inline int64_t first_row(int64_t worker, int64_t n_workers, int64_t rows) {
  return worker * (rows / n_workers) + (worker < rows % n_workers ? worker : rows % n_workers);
}

template <typename T, int E>
__device__ __forceinline__ void load_weights(const void* w, int64_t at, bool fp32, float missing, float (&out)[E]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < E; ++i) out[i] = missing;
  } else if (fp32) {
    const float* p = reinterpret_cast<const float*>(w) + at;
#pragma unroll
    for (int i = 0; i < E; ++i) out[i] = p[i];
  } else {
    const T* p = reinterpret_cast<const T*>(w) + at;
#pragma unroll
    for (int i = 0; i < E; ++i) out[i] = to_float<T>(p[i]);
  }
}

// Sums N values over the worker's threads, in an order that depends on its size alone; every thread gets the sums.
// Inside a warp the values are halved with the lanes (after log2 N exchanges a lane carries one of them), so that N sums
// take little more than one.  A CTA's warps meet in `slot`, which the caller alternates so that one barrier a call is
// enough.
template <int N, bool kCta>
__device__ __forceinline__ void worker_sum(float (&v)[N], float (*slot)[N]) {
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
  for (int o = N; o < 32; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
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
      v[i] = __shfl_sync(0xffffffffu, sum, from);
    }
  }
}

// Two fp32 values in a 64-bit register: one instruction adds or multiplies both.
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit F2(float a) : F2(a, a) {}
  __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
  __device__ __forceinline__ float sum() const {
    float a, b;
    get(a, b);
    return a + b;
  }
};
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// The rows ahead of a worker, of one tensor.  kRing: through shared memory as above; otherwise (single 16-bit values,
// rows too long for shared memory) the next R rows through registers.
template <typename T, int E, int NV, int R, bool kRing>
struct RowsAhead {
  Vec<T, E> next[kRing ? 1 : R][kRing ? 1 : NV];
  const T* from;  // this thread's first value of the next row to be fetched
  int64_t stride;
  char* ring;  // this thread's places, `lanes` vectors from one to the next
  int lanes, t, dim;

  __device__ __forceinline__ void fetch(int n, int batch) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (k >= n) break;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if ((v * lanes + t) * E < dim) {
          const T* at = from + v * lanes * E;
          if constexpr (kRing) {
            char* to = place(batch * R + k, v);
            if constexpr (E * sizeof(T) == 16)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                           "l"(at)
                           : "memory");
            else
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                           "l"(at)
                           : "memory");
          } else {
            next[k][v] = load_once<T, E>(at);
          }
        }
      }
      from += stride;
    }
  }
  // Makes what lies beyond the row zero, once: nothing is ever fetched to there.
  __device__ __forceinline__ void clear_beyond() {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Vec<T, E> zero;
      zero.clear();
      if constexpr (kRing) {
        if ((v * lanes + t) * E >= dim)
          for (int k = 0; k < kAhead * R; ++k) store_vec(reinterpret_cast<T*>(place(k, v)), zero);
      } else {
#pragma unroll
        for (int k = 0; k < R; ++k) next[k][v] = zero;
      }
    }
  }
  // Row k of a batch as pairs, zeros beyond the row.  Where the batch has no row k, of an earlier one, or anything.
  __device__ __forceinline__ void values(F2 (&out)[NV * E / 2], int k, int batch) const {
    float f[NV * E];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Vec<T, E> x;
      if constexpr (kRing)
        x = load_vec<T, E>(reinterpret_cast<const T*>(place(batch * R + k, v)));
      else
        x = next[k][v];
#pragma unroll
      for (int i = 0; i < E; ++i) f[v * E + i] = x[i];
    }
#pragma unroll
    for (int j = 0; j < NV * E / 2; ++j) out[j] = F2(f[2 * j], f[2 * j + 1]);
  }
  __device__ __forceinline__ char* place(int row, int v) const {
    return ring + (row * NV + v) * lanes * (int)(E * sizeof(T));
  }
  // Makes pair j zero where it lies beyond the row.
  __device__ __forceinline__ void inside(F2& x, int j) const {
    if constexpr (E > 1) {
      if ((2 * j / E * lanes + t) * E >= dim) x = F2(0.0f);
    } else {
      float a, b;
      x.get(a, b);
      x = F2(2 * j * lanes + t < dim ? a : 0.0f, (2 * j + 1) * lanes + t < dim ? b : 0.0f);
    }
  }
};
// One group of copies per batch of rows (an empty one past the end); waits for the oldest batch.
__device__ __forceinline__ void close_batch() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_batch() { asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory"); }

// A worker's rows in batches: at most R rows at a time, and none across two groups of weights.
struct Batches {
  int left, in_group, per_group;  // rows yet to be fetched, of them in the group
  __device__ __forceinline__ int size(int R) const { return min(R, min(left, in_group)); }
  __device__ __forceinline__ void take(int n) {
    left -= n;
    in_group -= n;
    if (in_group == 0) in_group = per_group;
  }
};

// A thread's weights of group g; zeros beyond the row.
template <typename T, int E, int NV>
__device__ __forceinline__ void load_pairs(const NormParams& p, const void* from, int64_t g, int lanes, int t,
                                           float missing, F2 (&out)[NV * E / 2]) {
  float f[NV * E];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = (v * lanes + t) * E;
    float part[E];
#pragma unroll
    for (int i = 0; i < E; ++i) part[i] = 0.0f;
    if (e < p.dim) load_weights<T, E>(from, g * p.dim + e, p.weights_fp32, missing, part);
#pragma unroll
    for (int i = 0; i < E; ++i) f[v * E + i] = part[i];
  }
#pragma unroll
  for (int j = 0; j < NV * E / 2; ++j) out[j] = F2(f[2 * j], f[2 * j + 1]);
}

template <typename T, int E, int kKind, bool kRing>
__global__ void __launch_bounds__(worker_threads(kKind), worker_ctas(kKind)) norm_fwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  constexpr int K = worker_values(kKind), NV = K / E, R = worker_rows(kKind, false);
  constexpr bool kCta = kKind >= kTeam;
  extern __shared__ __align__(16) char ring[];
  __shared__ float slots[4][32][R];
  const int lanes = kCta ? blockDim.x : 32;
  const int t = kCta ? threadIdx.x : (threadIdx.x & 31);
  const int64_t worker = kCta ? blockIdx.x : (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
  if (worker >= p.n_workers) return;
  const int64_t r = first_row(worker, p.n_workers, p.rows);
  int todo = (int)(first_row(worker + 1, p.n_workers, p.rows) - r);
  int64_t g = r / p.rows_per_group;
  const int per_group = (int)min(p.rows_per_group, (int64_t)0x7fffffff);
  int here = (int)min((int64_t)todo, (g + 1) * p.rows_per_group - r);  // rows of the group at work
  Batches ahead = {todo, (int)min((g + 1) * p.rows_per_group - r, (int64_t)0x7fffffff), per_group};
  T* out = reinterpret_cast<T*>(p.y) + r * p.stride_y + t * E;
  RowsAhead<T, E, NV, R, kRing> rows;
  rows.from = reinterpret_cast<const T*>(x) + r * p.stride_x + t * E;
  rows.stride = p.stride_x;
  rows.ring = ring + (kCta ? 0 : (threadIdx.x >> 5) * p.ring_bytes) + t * (E * sizeof(T));
  rows.lanes = lanes;
  rows.t = t;
  rows.dim = p.dim;
  rows.clear_beyond();
  // n[0]: rows of the batch at work, n[1], n[2]: of the ones after it
  int n[3];
  n[0] = ahead.size(R);
  rows.fetch(n[0], 0);
  ahead.take(n[0]);
  n[1] = n[2] = 0;
  if constexpr (kRing) {
    close_batch();
    n[1] = ahead.size(R);
    rows.fetch(n[1], 1);
    close_batch();
    ahead.take(n[1]);
  }
  float* mean = p.mean == nullptr ? nullptr : p.mean + r;
  float* rstds = p.rstd + (p.mean == nullptr ? 0 : r);
  int phase = 0, at = 0;
  for (; todo > 0; todo -= here, ++g, here = min(todo, per_group)) {
    F2 w[K / 2], b[K / 2];
    load_pairs<T, E, NV>(p, p.weight, g, lanes, t, 1.0f, w);
    load_pairs<T, E, NV>(p, p.bias, g, lanes, t, 0.0f, b);
#pragma unroll 1
    for (int left = here; left > 0;) {
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
      // the batch after the next: into the places of the one before this, or the registers that were just emptied
      const int more = ahead.size(R);
      rows.fetch(more, at == 0 ? 2 : at - 1);
      if constexpr (kRing) close_batch();
      ahead.take(more);
      worker_sum<R, kCta>(sum, slots[phase]);
      float sq[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        sum[k] *= p.inv_dim;
        const F2 minus(-sum[k]);
        F2 q(0.0f);
#pragma unroll
        for (int j = 0; j < K / 2; ++j) {
          cur[k][j] = cur[k][j] + minus;
          rows.inside(cur[k][j], j);  // what lies beyond the row is no deviation
          q = fma(cur[k][j], cur[k][j], q);
        }
        sq[k] = q.sum();
      }
      worker_sum<R, kCta>(sq, slots[phase + 1]);
      phase ^= 2;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k >= n[0]) continue;
        const float rstd = rsqrtf(sq[k] * p.inv_dim + p.eps);
        const F2 scale(rstd);
        float y[K];
#pragma unroll
        for (int j = 0; j < K / 2; ++j) fma(cur[k][j] * scale, w[j], b[j]).get(y[2 * j], y[2 * j + 1]);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          if ((v * lanes + t) * E < p.dim) {
            Vec<T, E> o;
            o.set(y + v * E);
            store_vec(out + v * lanes * E, o);
          }
        }
        out += p.stride_y;
        if (mean != nullptr && t == 0) {
          mean[k] = sum[k];
          rstds[k] = rstd;
        }
      }
      if (mean != nullptr) {
        mean += n[0];
        rstds += n[0];
      }
      left -= n[0];
      if constexpr (kRing) {
        n[0] = n[1];
        n[1] = more;
        at = at == 2 ? 0 : at + 1;
      } else {
        n[0] = more;
      }
    }
  }
}

// The gradients of the weights are sums over rows: each worker keeps those of its rows in registers and writes them out
// when its group or its rows end, into slot worker + group, which no other (worker, group) has, as rows and with them
// groups ascend from worker to worker.  norm_weights_kernel adds a group's slots.
template <typename T, int E, int kKind, bool kRing>
__global__ void __launch_bounds__(worker_threads(kKind), worker_ctas(kKind)) norm_bwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  constexpr int K = worker_values(kKind), NV = K / E, R = worker_rows(kKind, true);
  constexpr bool kCta = kKind >= kTeam;
  extern __shared__ __align__(16) char ring[];
  __shared__ float slots[2][32][2 * R];
  const int lanes = kCta ? blockDim.x : 32;
  const int t = kCta ? threadIdx.x : (threadIdx.x & 31);
  const int64_t worker = kCta ? blockIdx.x : (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
  if (worker >= p.n_workers) return;
  const int64_t r = first_row(worker, p.n_workers, p.rows);
  int todo = (int)(first_row(worker + 1, p.n_workers, p.rows) - r);
  int64_t g = r / p.rows_per_group;
  const int per_group = (int)min(p.rows_per_group, (int64_t)0x7fffffff);
  int here = (int)min((int64_t)todo, (g + 1) * p.rows_per_group - r);  // rows of the group at work
  Batches ahead = {todo, (int)min((g + 1) * p.rows_per_group - r, (int64_t)0x7fffffff), per_group};
  T* out = reinterpret_cast<T*>(p.y) + r * p.stride_x + t * E;
  RowsAhead<T, E, NV, R, kRing> xs, ys;
  xs.from = reinterpret_cast<const T*>(x) + r * p.stride_x + t * E;
  ys.from = reinterpret_cast<const T*>(p.dy) + r * p.stride_y + t * E;
  xs.stride = p.stride_x;
  ys.stride = p.stride_y;
  xs.ring = ring + (kCta ? 0 : (threadIdx.x >> 5) * p.ring_bytes) + t * (E * sizeof(T));
  ys.ring = xs.ring + p.ring_bytes / 2;
  xs.lanes = ys.lanes = lanes;
  xs.t = ys.t = t;
  xs.dim = ys.dim = p.dim;
  xs.clear_beyond();
  ys.clear_beyond();
  float mean[R], rstd[R];  // of the next batch
  const float* means = p.mean_in + r;
  const float* rstds = p.rstd_in + r;
  auto stats = [&](int n) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = k < n ? means[k] : 0.0f;
      rstd[k] = k < n ? rstds[k] : 0.0f;
    }
    means += n;
    rstds += n;
  };
  int n[3];
  n[0] = ahead.size(R);
  xs.fetch(n[0], 0);
  ys.fetch(n[0], 0);
  stats(n[0]);
  ahead.take(n[0]);
  n[1] = n[2] = 0;
  if constexpr (kRing) {
    close_batch();
    n[1] = ahead.size(R);
    xs.fetch(n[1], 1);
    ys.fetch(n[1], 1);
    close_batch();
    ahead.take(n[1]);
  }
  int phase = 0, at = 0;
  for (; todo > 0; todo -= here, ++g, here = min(todo, per_group)) {
    F2 w[K / 2], dw[K / 2], db[K / 2];
    load_pairs<T, E, NV>(p, p.weight, g, lanes, t, 1.0f, w);
#pragma unroll
    for (int j = 0; j < K / 2; ++j) dw[j] = db[j] = F2(0.0f);
#pragma unroll 1
    for (int left = here; left > 0;) {
      if constexpr (kRing) wait_batch();
      F2 xh[R][K / 2], a[R][K / 2], scale[R];
      float sum[2 * R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        scale[k] = F2(rstd[k]);
        const F2 shift(-mean[k]);
        // beyond the row there is no gradient: dy is 0 there
        xs.values(xh[k], k, at);
        ys.values(a[k], k, at);
        sum[2 * k] = sum[2 * k + 1] = 0.0f;
        if (R > 1 && k >= n[0]) continue;
        F2 s0(0.0f), s1(0.0f);
#pragma unroll
        for (int j = 0; j < K / 2; ++j) {
          const F2 dy = a[k][j];
          xh[k][j] = (xh[k][j] + shift) * scale[k];
          a[k][j] = dy * w[j];
          s0 = s0 + a[k][j];
          s1 = fma(a[k][j], xh[k][j], s1);
          dw[j] = fma(dy, xh[k][j], dw[j]);
          db[j] = db[j] + dy;
        }
        sum[2 * k] = s0.sum();
        sum[2 * k + 1] = s1.sum();
      }
      const int more = ahead.size(R);
      xs.fetch(more, at == 0 ? 2 : at - 1);
      ys.fetch(more, at == 0 ? 2 : at - 1);
      if constexpr (kRing) close_batch();
      ahead.take(more);
      stats(kRing ? n[1] : more);
      worker_sum<2 * R, kCta>(sum, slots[phase]);
      phase ^= 1;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (k >= n[0]) continue;
        const F2 c0(-sum[2 * k] * p.inv_dim), c1(-sum[2 * k + 1] * p.inv_dim);
        float dx[K];
#pragma unroll
        for (int j = 0; j < K / 2; ++j) (scale[k] * fma(xh[k][j], c1, a[k][j] + c0)).get(dx[2 * j], dx[2 * j + 1]);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          if ((v * lanes + t) * E < p.dim) {
            Vec<T, E> o;
            o.set(dx + v * E);
            store_vec(out + v * lanes * E, o);
          }
        }
        out += p.stride_x;
      }
      left -= n[0];
      if constexpr (kRing) {
        n[0] = n[1];
        n[1] = more;
        at = at == 2 ? 0 : at + 1;
      } else {
        n[0] = more;
      }
    }
    if (p.want_weights) {
      float* mine = p.partial + (worker + g) * 2 * p.dim;
#pragma unroll
      for (int j = 0; j < K; j += 2) {
        float a[2], c[2];
        dw[j / 2].get(a[0], a[1]);
        db[j / 2].get(c[0], c[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int e = ((j + i) / E * lanes + t) * E;
          if (e < p.dim) {
            mine[e + (j + i) % E] = a[i];
            mine[p.dim + e + (j + i) % E] = c[i];
          }
        }
      }
    }
  }
}

// Adds the slots of each group.  A CTA has 32 columns of one group; its 8 warps take every 8th slot each and meet in
// shared memory, so the order is the same whatever runs when.
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* partial, int64_t rows, int64_t rows_per_group,
                                                           int64_t n_workers, int dim, void* dweight, void* dbias,
                                                           int dtype) {
  enter_grid(partial);
  __shared__ float s[2][8][32];
  const int tiles = (dim + 31) / 32;
  const int64_t g = blockIdx.x / tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (blockIdx.x % tiles) * 32 + lane;
  float sw = 0.0f, sb = 0.0f;
  if (rows > 0) {
    // workers with rows of this group: from the one that has the group's first row to the one that has its last
    const int64_t lo = g * rows_per_group, hi = min(lo + rows_per_group, rows) - 1;
    const int64_t q = rows / n_workers, m = rows % n_workers;
    const int64_t cut = m * (q + 1);  // rows of the workers that have one more
    const int64_t w0 = lo < cut ? lo / (q + 1) : m + (lo - cut) / q;
    const int64_t w1 = hi < cut ? hi / (q + 1) : m + (hi - cut) / q;
    if (col < dim)
      for (int64_t w = w0 + warp; w <= w1; w += 8) {
        const float* slot = partial + (w + g) * 2 * dim + col;
        sw += slot[0];
        sb += slot[dim];
      }
  }
  s[0][warp][lane] = sw;
  s[1][warp][lane] = sb;
  __syncthreads();
  if (warp < 2 && col < dim) {
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += s[warp][k][lane];
    void* to = warp == 0 ? dweight : dbias;
    if (to != nullptr) {
      const int64_t at = g * dim + col;
      if (dtype == SPARSP_FP32)
        reinterpret_cast<float*>(to)[at] = v;
      else if (dtype == SPARSP_FP16)
        reinterpret_cast<__half*>(to)[at] = __float2half_rn(v);
      else
        reinterpret_cast<__nv_bfloat16*>(to)[at] = __float2bfloat16_rn(v);
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------

int64_t norm_groups(const sparsp_norm& n) {
  return n.rows_per_group == 0 ? 1 : (n.rows + n.rows_per_group - 1) / n.rows_per_group;
}

// How the rows are shared out.
struct NormPlan {
  bool vectors, ring;
  int kind, threads;           // of a CTA
  int ring_bytes, smem_bytes;  // of a worker, of a CTA
  int64_t n_workers;
  unsigned grid;
};

constexpr int kNormSmem = 224 * 1024;  // of a multiprocessor, for rings

static NormPlan plan_norm(const sparsp_norm& n, bool vectors, bool bwd) {
  NormPlan p;
  p.vectors = vectors;
  const int bytes = element_bytes(n.dtype), E = vectors ? 16 / bytes : 1;
  p.kind = n.dim <= 256 ? kWarp8 : n.dim <= 512 ? kWarp16 : n.dim <= 5120 ? kTeam : n.dim <= 8192 ? kLongTeam : kLongestTeam;
  const bool cta = p.kind >= kTeam;
  p.threads = kNormThreads;
  if (cta) {
    const int units = (n.dim + E - 1) / E, per_thread = worker_values(p.kind) / E;
    p.threads = ((units + per_thread - 1) / per_thread + 31) / 32 * 32;
  }
  int resident = std::min(32, 65536 / (p.threads * worker_registers(p.kind)));
  const int workers = cta ? 1 : kNormThreads / 32;  // of a CTA
  const int lanes = cta ? p.threads : 32;
  p.ring_bytes = kAhead * worker_rows(p.kind, bwd) * lanes * worker_values(p.kind) * bytes * (bwd ? 2 : 1);
  p.ring = E * bytes >= 4 && p.ring_bytes * workers <= kNormSmem - 4096;
  p.smem_bytes = p.ring ? p.ring_bytes * workers : 0;
  if (p.ring) resident = std::min(resident, kNormSmem / (p.smem_bytes + 4096));
  p.n_workers = std::min<int64_t>(n.rows, (int64_t)kSms * resident * workers);
  p.grid = (unsigned)((p.n_workers + workers - 1) / workers);
  return p;
}

int64_t norm_workspace_bytes(const sparsp_norm& n) {
  const int64_t workers = std::max(plan_norm(n, true, true).n_workers, plan_norm(n, false, true).n_workers);
  return kStatusWords * 4 + (workers + norm_groups(n)) * 2 * n.dim * 4;
}

static bool norm_vectors(const sparsp_norm& n, const void* a, const void* b, const void* c) {
  const int E = 16 / element_bytes(n.dtype);
  return n.dim % E == 0 && (n.rows <= 1 || (n.stride_x % E == 0 && n.stride_y % E == 0)) && (uintptr_t)a % 16 == 0 &&
         (uintptr_t)b % 16 == 0 && (uintptr_t)c % 16 == 0;
}

template <typename T, int E, int kKind, bool kRing>
static cudaError_t launch_norm_r(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  auto kern = bwd ? norm_bwd_kernel<T, E, kKind, kRing> : norm_fwd_kernel<T, E, kKind, kRing>;
  if (kRing) {
    const cudaError_t e = ensure_dynamic_smem((const void*)kern, plan.smem_bytes);
    if (e != cudaSuccess) return e;
  }
  return launch_kernel(kern, dim3(plan.grid), plan.threads, plan.smem_bytes, st, p);
}

// Without a ring: single 16-bit values, and rows that are too long for shared memory.
template <typename T, int E, int kKind>
static cudaError_t launch_norm_t(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  if constexpr (E * sizeof(T) < 4)
    return launch_norm_r<T, E, kKind, false>(p, plan, bwd, st);
  else if constexpr (kKind == kLongestTeam)
    return plan.ring ? launch_norm_r<T, E, kKind, true>(p, plan, bwd, st)
                     : launch_norm_r<T, E, kKind, false>(p, plan, bwd, st);
  else
    return launch_norm_r<T, E, kKind, true>(p, plan, bwd, st);
}

template <typename T, int E>
static cudaError_t launch_norm_e(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  switch (plan.kind) {
    case kWarp8: return launch_norm_t<T, E, kWarp8>(p, plan, bwd, st);
    case kWarp16: return launch_norm_t<T, E, kWarp16>(p, plan, bwd, st);
    case kTeam: return launch_norm_t<T, E, kTeam>(p, plan, bwd, st);
    case kLongTeam: return launch_norm_t<T, E, kLongTeam>(p, plan, bwd, st);
    default: return launch_norm_t<T, E, kLongestTeam>(p, plan, bwd, st);
  }
}

static cudaError_t launch_norm(int dtype, const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  SPARSP_WITH_TYPE(dtype, T, {
    e = plan.vectors ? launch_norm_e<T, 16 / sizeof(T)>(p, plan, bwd, st) : launch_norm_e<T, 1>(p, plan, bwd, st);
  });
  return e;
}

static NormParams norm_params(const sparsp_norm& n, const NormPlan& plan) {
  NormParams p = {};
  p.rows = n.rows;
  p.rows_per_group = n.rows_per_group == 0 ? std::max<int64_t>(n.rows, 1) : n.rows_per_group;
  p.stride_x = n.stride_x;
  p.stride_y = n.stride_y;
  p.dim = n.dim;
  p.weights_fp32 = n.weight_dtype == SPARSP_FP32;
  p.n_workers = (int32_t)plan.n_workers;
  p.ring_bytes = plan.ring_bytes;
  p.eps = n.eps;
  p.inv_dim = 1.0f / (float)n.dim;
  return p;
}

int launch_norm_fwd(const sparsp_norm& n, const void* X, const void* w, const void* b, void* Y, float* mean,
                    float* rstd, cudaStream_t st) {
  if (n.rows == 0) return SPARSP_OK;
  const NormPlan plan = plan_norm(n, norm_vectors(n, X, Y, nullptr), false);
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
  const NormPlan plan = plan_norm(n, norm_vectors(n, X, dY, dX), true);
  NormParams p = norm_params(n, plan);
  p.want_weights = dw != nullptr || db != nullptr;
  if (n.rows > 0) {
    p.x = X;
    p.dy = dY;
    p.weight = w;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.y = dX;
    p.partial = reinterpret_cast<float*>(ws + kStatusWords * 4);
    SPARSP_CUDA_OK(launch_norm(n.dtype, p, plan, true, st));
  }
  if (p.want_weights && norm_groups(n) > 0) {
    const unsigned grid = (unsigned)(norm_groups(n) * ((n.dim + 31) / 32));
    SPARSP_CUDA_OK(launch_kernel(norm_weights_kernel, dim3(grid), 256, 0, st, p.partial, n.rows, p.rows_per_group,
                                 std::max<int64_t>(plan.n_workers, 1), n.dim, dw, db, n.weight_dtype));
  }
  return SPARSP_OK;
}

}  // namespace sparsp
