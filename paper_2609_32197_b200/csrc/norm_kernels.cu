// Layer norm: forward, and backward with the reduction of the weights' gradients.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

// Rows are worked on by "workers": a warp each where a row fits its registers, otherwise a CTA.  Worker i of n has the
// consecutive rows [i rows / n, (i + 1) rows / n) and holds the weights of the group it is in, so that they are read once
// per worker, not once per row; the values of a row stay in registers from their load to the store, with the next row's
// loads in flight meanwhile.
constexpr int kNormThreads = 256;  // of a CTA whose warps are workers
constexpr int kNormCta = 512;      // most threads of a CTA that is a worker: 128 registers each

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

// Sums over the worker's threads, in an order that depends on its size alone; every thread gets the sums.  A CTA's
// warps meet in `slot`, which the caller alternates so that one barrier a call is enough.
template <int N, bool kCta>
__device__ __forceinline__ void worker_sum(float (&v)[N], float (*slot)[N]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if constexpr (kCta) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slot[warp][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane < warps ? slot[lane][k] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
}

template <typename T, int E, int NV, bool kCta>
__global__ void __launch_bounds__(kCta ? kNormCta : kNormThreads) norm_fwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  __shared__ float slots[4][32][1];
  const int lanes = kCta ? blockDim.x : 32;
  const int t = kCta ? threadIdx.x : (threadIdx.x & 31);
  const int64_t worker = kCta ? blockIdx.x : (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
  if (worker >= p.n_workers) return;
  const int64_t r1 = first_row(worker + 1, p.n_workers, p.rows);
  int64_t r = first_row(worker, p.n_workers, p.rows);
  if (r >= r1) return;
  const T* in = reinterpret_cast<const T*>(x);
  T* out = reinterpret_cast<T*>(p.y);
  float w[NV][E], b[NV][E];
  Vec<T, E> next[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = (v * lanes + t) * E;
    if (e < p.dim) next[v] = load_once<T, E>(in + r * p.stride_x + e);
  }
  int64_t group_end = r;
  int phase = 0;
  for (; r < r1; ++r) {
    if (r >= group_end) {
      const int64_t g = r / p.rows_per_group;
      group_end = (g + 1) * p.rows_per_group;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) {
          load_weights<T, E>(p.weight, g * p.dim + e, p.weights_fp32, 1.0f, w[v]);
          load_weights<T, E>(p.bias, g * p.dim + e, p.weights_fp32, 0.0f, b[v]);
        }
      }
    }
    Vec<T, E> cur[NV];
    float sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      cur[v] = next[v];
      if (e < p.dim) {
        if (r + 1 < r1) next[v] = load_once<T, E>(in + (r + 1) * p.stride_x + e);
#pragma unroll
        for (int i = 0; i < E; ++i) sum[0] += cur[v][i];
      }
    }
    worker_sum<1, kCta>(sum, slots[phase]);
    const float mean = sum[0] * p.inv_dim;
    float sq[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      if (e < p.dim) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float d = cur[v][i] - mean;
          sq[0] = fmaf(d, d, sq[0]);
        }
      }
    }
    worker_sum<1, kCta>(sq, slots[phase + 1]);
    phase ^= 2;
    const float rstd = 1.0f / sqrtf(sq[0] * p.inv_dim + p.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      if (e < p.dim) {
        Vec<T, E> o;
#pragma unroll
        for (int i = 0; i < E; ++i) o.set(i, fmaf((cur[v][i] - mean) * rstd, w[v][i], b[v][i]));
        store_vec<T, E>(out + r * p.stride_y + e, o);
      }
    }
    if (p.mean != nullptr && t == 0) {
      p.mean[r] = mean;
      p.rstd[r] = rstd;
    }
  }
}

// The gradients of the weights are sums over rows: each worker keeps those of its rows in registers and writes them out
// when its group or its rows end, into slot worker + group, which no other (worker, group) has, as rows and with them
// groups ascend from worker to worker.  norm_weights_kernel adds a group's slots.
template <typename T, int E, int NV, bool kCta>
__global__ void __launch_bounds__(kCta ? kNormCta : kNormThreads) norm_bwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  __shared__ float slots[2][32][2];
  const int lanes = kCta ? blockDim.x : 32;
  const int t = kCta ? threadIdx.x : (threadIdx.x & 31);
  const int64_t worker = kCta ? blockIdx.x : (int64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
  if (worker >= p.n_workers) return;
  const int64_t r1 = first_row(worker + 1, p.n_workers, p.rows);
  int64_t r = first_row(worker, p.n_workers, p.rows);
  if (r >= r1) return;
  const T* in = reinterpret_cast<const T*>(x);
  const T* grad = reinterpret_cast<const T*>(p.dy);
  T* out = reinterpret_cast<T*>(p.y);
  float w[NV][E], dw[NV][E], db[NV][E];
  Vec<T, E> next_x[NV], next_dy[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = (v * lanes + t) * E;
    if (e < p.dim) {
      next_x[v] = load_once<T, E>(in + r * p.stride_x + e);
      next_dy[v] = load_once<T, E>(grad + r * p.stride_y + e);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) dw[v][i] = db[v][i] = 0.0f;
  }
  int64_t g = r / p.rows_per_group, group_end = r;
  int phase = 0;
  for (; r < r1; ++r) {
    if (r >= group_end) {
      g = r / p.rows_per_group;
      group_end = (g + 1) * p.rows_per_group;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) load_weights<T, E>(p.weight, g * p.dim + e, p.weights_fp32, 1.0f, w[v]);
      }
    }
    const float mean = p.mean_in[r], rstd = p.rstd_in[r];
    Vec<T, E> cx[NV], cy[NV];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      cx[v] = next_x[v];
      cy[v] = next_dy[v];
      if (e < p.dim) {
        if (r + 1 < r1) {
          next_x[v] = load_once<T, E>(in + (r + 1) * p.stride_x + e);
          next_dy[v] = load_once<T, E>(grad + (r + 1) * p.stride_y + e);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float xh = (cx[v][i] - mean) * rstd, dy = cy[v][i], a = dy * w[v][i];
          sum[0] += a;
          sum[1] = fmaf(a, xh, sum[1]);
          dw[v][i] = fmaf(dy, xh, dw[v][i]);
          db[v][i] += dy;
        }
      }
    }
    worker_sum<2, kCta>(sum, slots[phase]);
    phase ^= 1;
    const float c0 = sum[0] * p.inv_dim, c1 = sum[1] * p.inv_dim;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      if (e < p.dim) {
        Vec<T, E> o;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float xh = (cx[v][i] - mean) * rstd;
          o.set(i, rstd * (cy[v][i] * w[v][i] - c0 - xh * c1));
        }
        store_vec<T, E>(out + r * p.stride_x + e, o);
      }
    }
    if (p.want_weights && (r + 1 == r1 || r + 1 == group_end)) {
      float* mine = p.partial + (worker + g) * 2 * p.dim;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) {
#pragma unroll
          for (int i = 0; i < E; ++i) {
            mine[e + i] = dw[v][i];
            mine[p.dim + e + i] = db[v][i];
            dw[v][i] = db[v][i] = 0.0f;
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

// How a row is shared out: by elements and vectors a thread.
struct NormPlan {
  bool vectors, cta;
  int per_thread, threads;  // vectors (or elements) a thread, threads of a CTA
  int64_t n_workers;
  unsigned grid;
};

static NormPlan plan_norm(const sparsp_norm& n, bool vectors) {
  NormPlan p;
  p.vectors = vectors;
  const int E = vectors ? 16 / element_bytes(n.dtype) : 1;
  const int units = (n.dim + E - 1) / E;  // vectors of a row
  const int most = vectors ? 2 : 16;      // a warp's vectors a thread
  p.cta = units > 32 * most;
  if (!p.cta) {
    p.per_thread = vectors ? (units <= 32 ? 1 : 2) : (units <= 128 ? 4 : 16);
    p.threads = kNormThreads;
    p.n_workers = std::min<int64_t>(n.rows, (int64_t)kSms * 4 * (kNormThreads / 32));
    p.grid = (unsigned)((p.n_workers + kNormThreads / 32 - 1) / (kNormThreads / 32));
  } else {
    p.per_thread = vectors ? 2 : 4;
    while (p.per_thread * kNormCta < units) p.per_thread *= 2;
    if (!vectors && p.per_thread == 8) p.per_thread = 16;
    p.threads = ((units + p.per_thread - 1) / p.per_thread + 31) / 32 * 32;
    const int resident = std::max(1, 1024 / p.threads);
    p.n_workers = std::min<int64_t>(n.rows, (int64_t)kSms * resident);
    p.grid = (unsigned)p.n_workers;
  }
  return p;
}

int64_t norm_workspace_bytes(const sparsp_norm& n) {
  const int64_t workers = std::max(plan_norm(n, true).n_workers, plan_norm(n, false).n_workers);
  return kStatusWords * 4 + (workers + norm_groups(n)) * 2 * n.dim * 4;
}

static bool norm_vectors(const sparsp_norm& n, const void* a, const void* b, const void* c) {
  const int E = 16 / element_bytes(n.dtype);
  return n.dim % E == 0 && (n.rows <= 1 || (n.stride_x % E == 0 && n.stride_y % E == 0)) && (uintptr_t)a % 16 == 0 &&
         (uintptr_t)b % 16 == 0 && (uintptr_t)c % 16 == 0;
}

template <typename T, int E, int NV, bool kCta>
static cudaError_t launch_norm_t(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  return launch_kernel(bwd ? norm_bwd_kernel<T, E, NV, kCta> : norm_fwd_kernel<T, E, NV, kCta>, dim3(plan.grid),
                       plan.threads, 0, st, p);
}

static cudaError_t launch_norm(int dtype, const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  SPARSP_WITH_TYPE(dtype, T, {
    constexpr int E = 16 / sizeof(T);
    if (plan.vectors && !plan.cta)
      e = plan.per_thread == 1 ? launch_norm_t<T, E, 1, false>(p, plan, bwd, st)
                               : launch_norm_t<T, E, 2, false>(p, plan, bwd, st);
    else if (plan.vectors)
      e = plan.per_thread == 2   ? launch_norm_t<T, E, 2, true>(p, plan, bwd, st)
          : plan.per_thread == 4 ? launch_norm_t<T, E, 4, true>(p, plan, bwd, st)
                                 : launch_norm_t<T, E, 32 / E, true>(p, plan, bwd, st);
    else if (!plan.cta)
      e = plan.per_thread == 4 ? launch_norm_t<T, 1, 4, false>(p, plan, bwd, st)
                               : launch_norm_t<T, 1, 16, false>(p, plan, bwd, st);
    else
      e = plan.per_thread == 4    ? launch_norm_t<T, 1, 4, true>(p, plan, bwd, st)
          : plan.per_thread == 16 ? launch_norm_t<T, 1, 16, true>(p, plan, bwd, st)
                                  : launch_norm_t<T, 1, 32, true>(p, plan, bwd, st);
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
  p.eps = n.eps;
  p.inv_dim = 1.0f / (float)n.dim;
  return p;
}

int launch_norm_fwd(const sparsp_norm& n, const void* X, const void* w, const void* b, void* Y, float* mean,
                    float* rstd, cudaStream_t st) {
  if (n.rows == 0) return SPARSP_OK;
  const NormPlan plan = plan_norm(n, norm_vectors(n, X, Y, nullptr));
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
  const NormPlan plan = plan_norm(n, norm_vectors(n, X, dY, dX));
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
