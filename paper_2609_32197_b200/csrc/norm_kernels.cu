// Layer norm: forward, and backward with the reduction of the weights' gradients.
#include <algorithm>

#include "layer.cuh"

namespace sparsp {

// Rows are worked on by "workers": a warp each where a row is at most 512 values, otherwise a CTA.  Worker i of n has the
// consecutive rows [i rows / n, (i + 1) rows / n) and holds the weights of the group it is in, so that they are read once
// per worker, not once per row.  It takes R rows at a time: their values stay in registers from their load to the store,
// the loads of the next R are in flight meanwhile, and the R rows share each barrier.  There are as many workers as fit
// the multiprocessors by their registers, so none waits for another to end.
constexpr int kNormThreads = 256;  // of a CTA whose warps are workers

// By values a thread: most threads of a CTA, and with them the registers that each may have.
constexpr int norm_threads(int values) { return values <= 8 ? 640 : 512; }
constexpr int norm_registers(int values) { return values <= 8 ? 96 : 128; }

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

template <typename T, int E, int NV, int R, bool kCta>
__global__ void __launch_bounds__(kCta ? norm_threads(NV * E) : kNormThreads, kCta ? 1 : 2) norm_fwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  __shared__ float slots[4][32][R];
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
  Vec<T, E> cur[R][NV], next[R][NV];
  int64_t g = r / p.rows_per_group, group_end = r;
  int n_next = (int)min((int64_t)R, min(r1, (g + 1) * p.rows_per_group) - r), phase = 0;
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      if (k < n_next && e < p.dim) next[k][v] = load_once<T, E>(in + (r + k) * p.stride_x + e);
    }
  while (r < r1) {
    if (r >= group_end) {
      g = r / p.rows_per_group;
      group_end = min(r1, (g + 1) * p.rows_per_group);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) {
          load_weights<T, E>(p.weight, g * p.dim + e, p.weights_fp32, 1.0f, w[v]);
          load_weights<T, E>(p.bias, g * p.dim + e, p.weights_fp32, 0.0f, b[v]);
        }
      }
    }
    const int n = n_next;
    const int64_t after = r + n;
    n_next = after < r1 ? (int)min((int64_t)R, (after < group_end ? group_end : min(r1, after + p.rows_per_group)) - after) : 0;
    float sum[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sum[k] = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        cur[k][v] = next[k][v];
        if (e < p.dim) {
          if (k < n_next) next[k][v] = load_once<T, E>(in + (after + k) * p.stride_x + e);
          if (k < n) {
#pragma unroll
            for (int i = 0; i < E; ++i) sum[k] += cur[k][v][i];
          }
        }
      }
    }
    worker_sum<R, kCta>(sum, slots[phase]);
    float sq[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sum[k] *= p.inv_dim;
      sq[k] = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (k < n && e < p.dim) {
#pragma unroll
          for (int i = 0; i < E; ++i) {
            const float d = cur[k][v][i] - sum[k];
            sq[k] = fmaf(d, d, sq[k]);
          }
        }
      }
    }
    worker_sum<R, kCta>(sq, slots[phase + 1]);
    phase ^= 2;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (k >= n) continue;
      const float rstd = 1.0f / sqrtf(sq[k] * p.inv_dim + p.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) {
          float y[E];
#pragma unroll
          for (int i = 0; i < E; ++i) y[i] = fmaf((cur[k][v][i] - sum[k]) * rstd, w[v][i], b[v][i]);
          Vec<T, E> o;
          o.set(y);
          store_vec<T, E>(out + (r + k) * p.stride_y + e, o);
        }
      }
      if (p.mean != nullptr && t == 0) {
        p.mean[r + k] = sum[k];
        p.rstd[r + k] = rstd;
      }
    }
    r = after;
  }
}

// The gradients of the weights are sums over rows: each worker keeps those of its rows in registers and writes them out
// when its group or its rows end, into slot worker + group, which no other (worker, group) has, as rows and with them
// groups ascend from worker to worker.  norm_weights_kernel adds a group's slots.
template <typename T, int E, int NV, int R, bool kCta>
__global__ void __launch_bounds__(kCta ? norm_threads(NV * E) : kNormThreads, kCta ? 1 : 2) norm_bwd_kernel(const NormParams p) {
  const void* x = p.x;
  enter_grid(x);
  __shared__ float slots[2][32][2 * R];
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
  Vec<T, E> cx[R][NV], cy[R][NV], next_x[R][NV], next_y[R][NV];
  float next_mean[R], next_rstd[R];
  int64_t g = r / p.rows_per_group, group_end = r;
  int n_next = (int)min((int64_t)R, min(r1, (g + 1) * p.rows_per_group) - r), phase = 0;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    next_mean[k] = next_rstd[k] = 0.0f;
    if (k < n_next) {
      next_mean[k] = p.mean_in[r + k];
      next_rstd[k] = p.rstd_in[r + k];
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = (v * lanes + t) * E;
      if (k < n_next && e < p.dim) {
        next_x[k][v] = load_once<T, E>(in + (r + k) * p.stride_x + e);
        next_y[k][v] = load_once<T, E>(grad + (r + k) * p.stride_y + e);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < E; ++i) dw[v][i] = db[v][i] = 0.0f;
  while (r < r1) {
    if (r >= group_end) {
      g = r / p.rows_per_group;
      group_end = min(r1, (g + 1) * p.rows_per_group);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) load_weights<T, E>(p.weight, g * p.dim + e, p.weights_fp32, 1.0f, w[v]);
      }
    }
    const int n = n_next;
    const int64_t after = r + n;
    n_next = after < r1 ? (int)min((int64_t)R, (after < group_end ? group_end : min(r1, after + p.rows_per_group)) - after) : 0;
    float sum[2 * R], mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = next_mean[k];
      rstd[k] = next_rstd[k];
      if (k < n_next) {
        next_mean[k] = p.mean_in[after + k];
        next_rstd[k] = p.rstd_in[after + k];
      }
      sum[2 * k] = sum[2 * k + 1] = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        cx[k][v] = next_x[k][v];
        cy[k][v] = next_y[k][v];
        if (e < p.dim) {
          if (k < n_next) {
            next_x[k][v] = load_once<T, E>(in + (after + k) * p.stride_x + e);
            next_y[k][v] = load_once<T, E>(grad + (after + k) * p.stride_y + e);
          }
          if (k < n) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
              const float xh = (cx[k][v][i] - mean[k]) * rstd[k], dy = cy[k][v][i], a = dy * w[v][i];
              sum[2 * k] += a;
              sum[2 * k + 1] = fmaf(a, xh, sum[2 * k + 1]);
              dw[v][i] = fmaf(dy, xh, dw[v][i]);
              db[v][i] += dy;
            }
          }
        }
      }
    }
    worker_sum<2 * R, kCta>(sum, slots[phase]);
    phase ^= 1;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (k >= n) continue;
      const float c0 = sum[2 * k] * p.inv_dim, c1 = sum[2 * k + 1] * p.inv_dim;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * lanes + t) * E;
        if (e < p.dim) {
          float dx[E];
#pragma unroll
          for (int i = 0; i < E; ++i) {
            const float xh = (cx[k][v][i] - mean[k]) * rstd[k];
            dx[i] = rstd[k] * (cy[k][v][i] * w[v][i] - c0 - xh * c1);
          }
          Vec<T, E> o;
          o.set(dx);
          store_vec<T, E>(out + (r + k) * p.stride_x + e, o);
        }
      }
    }
    r = after;
    if (p.want_weights && r == group_end) {
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

// How a row is shared out: by values a thread.
struct NormPlan {
  bool vectors, cta;
  int values, threads;  // of a thread, of a CTA
  int64_t n_workers;
  unsigned grid;
};

static NormPlan plan_norm(const sparsp_norm& n, bool vectors) {
  NormPlan p;
  p.vectors = vectors;
  p.cta = n.dim > 512;
  if (!p.cta) {
    p.values = n.dim <= 256 ? 8 : 16;
    p.threads = kNormThreads;
    p.n_workers = std::min<int64_t>(n.rows, (int64_t)kSms * 2 * (kNormThreads / 32));
    p.grid = (unsigned)((p.n_workers + kNormThreads / 32 - 1) / (kNormThreads / 32));
  } else {
    p.values = 8;
    while (p.values * norm_threads(p.values) < n.dim) p.values *= 2;
    const int E = vectors ? 16 / element_bytes(n.dtype) : 1, per_thread = p.values / E;
    const int units = (n.dim + E - 1) / E;
    p.threads = ((units + per_thread - 1) / per_thread + 31) / 32 * 32;
    const int resident = std::max(1, 65536 / (p.threads * norm_registers(p.values)));
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

// Values a thread, and rows at a time by what its registers hold: forward two vectors a row, backward four and three
// accumulators.
template <typename T, int E, int kValues, bool kCta>
static cudaError_t launch_norm_t(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  constexpr int kFwdRows = kValues <= 8 ? 4 : kValues <= 16 ? 2 : 1, kBwdRows = kValues <= 8 ? 2 : 1;
  return launch_kernel(bwd ? norm_bwd_kernel<T, E, kValues / E, kBwdRows, kCta>
                           : norm_fwd_kernel<T, E, kValues / E, kFwdRows, kCta>,
                       dim3(plan.grid), plan.threads, 0, st, p);
}

template <typename T, int E>
static cudaError_t launch_norm_e(const NormParams& p, const NormPlan& plan, bool bwd, cudaStream_t st) {
  if (!plan.cta)
    return plan.values == 8 ? launch_norm_t<T, E, 8, false>(p, plan, bwd, st)
                            : launch_norm_t<T, E, 16, false>(p, plan, bwd, st);
  return plan.values == 8    ? launch_norm_t<T, E, 8, true>(p, plan, bwd, st)
         : plan.values == 16 ? launch_norm_t<T, E, 16, true>(p, plan, bwd, st)
                             : launch_norm_t<T, E, 32, true>(p, plan, bwd, st);
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
