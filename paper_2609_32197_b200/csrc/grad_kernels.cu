// The norm over a list of gradients, and their clipping.
//
// A table in device memory, made once for a list, says where its tensors are; nothing of it goes through a call, so that
// calls cost the host the same for one tensor and for thousands (as kernel parameters, 12 KB for 300 tensors, they cost
// 10 us each; making it costs 180 us for 300 tensors in Python, most of it questions to each).  Tensors are cut into
// chunks of 16 KB; a CTA has a run of them and is told which tensor that begins in.  Squares are added in fp32 over the 32
// values at most that a thread has of a chunk, then in fp64, and CTAs' sums in their order by the one that ends last: the
// same list gives the same bits.  Scaling goes through each run from its end, so that what the first pass read last is
// still in L2.
//
// Bound by HBM: every value is read once for the norm, and read again and written where the norm is over the limit.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "layer.cuh"

namespace sparsp {

constexpr int kChunkBytes = 16384;
constexpr int kGradThreads = 256;

struct GradTensor {
  const void* from;
  void* to;
  int64_t size;
  int64_t first_chunk;  // that of the entry behind the last tensor: the number of chunks
};
// The table: tensors that have values, one entry behind them, then int32 [ctas + 1]: the tensor of the first chunk of each
// CTA's run.
struct GradParams {
  const GradTensor* tensors;
  const int32_t* begins_in;
  double* sum;
  double* partial;  // of each CTA
  uint32_t* ticket;
  float* norm;
  double limit;
  int32_t chunks, accumulate, in_place;
};

// elements before the first 16-byte boundary
template <typename T>
__host__ __device__ inline int64_t ahead(const void* p, int64_t size) {
  const int64_t n = (16 - (int64_t)((uintptr_t)p & 15)) / (int)sizeof(T) % (16 / (int)sizeof(T));
  return n < size ? n : size;
}

// The run of chunks of a CTA: the first `more` have one more than the others.
struct Runs {
  int each, more;
  __host__ __device__ Runs(int chunks, int ctas) : each(chunks / ctas), more(chunks % ctas) {}
  __host__ __device__ int begin(int cta) const { return cta * each + (cta < more ? cta : more); }
};

// Chunk number c of the list, one of tensor x: its elements [first, last).  Chunks are cut at 16-byte boundaries of where
// the tensor is read; what lies before the first one belongs to the first chunk.
template <typename T>
__device__ __forceinline__ void chunk_of(const GradTensor& x, int c, int64_t& first, int64_t& last) {
  const int64_t skip = ahead<T>(x.from, x.size), k = c - x.first_chunk;
  constexpr int64_t kEach = kChunkBytes / sizeof(T);
  first = k == 0 ? 0 : skip + k * kEach;
  last = min(skip + (k + 1) * kEach, x.size);
}

// f(values, from index, how many) for what this thread has of the elements [first, last): 16-byte pieces where
// `pieces`, single elements at the ends
template <typename T, typename Piece, typename Single>
__device__ __forceinline__ void walk_chunk(const T* from, int64_t first, int64_t last, bool pieces, Piece piece,
                                           Single single) {
  constexpr int E = 16 / sizeof(T), kMine = kChunkBytes / 16 / kGradThreads;
  const int64_t at = first + ahead<T>(from + first, last - first);
  if (!pieces) {
    for (int64_t i = first + threadIdx.x; i < last; i += kGradThreads) single(i);
    return;
  }
  if (first + threadIdx.x < at) single(first + threadIdx.x);
  Vec<T, E> v[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int64_t i = at + (k * kGradThreads + threadIdx.x) * E;
    if (i + E <= last)
      v[k] = load_vec<T, E>(from + i);
    else
      v[k].clear();
  }
  piece(v, at);
  const int64_t rest = at + (last - at) / E * E;
  if (rest + threadIdx.x < last) single(rest + threadIdx.x);
}

__device__ __forceinline__ double block_sum(double v, double* room) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kGradThreads / 32; ++w) v += room[w];
  __syncthreads();
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kGradThreads) grad_squares_kernel(GradParams p) {
  enter_grid(p.tensors, p.begins_in, p.partial, p.ticket);
  __shared__ double room[kGradThreads / 32];
  __shared__ bool s_last;
  constexpr int E = 16 / sizeof(T);
  const Runs runs(p.chunks, gridDim.x);
  const int end = runs.begin(blockIdx.x + 1);
  double sum = 0.0;
  int t = p.begins_in[blockIdx.x];
  for (int c = runs.begin(blockIdx.x); c < end; ++c) {
    if (c == p.tensors[t + 1].first_chunk) ++t;
    const GradTensor x = p.tensors[t];
    int64_t first, last;
    chunk_of<T>(x, c, first, last);
    const T* from = static_cast<const T*>(x.from);
    walk_chunk(
        from, first, last, true,
        [&](const auto& v, int64_t) {
          float s = 0.0f;
#pragma unroll
          for (const auto& w : v)
#pragma unroll
            for (int e = 0; e < E; ++e) s = fmaf(w[e], w[e], s);
          // outside these, squares may have been lost below fp32's range or gone beyond it
          if (s >= 0x1p-80f && s <= 0x1p100f) {
            sum += (double)s;
          } else {
            for (const auto& w : v)
#pragma unroll
              for (int e = 0; e < E; ++e) sum += (double)w[e] * (double)w[e];
          }
        },
        [&](int64_t i) {
          const double v = to_float(from[i]);
          sum += v * v;
        });
  }
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) {
    p.partial[blockIdx.x] = sum;
    __threadfence();
    s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  sum = 0.0;
  for (int i = threadIdx.x; i < gridDim.x; i += kGradThreads) sum += __ldcg(p.partial + i);
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) {
    *p.sum = p.accumulate ? *p.sum + sum : sum;
    *p.ticket = 0;
  }
}

template <typename T>
__global__ void __launch_bounds__(kGradThreads) grad_clip_kernel(GradParams p) {
  enter_grid(p.tensors, p.begins_in, p.sum);
  constexpr int E = 16 / sizeof(T);
  const double norm = sqrt(*p.sum);
  if (p.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = (float)norm;
  // (a norm that is not a number is no reason to change anything: the caller sees it)
  const float factor = isfinite(norm) ? (float)fmin(p.limit / (norm + 1e-6), 1.0) : 1.0f;
  if (factor == 1.0f && p.in_place) return;
  const Runs runs(p.chunks, gridDim.x);
  const int begin = runs.begin(blockIdx.x);
  int t = p.begins_in[blockIdx.x + 1];
  for (int c = runs.begin(blockIdx.x + 1) - 1; c >= begin; --c) {
    if (c < p.tensors[t].first_chunk) --t;
    const GradTensor x = p.tensors[t];
    int64_t first, last;
    chunk_of<T>(x, c, first, last);
    const T* from = static_cast<const T*>(x.from);
    T* to = static_cast<T*>(x.to);
    const bool pieces = (((uintptr_t)from ^ (uintptr_t)to) & 15) == 0;
    walk_chunk(
        from, first, last, pieces,
        [&](auto& v, int64_t at) {
#pragma unroll
          for (int k = 0; k < kChunkBytes / 16 / kGradThreads; ++k) {
            const int64_t i = at + (k * kGradThreads + threadIdx.x) * E;
            if (i + E > last) continue;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = v[k][e] * factor;
            v[k].set(y);
            store_vec<T, E>(to + i, v[k]);
          }
        },
        [&](int64_t i) { to[i] = from_float<T>(to_float(from[i]) * factor); });
  }
}

// ---- host side ------------------------------------------------------------------------------------------------------

int64_t grad_workspace_bytes() { return 512 + kGradCtas * 8; }

int64_t grad_table_bytes(const sparsp_grad_list& l) {
  return ((int64_t)l.count + 1) * (int64_t)sizeof(GradTensor) + (kGradCtas + 1) * 4;
}

int fill_grad_table(sparsp_grad_list* l, void* table) {
  GradTensor* tensor = static_cast<GradTensor*>(table);
  int32_t* begins_in = reinterpret_cast<int32_t*>(tensor + l->count + 1);
  const int e = element_bytes(l->dtype);
  const int64_t each = kChunkBytes / e;
  int64_t chunks = 0;
  int n = 0;
  l->in_place = 1;
  for (int i = 0; i < l->count; ++i) {
    const int64_t size = l->sizes[i];
    if (size == 0) continue;
    void* to = l->outs != nullptr ? l->outs[i] : const_cast<void*>(l->grads[i]);
    if (to != l->grads[i]) l->in_place = 0;
    tensor[n++] = {l->grads[i], to, size, chunks};
    const int64_t skip = e == 4 ? ahead<float>(l->grads[i], size) : ahead<__half>(l->grads[i], size);
    chunks += std::max<int64_t>(1, (size - skip + each - 1) / each);
    if (chunks > 0x7fffffff - 2 * kGradCtas) {
      set_error("the gradients are too large");
      return SPARSP_ERR_UNSUPPORTED;
    }
  }
  tensor[n] = {nullptr, nullptr, 0, chunks};
  l->chunks = (int32_t)chunks;
  l->ctas = (int32_t)std::max<int64_t>(1, std::min<int64_t>(chunks, kGradCtas));
  const Runs runs(l->chunks, l->ctas);
  for (int b = 0, t = 0; b <= l->ctas; ++b) {
    while (t < n && tensor[t + 1].first_chunk <= runs.begin(b)) ++t;
    begins_in[b] = t;
  }
  return SPARSP_OK;
}

static GradParams grad_params(const sparsp_grad_list& l, const void* table, char* ws) {
  GradParams p = {};
  p.tensors = static_cast<const GradTensor*>(table);
  p.begins_in = reinterpret_cast<const int32_t*>(p.tensors + l.count + 1);
  p.ticket = reinterpret_cast<uint32_t*>(ws + 128);
  p.sum = reinterpret_cast<double*>(ws + 256);
  p.partial = reinterpret_cast<double*>(ws + 512);
  p.chunks = l.chunks;
  p.in_place = l.in_place;
  return p;
}

int launch_grad_squares(const sparsp_grad_list& l, const void* table, int accumulate, char* ws, cudaStream_t st) {
  GradParams p = grad_params(l, table, ws);
  p.accumulate = accumulate;
  SPARSP_WITH_TYPE(l.dtype, T, SPARSP_CUDA_OK(launch_kernel(grad_squares_kernel<T>, dim3((unsigned)l.ctas), kGradThreads, 0,
                                                            st, p)));
  return SPARSP_OK;
}

int launch_grad_clip(const sparsp_grad_list& l, const void* table, double limit, float* norm, char* ws,
                     cudaStream_t st) {
  GradParams p = grad_params(l, table, ws);
  p.limit = limit;
  p.norm = norm;
  SPARSP_WITH_TYPE(l.dtype, T, SPARSP_CUDA_OK(launch_kernel(grad_clip_kernel<T>, dim3((unsigned)l.ctas), kGradThreads, 0, st,
                                                            p)));
  return SPARSP_OK;
}

// Whether something is written where something else is read or written; -1: no host memory to find out.  A gradient that
// is clipped in place counts as written alone.
int grad_outputs_overlap(const sparsp_grad_list& l) {
  const int64_t e = element_bytes(l.dtype);
  auto out = [&](int i) { return l.outs != nullptr ? l.outs[i] : l.grads[i]; };
  uintptr_t end = 0;
  bool ordered = true;  // all in place, one behind the other
  for (int i = 0; i < l.count && ordered; ++i) {
    if (l.sizes[i] == 0) continue;
    ordered = out(i) == l.grads[i] && (uintptr_t)out(i) >= end;
    end = (uintptr_t)out(i) + l.sizes[i] * e;
  }
  if (ordered) return 0;
  struct Run {
    uintptr_t begin, end;
    bool written;
  };
  try {
    std::vector<Run> runs;
    runs.reserve(2 * (size_t)l.count);
    for (int i = 0; i < l.count; ++i) {
      if (l.sizes[i] == 0) continue;
      const uintptr_t at = (uintptr_t)out(i), from = (uintptr_t)l.grads[i], bytes = l.sizes[i] * e;
      runs.push_back({at, at + bytes, true});
      if (from != at) runs.push_back({from, from + bytes, false});
    }
    std::sort(runs.begin(), runs.end(), [](const Run& a, const Run& b) { return a.begin < b.begin; });
    uintptr_t read = 0, written = 0;  // ends of what has begun
    for (const Run& r : runs) {
      if (r.begin < written || (r.written && r.begin < read)) return 1;
      (r.written ? written : read) = std::max(r.written ? written : read, r.end);
    }
  } catch (const std::bad_alloc&) {
    return -1;
  }
  return 0;
}

}  // namespace sparsp
