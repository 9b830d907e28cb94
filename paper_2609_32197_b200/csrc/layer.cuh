// What the token-wise operators of a layer (rotary positions, layer norm, gated feed-forward) share: element types,
// 16-byte vectors of them, and their launchers.
#pragma once

#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace sparsp {

constexpr int kMaxRotaryHeadDim = 256;
constexpr int kMaxNormDim = 16384;
// Work is shared out for the multiprocessors of a B200, whatever device a size of workspace is asked on: the shares
// also decide in which order sums are made.
constexpr int kSms = 148;

inline int element_bytes(int dtype) { return dtype == SPARSP_FP32 ? 4 : 2; }

#ifdef __CUDACC__
template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float to_float<__half>(__half v) {
  return __half2float(v);
}
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) {
  return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __half from_float<__half>(float v) {
  return __float2half_rn(v);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}
// two values as the type's 32-bit pair, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// E consecutive elements as they lie in memory: one 16-byte access, or single elements.  Pairs of 16-bit values stay in
// the 32-bit words they were loaded in until they are used: taken apart at the load, they would make it be waited for.
template <typename T, int E>
struct Vec {
  static_assert(E == 1, "");
  T v;
  __device__ __forceinline__ float operator[](int) const { return to_float<T>(v); }
  __device__ __forceinline__ void set(const float* x) { v = from_float<T>(x[0]); }
  __device__ __forceinline__ void clear() { v = from_float<T>(0.0f); }
};
template <>
struct alignas(16) Vec<float, 4> {
  uint32_t w[4];
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i]); }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
};
template <typename T>
struct alignas(16) Vec<T, 8> {
  uint32_t w[4];
  __device__ __forceinline__ float operator[](int i) const {
    const uint32_t x = w[i / 2];
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
    } else {
      const __half2 h = *reinterpret_cast<const __half2*>(&x);
      return i & 1 ? __high2float(h) : __low2float(h);
    }
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
};
template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_vec(const T* p) {
  Vec<T, E> r;
  if constexpr (E == 1) {
    r.v = *p;
  } else {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    r.w[0] = x.x;
    r.w[1] = x.y;
    r.w[2] = x.z;
    r.w[3] = x.w;
  }
  return r;
}
// ... of data that this kernel reads once: it need not stay in L1
template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_once(const T* p) {
  Vec<T, E> r;
  if constexpr (E == 1) {
    r.v = *p;
  } else {
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
    r.w[0] = x.x;
    r.w[1] = x.y;
    r.w[2] = x.z;
    r.w[3] = x.w;
  }
  return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, E>& x) {
  if constexpr (E == 1)
    *p = x.v;
  else
    *reinterpret_cast<uint4*>(p) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
}

// Runs the statements with T as the element type.
#define SPARSP_WITH_TYPE(dtype, T, ...)      \
  do {                                       \
    if ((dtype) == SPARSP_BF16) {            \
      using T = __nv_bfloat16;               \
      __VA_ARGS__;                           \
    } else if ((dtype) == SPARSP_FP16) {     \
      using T = __half;                      \
      __VA_ARGS__;                           \
    } else {                                 \
      using T = float;                       \
      __VA_ARGS__;                           \
    }                                        \
  } while (0)
#endif

int launch_rotary_table(const sparsp_rotary& r, const double* inv_freq, double amplitude, float* table,
                        cudaStream_t st);
int launch_rotary(const sparsp_shape& s, const sparsp_rotary& r, const float* table, const int32_t* positions,
                  int64_t positions_stride_batch, const int32_t* origin, const void* Q, const void* K, void* Qo,
                  void* Ko, int inverse, int32_t* status, cudaStream_t st);

int64_t norm_groups(const sparsp_norm& n);
int64_t norm_workspace_bytes(const sparsp_norm& n);
int launch_norm_fwd(const sparsp_norm& n, const void* X, const void* w, const void* b, void* Y, float* mean,
                    float* rstd, cudaStream_t st);
int launch_norm_bwd(const sparsp_norm& n, const void* dY, const void* X, const void* w, const float* mean,
                    const float* rstd, void* dX, void* dw, void* db, char* ws, cudaStream_t st);

int64_t ffn_workspace_bytes(const sparsp_ffn& f, bool backward);
int launch_ffn_fwd(const sparsp_ffn& f, const void* X, const void* Wg, const void* Wu, void* H, void* gate, void* up,
                   char* ws, cudaStream_t st);
int launch_ffn_bwd(const sparsp_ffn& f, const void* dH, const void* X, const void* Wg, const void* Wu,
                   const void* gate, const void* up, void* dX, void* dWg, void* dWu, char* ws, cudaStream_t st);

}  // namespace sparsp
