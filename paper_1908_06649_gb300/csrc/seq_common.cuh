// seq_common.cuh -- what the sequence operators' kernels share: element types
// and their vector accesses, the activations, packed sequences, and the
// argument checks of their entry points (include/tcu_seq.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/tcu_seq.h"

namespace tcu {
namespace seq {

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(f16 v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ f16 from_f<f16>(float v) { return __float2half_rn(v); }

// V adjacent values, accessed as one word of V * sizeof(T) <= 16 bytes; the
// address is aligned to that (vector_width below).
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ void load_vec(float (&out)[V], const T *p) {
  const Vec<T, V> w = *reinterpret_cast<const Vec<T, V> *>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) out[i] = to_f(w.v[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&in)[V]) {
  Vec<T, V> w;
#pragma unroll
  for (int i = 0; i < V; ++i) w.v[i] = from_f<T>(in[i]);
  *reinterpret_cast<Vec<T, V> *>(p) = w;
}

// 2^x by the special function unit (relative error 2^-22; 2^-inf = 0).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float sigmoid(float v) {
  return __fdividef(1.f, 1.f + exp2_fast(-kLog2e * v));
}
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
__device__ __forceinline__ float dsilu(float v) {
  const float s = sigmoid(v);
  return s * (1.f + v * (1.f - s));
}

// A row tensor of element type T.
template <typename T>
struct Rows {
  T *p;
  int64_t batch, row;
  __device__ __forceinline__ T *at(int64_t b, int64_t t) const { return p + b * batch + t * row; }
};

// The sequence that holds row t of a packed tensor: the last s with
// offsets[s] <= t < offsets[s + 1], -1 if t is in none (values out of order
// still give -1 <= s < count).
__device__ __forceinline__ int sequence_of(const int32_t *offsets, int count, int64_t t) {
  int lo = 0, hi = count;  // offsets[lo] <= t unless lo == 0
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (offsets[mid + 1] <= t) lo = mid + 1; else hi = mid;
  }
  return lo < count && offsets[lo] <= t ? lo : -1;
}

// ------------------------------------------------------------- host side
inline int type_size(int type) { return type == TCU_SEQ_F32 ? 4 : 2; }

// Whether every row of r starts at a multiple of `bytes`, so that rows can be
// accessed in words of that many bytes (entries without rows to step over
// have no say).
inline bool rows_aligned(const tcu_seq_rows &r, int type, int64_t batches, int64_t rows,
                         int bytes) {
  const int64_t sz = type_size(type);
  return (uintptr_t)r.ptr % bytes == 0 && (rows <= 1 || r.row_stride * sz % bytes == 0) &&
         (batches <= 1 || r.batch_stride * sz % bytes == 0);
}

inline bool row_ok(const tcu_seq_rows &r, int size) {
  return r.ptr && (uintptr_t)r.ptr % size == 0;
}
inline bool f32_ok(const void *p) { return p && (uintptr_t)p % 4 == 0; }
inline bool opt_ok(const void *p, int size) { return (uintptr_t)p % size == 0; }

inline int launched() {
  return cudaGetLastError() == cudaSuccess ? TCU_DFT_OK : TCU_DFT_ERR_CUDA;
}

template <typename T>
inline Rows<T> rows_of(const tcu_seq_rows &r) {
  return {static_cast<T *>(r.ptr), r.batch_stride, r.row_stride};
}

// Streaming multiprocessors of the current device.
inline int num_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return 1;
  }
  return n;
}

// Sums partial[p][i] over p < parts in order, one value per thread: the
// second step of the parameter gradients (the same result in every run).
__global__ void sum_parts_kernel(float *out, const float *partial, int64_t parts, int64_t count);
int sum_parts(float *out, const float *partial, int64_t parts, int64_t count, cudaStream_t st);

}  // namespace seq
}  // namespace tcu
