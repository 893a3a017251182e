// seq_common.cuh -- what the sequence operators' kernels share: element types
// and their vector accesses, the activations, packed sequences, and the
// argument checks of their entry points (include/tcu_seq.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/tcu_seq.h"
#include "seq_index.h"

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
// address is aligned to that.
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T v[V];
};
// 2^x by the special function unit (relative error 2^-22; 2^-inf = 0).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float rcp_fast(float x) {  // 1 / inf = 0
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float sigmoid(float v) {
  return rcp_fast(1.f + exp2_fast(-kLog2e * v));
}
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
__device__ __forceinline__ float2 sigmoid2(float2 v) {
  const float2 e = __fmul2_rn(v, make_float2(-kLog2e, -kLog2e));
  const float2 w = __fadd2_rn(make_float2(exp2_fast(e.x), exp2_fast(e.y)), make_float2(1.f, 1.f));
  return make_float2(rcp_fast(w.x), rcp_fast(w.y));
}
__device__ __forceinline__ float2 silu2(float2 v) { return __fmul2_rn(v, sigmoid2(v)); }
// (v sigma(v))' = s + v s (1 - s)
__device__ __forceinline__ float2 dsilu2(float2 v) {
  const float2 s = sigmoid2(v), vs = __fmul2_rn(v, s);
  return __ffma2_rn(vs, __ffma2_rn(s, make_float2(-1.f, -1.f), make_float2(1.f, 1.f)), s);
}

// log(1 + exp(v)) of two values: max(v, 0) + log1p(e), e = exp(-|v|) <= 1, and
// log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3.  2 artanh(s) / s is a
// polynomial of degree 4 in s^2, fitted at the Chebyshev nodes of [0, 1/9]
// (relative error 7.6e-9), so that small e keep their relative accuracy, which
// log(1 + e) would lose.
__device__ __forceinline__ float2 softplus2(float2 v) {
  const float2 e = make_float2(exp2_fast(-kLog2e * fabsf(v.x)), exp2_fast(-kLog2e * fabsf(v.y)));
  const float2 w = __fadd2_rn(e, make_float2(2.f, 2.f));
  const float2 s = __fmul2_rn(e, make_float2(rcp_fast(w.x), rcp_fast(w.y)));
  const float2 q = __fmul2_rn(s, s);
  float2 p = make_float2(0.28157779f, 0.28157779f);
  p = __ffma2_rn(p, q, make_float2(0.27965158f, 0.27965158f));
  p = __ffma2_rn(p, q, make_float2(0.40024596f, 0.40024596f));
  p = __ffma2_rn(p, q, make_float2(0.66666323f, 0.66666323f));
  p = __ffma2_rn(p, q, make_float2(2.f, 2.f));
  return __ffma2_rn(s, p, make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}

// Two adjacent values of a type in 32-bit words, and back.
template <typename T>
struct Pair;
template <>
struct Pair<float> {
  static constexpr int kWords = 2;
  static __device__ __forceinline__ float2 get(const uint32_t *w) {
    return make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
  }
  static __device__ __forceinline__ void put(uint32_t *w, float2 v) {
    w[0] = __float_as_uint(v.x);
    w[1] = __float_as_uint(v.y);
  }
};
template <>
struct Pair<bf16> {
  static constexpr int kWords = 1;
  static __device__ __forceinline__ float2 get(const uint32_t *w) {
    return make_float2(__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u));
  }
  static __device__ __forceinline__ void put(uint32_t *w, float2 v) {
    const __nv_bfloat162 p = __float22bfloat162_rn(v);
    w[0] = *reinterpret_cast<const uint32_t *>(&p);
  }
};
template <>
struct Pair<f16> {
  static constexpr int kWords = 1;
  static __device__ __forceinline__ float2 get(const uint32_t *w) {
    return __half22float2(*reinterpret_cast<const __half2 *>(w));
  }
  static __device__ __forceinline__ void put(uint32_t *w, float2 v) {
    const __half2 p = __float22half2_rn(v);
    w[0] = *reinterpret_cast<const uint32_t *>(&p);
  }
};

// One value as it lies in memory, in a word of its own, and back.
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(bf16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ uint32_t bits_of(f16 v) { return __half_as_ushort(v); }
template <typename T>
__device__ __forceinline__ float of_bits(uint32_t w);
template <>
__device__ __forceinline__ float of_bits<float>(uint32_t w) { return __uint_as_float(w); }
template <>
__device__ __forceinline__ float of_bits<bf16>(uint32_t w) { return __uint_as_float(w << 16); }
template <>
__device__ __forceinline__ float of_bits<f16>(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)w));
}

// V values (V even) as they lie in memory, in words (kApart: one value each)
// so that nothing waits for them before they are used: adjacent ones in loads and stores of up to 16
// bytes where kWide, value by value at a pitch of `gap` otherwise; those from
// `count` on are neither read nor written (kWide: count is V or at most 0).
template <typename T, int V, bool kApart = false>
struct Raw {
  static constexpr int kPairWords = kApart ? 2 : Pair<T>::kWords, kWords = V / 2 * kPairWords;
  static constexpr int kStep = kWords % 4 == 0 ? 4 : kWords % 2 == 0 ? 2 : 1;
  uint32_t w[kWords];
  __device__ __forceinline__ float2 pair(int i) const {
    if constexpr (kApart) return make_float2(of_bits<T>(w[2 * i]), of_bits<T>(w[2 * i + 1]));
    else return Pair<T>::get(w + i * kPairWords);
  }
  __device__ __forceinline__ void set(int i, float2 v) {
    if constexpr (kApart) w[2 * i] = bits_of(from_f<T>(v.x)), w[2 * i + 1] = bits_of(from_f<T>(v.y));
    else Pair<T>::put(w + i * kPairWords, v);
  }
  template <bool kWide>
  __device__ __forceinline__ void load(const T *p, int count, int64_t gap = 1) {
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = 0;
      if (count > 0) {
#pragma unroll
        for (int i = 0; i < kWords / kStep; ++i) {
          const Vec<uint32_t, kStep> v = reinterpret_cast<const Vec<uint32_t, kStep> *>(p)[i];
#pragma unroll
          for (int j = 0; j < kStep; ++j) w[i * kStep + j] = v.v[j];
        }
      }
    } else if constexpr (kApart) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = i < count ? bits_of(p[i * gap]) : 0;
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i)
        set(i, make_float2(2 * i < count ? to_f(p[2 * i * gap]) : 0.f,
                           2 * i + 1 < count ? to_f(p[(2 * i + 1) * gap]) : 0.f));
    }
  }
  template <bool kWide>
  __device__ __forceinline__ void store(T *p, int count, int64_t gap = 1) const {
    if constexpr (kWide) {
      if (count > 0) {
#pragma unroll
        for (int i = 0; i < kWords / kStep; ++i) {
          Vec<uint32_t, kStep> v;
#pragma unroll
          for (int j = 0; j < kStep; ++j) v.v[j] = w[i * kStep + j];
          reinterpret_cast<Vec<uint32_t, kStep> *>(p)[i] = v;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float2 v = pair(i);
        if (2 * i < count) p[2 * i * gap] = from_f<T>(v.x);
        if (2 * i + 1 < count) p[(2 * i + 1) * gap] = from_f<T>(v.y);
      }
    }
  }
};

// A row tensor of element type T.
template <typename T>
struct Rows {
  T *p;
  int64_t batch;
  int32_t row;  // one 32-bit product for a row's address (pitch_fits)
  __device__ __forceinline__ T *at(int64_t b, int32_t t) const {
    return p + b * batch + (int64_t)t * row;
  }
};

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
// Rows, and the pitch of `rows` rows, within 32 bits, with room to step past
// the end (one row's pitch is never taken, whatever it is cut to).
constexpr int64_t kMostRows = INT32_MAX - 4096;
inline bool pitch_fits(int64_t rows, int64_t stride) {
  return rows <= 1 || (stride >= INT32_MIN && stride <= INT32_MAX);
}
inline bool f32_ok(const void *p) { return p && (uintptr_t)p % 4 == 0; }
inline bool opt_ok(const void *p, int size) { return (uintptr_t)p % size == 0; }

// Whether the `bytes` at p, advanced in place, share one with `count` rows of
// `run` bytes at q, `stride` bytes apart (of any size: these are the caller's).
using wide_int = __int128;
inline bool over(const void *p, wide_int bytes, const void *q, int64_t run, int64_t count = 1,
                 int64_t stride = 0) {
  if (!p || !q || bytes <= 0 || run <= 0 || count <= 0) return false;
  const wide_int lo = (wide_int)(uintptr_t)p, hi = lo + bytes;
  wide_int a = (wide_int)(uintptr_t)q, s = count > 1 ? stride : 0;
  if (s < 0) a += s * (count - 1), s = -s;
  // the first row that ends behind lo
  const wide_int k = a + run > lo || s == 0 ? 0 : (lo - run - a) / s + 1;
  return k < count && a + k * s < hi && a + k * s + run > lo;
}

inline int launched() {
  return cudaGetLastError() == cudaSuccess ? TCU_DFT_OK : TCU_DFT_ERR_CUDA;
}

template <typename T>
inline Rows<T> rows_of(const tcu_seq_rows &r) {
  return {static_cast<T *>(r.ptr), r.batch_stride, (int32_t)r.row_stride};
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

// The second step of the parameter gradients: out[i] = sum over p < parts of
// parts[p * stride + i], always in the same order; up to three at once.  A
// stride of 0 is each sum's own count.
struct Sum {
  float *out;
  const float *parts;
  int64_t count;
};
int sum_parts(const Sum *sums, int count, int64_t parts, int64_t stride, cudaStream_t st);

}  // namespace seq
}  // namespace tcu
