// norm_rotate.cu -- the norm of each head of queries and keys with the rotation
// by position, and its gradient (include/tcu_attn.h).
//
// Per head of d values x, with weights w:
//     r = 1 / sqrt(sum x^2 / d + eps),   n = x r,   y = R (n w)
// R turning pairs of values by position x rate; its gradient, g = R^T dy:
//     dw = sum over rows and heads of g n
//     dx = r g w - x r^3 (sum g w x) / d
// Some ten operations for each value read and written: HBM bounds it.  A warp
// owns a row, with a few lanes for each head; a lane holds the same pairs of
// every head, so that a row's angles are formed once for all its heads.  Both
// values of a pair are in the same lane: rows may be written over those that
// they come from.
//
// Measured, bf16, 16384 rows x 40 heads x 128: forward (336 MB) 60 us, 5.6 TB/s;
// gradient (503 MB) 110 us and 10 for the sum of its shares, 4.2 TB/s.
#include <algorithm>

#include "../../include/tcu_attn.h"
#include "seq_common.cuh"

namespace tcu {
namespace seq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;

template <typename T>
struct RotateArgs {
  Rows<const T> q, k, dyq, dyk;
  Rows<T> yq, yk, dq, dk;
  const float *rates, *q_weight, *k_weight;
  float *parts;  // [block]{q: dim, k: dim}
  const int32_t *offsets, *positions;
  int64_t rows, total;  // of a batch entry, of all
  int sequences, heads, kv_heads, dim, turned;
  int lanes;  // of a head, a power of two
  float eps;
};

// The turns of one position, in 2^-64, of each pair of a head; whole turns
// change nothing.  1 / (2 pi) is taken in two parts, 2^-110 off, and the product
// with the first in two, so that a position near 2^31 multiplies 2^-63 turns, not
// the 2^-55 of one product (rates up to 2^32; larger ones lose what they are).
constexpr int kPairs = TCU_ATTN_MAX_NORM_DIM / 2;
struct Turns {
  uint64_t of_one[kPairs];
  float unit[kPairs];  // half turns of the upper 32 bits' unit; no number where the rate is none
};
__device__ __forceinline__ uint64_t fraction(double t) {
  const double f = fabs(t) - floor(fabs(t));
  const uint64_t u = (uint64_t)(f * 18446744073709551616.0);
  return t < 0 ? 0 - u : u;
}
template <typename T>
__device__ __forceinline__ void fill_turns(const RotateArgs<T> &a, Turns &turns) {
  for (int p = threadIdx.x; p < kPairs; p += kThreads) {
    uint64_t u = 0;
    float unit = 4.656612873077393e-10f;  // 2^-31
    if (p < a.turned) {
      constexpr double kTurn = 0.15915494309189535, kRest = -9.839338337591243e-18;
      const double rate = a.rates[p], t = rate * kTurn;
      if (fabs(rate) < INFINITY) u = fraction(t) + fraction(fma(rate, kRest, fma(rate, kTurn, -t)));
      else unit = __int_as_float(0x7fffffff);
    }
    turns.of_one[p] = u;
    turns.unit[p] = unit;
  }
  __syncthreads();
}

// A lane's part of a head: kParts parts of VP adjacent pairs, in two words of
// VP values each.  Pairs that are turned with their partner `turned` values on
// lie at (p, p + turned), others at (2p, 2p + VP).
template <int VP>
struct Part {
  static constexpr int kParts = VP >= 4 ? 1 : 4 / VP;
};

// A lane's values of a head as they lie in memory.
template <typename T, int VP>
struct Words {
  Vec<T, VP> w[Part<VP>::kParts][2];
};

template <typename T, int VP, bool kInter>
struct Lane {
  static constexpr int kParts = Part<VP>::kParts;
  int first[kParts], at[kParts][2];  // pair, values
  bool has[kParts];

  __device__ __forceinline__ void init(const RotateArgs<T> &a, int j) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int p = (j + k * a.lanes) * VP;
      has[k] = p < a.dim / 2;
      first[k] = has[k] ? p : 0;
      const bool apart = !kInter && p < a.turned;
      at[k][0] = apart ? p : 2 * p;
      at[k][1] = apart ? p + a.turned : 2 * p + VP;
    }
  }
  // The lane's values in pairs, for packed arithmetic: a pair and its partner
  // where they are adjacent (or VP is 1), else two values of a word, words in
  // order.
  static constexpr bool kTogether = kInter || VP == 1;
  using Values = float2[kParts][VP];
  struct Angles {
    float c[kParts][VP], s[kParts][VP];
  };

  // cos and sin of the lane's angles at a position: the product wraps as turns
  // do; of its 32 bits fp32 keeps 24, 2^-26 turns
  __device__ __forceinline__ void angles(const Turns &turns, int64_t position, Angles &a) const {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int i = 0; i < VP; ++i) {
        const int p = first[k] + i;
        const int32_t t = (int32_t)(uint32_t)(((uint64_t)position * turns.of_one[p]) >> 32);
        sincospif((float)t * turns.unit[p], &a.s[k][i], &a.c[k][i]);
      }
  }
  __device__ __forceinline__ void load(const T *head, bool in, Words<T, VP> &v) const {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (in && has[k]) {
          v.w[k][j] = *reinterpret_cast<const Vec<T, VP> *>(head + at[k][j]);
        } else {
#pragma unroll
          for (int i = 0; i < VP; ++i) v.w[k][j].v[i] = from_f<T>(0.f);
        }
      }
  }
  static __device__ __forceinline__ void values(const Words<T, VP> &w, Values &v) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      if constexpr (VP == 1) {
        v[k][0] = make_float2(to_f(w.w[k][0].v[0]), to_f(w.w[k][1].v[0]));
      } else {
        constexpr int kWords = Pair<T>::kWords;
#pragma unroll
        for (int i = 0; i < VP; ++i)
          v[k][i] = Pair<T>::get(reinterpret_cast<const uint32_t *>(&w.w[k][i / (VP / 2)]) +
                                 i % (VP / 2) * kWords);
      }
    }
  }
  __device__ __forceinline__ void store(T *head, bool in, const Values &v) const {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (!in || !has[k]) continue;
        Vec<T, VP> w;
        if constexpr (VP == 1) {
          w.v[0] = from_f<T>(j ? v[k][0].y : v[k][0].x);
        } else {
#pragma unroll
          for (int i = 0; i < VP / 2; ++i)
            Pair<T>::put(reinterpret_cast<uint32_t *>(&w) + i * Pair<T>::kWords, v[k][j * (VP / 2) + i]);
        }
        *reinterpret_cast<Vec<T, VP> *>(head + at[k][j]) = w;
      }
  }
  // turns by the angles (kBack: against them)
  template <bool kBack>
  static __device__ __forceinline__ void rotate(Values &v, const Angles &a) {
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      if constexpr (kTogether) {
#pragma unroll
        for (int i = 0; i < VP; ++i) {
          const float c = a.c[k][i], s = kBack ? -a.s[k][i] : a.s[k][i];
          const float2 x = v[k][i];
          v[k][i] = __ffma2_rn(x, make_float2(c, c), __fmul2_rn(make_float2(x.y, x.x), make_float2(-s, s)));
        }
      } else {
#pragma unroll
        for (int i = 0; i < VP / 2; ++i) {
          const float2 c = make_float2(a.c[k][2 * i], a.c[k][2 * i + 1]);
          const float2 s = make_float2(a.s[k][2 * i], a.s[k][2 * i + 1]), n = make_float2(-s.x, -s.y);
          const float2 x = v[k][i], y = v[k][VP / 2 + i];
          v[k][i] = __ffma2_rn(x, c, __fmul2_rn(y, kBack ? s : n));
          v[k][VP / 2 + i] = __ffma2_rn(y, c, __fmul2_rn(x, kBack ? n : s));
        }
      }
    }
  }
  // Where value j (0, 1) of pair i of part k lies in a head.
  __device__ __forceinline__ int place(int k, int i, int j) const {
    if constexpr (VP == 1) return at[k][j];
    else return at[k][i / (VP / 2)] + 2 * (i % (VP / 2)) + j;
  }
  __device__ __forceinline__ void weights(const float *w, Values &v) const {
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int i = 0; i < VP; ++i)
        v[k][i] = !has[k] ? make_float2(0.f, 0.f)
                  : w     ? make_float2(w[place(k, i, 0)], w[place(k, i, 1)])
                          : make_float2(1.f, 1.f);
  }
};

__device__ __forceinline__ float sum_lanes(float v, int lanes) {
  for (int m = 1; m < lanes; m *= 2) v += __shfl_xor_sync(~0u, v, m);
  return v;
}

// The row's batch entry, number and position; false for a row of no sequence.
template <typename T>
__device__ __forceinline__ bool place_of(const RotateArgs<T> &a, int64_t id, int64_t &b, int &t,
                                         int64_t &position) {
  b = id / a.rows;
  t = (int)(id - b * a.rows);
  position = t;
  if (a.offsets) {
    const int s = sequence_of(a.offsets, a.sequences, t);
    if (s < 0) return false;
    position = t - a.offsets[s];
  }
  if (a.positions) position = a.positions[id];
  return true;
}

// Heads of a lane whose loads are on their way together, and the longest word.
// At 16384 rows x 40 heads x 128, bf16 (168 MB), launches included, forward: words
// of 8 values, 4 heads 66 us, 5 heads 68, of 4 values 83.  The gradient holds two
// tensors and its sums beside them: words of 4, 4 heads 123 us, 2 heads 140, 3
// heads 136; words of 8 146.  Three blocks an SM: 91 and 146.
template <int VP>
constexpr int kAtOnce = VP >= 4 ? 4 : 2;
template <typename T, int VP>
constexpr int kGradAtOnce = VP == 4 && sizeof(T) == 2 ? 4 : 2;
constexpr int kGradWord = 4;

template <typename T, int VP, bool kInter>
__global__ void __launch_bounds__(kThreads, 2) rotate_kernel(const RotateArgs<T> a) {
  constexpr int kParts = Part<VP>::kParts, kMany = kAtOnce<VP>;
  __shared__ Turns turns;
  fill_turns(a, turns);
  const int lane = threadIdx.x % 32, per = 32 / a.lanes, sub = lane / a.lanes;
  using L = Lane<T, VP, kInter>;
  L own;
  own.init(a, lane % a.lanes);
  const float inv = 1.f / a.dim;
  const int64_t step = (int64_t)gridDim.x * kWarps;
  for (int64_t id = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; id < a.total; id += step) {
    int64_t b, position;
    int t;
    if (!place_of(a, id, b, t, position)) continue;
    typename L::Angles angles;
    own.angles(turns, position, angles);
    auto heads = [&](const T *from, T *to, int count, const float *weight) {
      typename L::Values w;
      own.weights(weight, w);
      for (int h0 = sub; h0 - sub < count; h0 += kMany * per) {
        Words<T, VP> words[kMany];
#pragma unroll
        for (int m = 0; m < kMany; ++m)
          own.load(from + (int64_t)(h0 + m * per) * a.dim, h0 + m * per < count, words[m]);
#pragma unroll
        for (int m = 0; m < kMany; ++m) {
          if (h0 - sub + m * per >= count) break;  // the whole warp
          typename L::Values v;
          own.values(words[m], v);
          float2 squares = make_float2(0.f, 0.f);
#pragma unroll
          for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < VP; ++i) squares = __ffma2_rn(v[k][i], v[k][i], squares);
          const float r = rsqrtf(fmaf(sum_lanes(squares.x + squares.y, a.lanes), inv, a.eps));
#pragma unroll
          for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int i = 0; i < VP; ++i)
              v[k][i] = __fmul2_rn(__fmul2_rn(v[k][i], make_float2(r, r)), w[k][i]);
          own.template rotate<false>(v, angles);
          own.store(to + (int64_t)(h0 + m * per) * a.dim, h0 + m * per < count, v);
        }
      }
    };
    heads(a.q.at(b, t), a.yq.at(b, t), a.heads, a.q_weight);
    heads(a.k.at(b, t), a.yk.at(b, t), a.kv_heads, a.k_weight);
  }
}

template <int VP>
struct GradShared {
  // each lane's shares of dw, [queries, keys][value][thread]
  float shares[2][2 * VP * Part<VP>::kParts][kThreads];
  float sums[kWarps][2 * TCU_ATTN_MAX_NORM_DIM];
  Turns turns;
};

template <typename T, int VP, bool kInter>
__global__ void __launch_bounds__(kThreads, 2) rotate_grad_kernel(const RotateArgs<T> a) {
  constexpr int kParts = Part<VP>::kParts, kMany = kGradAtOnce<T, VP>;
  extern __shared__ __align__(16) uint8_t raw[];
  GradShared<VP> &sh = *reinterpret_cast<GradShared<VP> *>(raw);
  fill_turns(a, sh.turns);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int per = 32 / a.lanes, sub = lane / a.lanes;
  using L = Lane<T, VP, kInter>;
  L own;
  own.init(a, lane % a.lanes);
#pragma unroll
  for (int i = 0; i < 2 * VP * kParts; ++i)
    sh.shares[0][i][threadIdx.x] = sh.shares[1][i][threadIdx.x] = 0.f;
  const float inv = 1.f / a.dim;
  const int64_t step = (int64_t)gridDim.x * kWarps;
  for (int64_t id = (int64_t)blockIdx.x * kWarps + warp; id < a.total; id += step) {
    int64_t b, position;
    int t;
    const bool row = place_of(a, id, b, t, position);
    typename L::Angles angles;
    if (row) own.angles(sh.turns, position, angles);
    auto heads = [&](const T *from, const T *dy, T *to, int count, const float *weight, int which) {
      typename L::Values w, dw;
      own.weights(weight, w);
#pragma unroll
      for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int i = 0; i < VP; ++i) dw[k][i] = make_float2(0.f, 0.f);
      for (int h0 = sub; h0 - sub < count; h0 += kMany * per) {
        Words<T, VP> xs[kMany], gs[kMany];
#pragma unroll
        for (int m = 0; m < kMany; ++m) {
          const bool in = row && h0 + m * per < count;
          own.load(from + (int64_t)(h0 + m * per) * a.dim, in, xs[m]);
          own.load(dy + (int64_t)(h0 + m * per) * a.dim, in, gs[m]);
        }
#pragma unroll
        for (int m = 0; m < kMany; ++m) {
          if (h0 - sub + m * per >= count) break;  // the whole warp
          typename L::Values x, g;
          own.values(xs[m], x);
          own.values(gs[m], g);
          if (row) {
            own.template rotate<true>(g, angles);
            float2 squares = make_float2(0.f, 0.f), dots = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kParts; ++k)
#pragma unroll
              for (int i = 0; i < VP; ++i) {
                squares = __ffma2_rn(x[k][i], x[k][i], squares);
                dots = __ffma2_rn(__fmul2_rn(g[k][i], w[k][i]), x[k][i], dots);
              }
            float square = squares.x + squares.y, dot = dots.x + dots.y;
            for (int i = 1; i < a.lanes; i *= 2) {
              square += __shfl_xor_sync(~0u, square, i);
              dot += __shfl_xor_sync(~0u, dot, i);
            }
            const float r = rsqrtf(fmaf(square, inv, a.eps)), back = -(r * r * dot * inv);
#pragma unroll
            for (int k = 0; k < kParts; ++k)
#pragma unroll
              for (int i = 0; i < VP; ++i) {
                const float2 n = __fmul2_rn(x[k][i], make_float2(r, r));
                dw[k][i] = __ffma2_rn(g[k][i], n, dw[k][i]);
                g[k][i] = __ffma2_rn(__fmul2_rn(g[k][i], w[k][i]), make_float2(r, r),
                                     __fmul2_rn(n, make_float2(back, back)));
              }
          }
          // zeros for a row of no sequence
          own.store(to + (int64_t)(h0 + m * per) * a.dim, h0 + m * per < count, g);
        }
      }
      if (a.parts && row) {
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
          for (int i = 0; i < VP; ++i) {
            sh.shares[which][2 * (k * VP + i)][threadIdx.x] += dw[k][i].x;
            sh.shares[which][2 * (k * VP + i) + 1][threadIdx.x] += dw[k][i].y;
          }
      }
    };
    heads(a.q.at(b, t), a.dyq.at(b, t), a.dq.at(b, t), a.heads, a.q_weight, 0);
    heads(a.k.at(b, t), a.dyk.at(b, t), a.dk.at(b, t), a.kv_heads, a.k_weight, 1);
  }
  if (!a.parts) return;
  // lanes of the same values, then warps, in a fixed order
#pragma unroll
  for (int k = 0; k < kParts; ++k)
#pragma unroll
    for (int i = 0; i < 2 * VP; ++i) {
      const int at = k * 2 * VP + i;
      float x = sh.shares[0][at][threadIdx.x], y = sh.shares[1][at][threadIdx.x];
      for (int m = a.lanes; m < 32; m *= 2) {
        x += __shfl_xor_sync(~0u, x, m);
        y += __shfl_xor_sync(~0u, y, m);
      }
      if (sub == 0 && own.has[k]) {
        sh.sums[warp][own.place(k, i / 2, i % 2)] = x;
        sh.sums[warp][a.dim + own.place(k, i / 2, i % 2)] = y;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += kThreads) {
    float x = 0.f;
    for (int w = 0; w < kWarps; ++w) x += sh.sums[w][i];
    a.parts[(int64_t)blockIdx.x * 2 * a.dim + i] = x;
  }
}

// ------------------------------------------------------------- host side
// Blocks of a call: as many as the card holds at once, so that each sums its
// shares of the weights' gradients over many rows.
int64_t blocks_of(const tcu_norm_rotate_args &a) {
  const int64_t total = (a.offsets ? 1 : (int64_t)a.sequences) * a.rows;
  return std::min<int64_t>((total + kWarps - 1) / kWarps, 2 * num_sms());
}

template <typename T, int VP, bool kInter>
int start(const tcu_norm_rotate_args &s, RotateArgs<T> a, bool grad, cudaStream_t st) {
  const int words = (s.dim / 2 + VP - 1) / VP;
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < words) a.lanes *= 2;
  const unsigned blocks = (unsigned)blocks_of(s);
  constexpr int bytes = sizeof(GradShared<VP>);
  if (!grad) {
    rotate_kernel<T, VP, kInter><<<blocks, kThreads, 0, st>>>(a);
    return launched();
  }
  if constexpr (VP <= kGradWord) {
    if (cudaFuncSetAttribute(rotate_grad_kernel<T, VP, kInter>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
      cudaGetLastError();
      return TCU_DFT_ERR_CUDA;
    }
    rotate_grad_kernel<T, VP, kInter><<<blocks, kThreads, bytes, st>>>(a);
  }
  return launched();
}

template <typename T, int VP>
int by_order(const tcu_norm_rotate_args &s, const RotateArgs<T> &a, bool grad, cudaStream_t st) {
  return s.interleaved ? start<T, VP, true>(s, a, grad, st) : start<T, VP, false>(s, a, grad, st);
}

template <typename T>
int run(const tcu_norm_rotate_args &s, bool grad, cudaStream_t st) {
  RotateArgs<T> a{};
  a.q = rows_of<const T>(s.q);
  a.k = rows_of<const T>(s.k);
  a.rates = s.rates;
  a.q_weight = s.q_weight;
  a.k_weight = s.k_weight;
  a.offsets = s.offsets;
  a.positions = s.positions;
  a.rows = s.rows;
  const int64_t batches = s.offsets ? 1 : s.sequences;
  a.total = batches * s.rows;
  a.sequences = s.sequences;
  a.heads = s.heads;
  a.kv_heads = s.kv_heads;
  a.dim = s.dim;
  a.turned = s.turned;
  a.eps = s.eps;
  const tcu_seq_rows *rows[6] = {&s.q, &s.k, &s.y_q, &s.y_k};
  int count = 4;
  if (grad) {
    a.dyq = rows_of<const T>(s.dy_q);
    a.dyk = rows_of<const T>(s.dy_k);
    a.dq = rows_of<T>(s.dq);
    a.dk = rows_of<T>(s.dk);
    a.parts = s.dq_weight || s.dk_weight ? static_cast<float *>(s.workspace) : nullptr;
    rows[2] = &s.dy_q, rows[3] = &s.dy_k, rows[4] = &s.dq, rows[5] = &s.dk;
    count = 6;
  } else {
    a.yq = rows_of<T>(s.y_q);
    a.yk = rows_of<T>(s.y_k);
  }
  int rc = TCU_DFT_OK;
  if (a.total > 0) {
    // the longest words that keep pairs of one kind together and lie aligned
    int vp = grad ? kGradWord : 16 / (int)sizeof(T);
    auto fits = [&](int n) {
      if (s.dim / 2 % n || s.turned % n) return false;
      for (int i = 0; i < count; ++i)
        if (!rows_aligned(*rows[i], s.type, batches, s.rows, n * (int)sizeof(T))) return false;
      return true;
    };
    while (vp > 1 && !fits(vp)) vp /= 2;
    switch (vp) {
      case 8:
        if constexpr (sizeof(T) == 2) rc = by_order<T, 8>(s, a, grad, st);
        break;
      case 4: rc = by_order<T, 4>(s, a, grad, st); break;
      case 2: rc = by_order<T, 2>(s, a, grad, st); break;
      default: rc = by_order<T, 1>(s, a, grad, st);
    }
  }
  if (rc || !grad) return rc;
  Sum sums[2];
  int n = 0;
  if (s.dq_weight) sums[n++] = {s.dq_weight, a.parts, s.dim};
  if (s.dk_weight) sums[n++] = {s.dk_weight, a.parts + s.dim, s.dim};
  return n ? sum_parts(sums, n, a.total > 0 ? blocks_of(s) : 0, 2 * s.dim, st) : TCU_DFT_OK;
}

int check_sizes(const tcu_norm_rotate_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->heads < 1 || a->kv_heads < 1 || a->dim < 2 || a->dim % 2 || a->turned < 1 ||
      a->turned > a->dim / 2 || !(a->eps >= 0))
    return TCU_DFT_ERR_INVALID;
  if (a->rows > kMostRows || a->dim > TCU_ATTN_MAX_NORM_DIM || a->heads > (1 << 20) ||
      a->kv_heads > (1 << 20))
    return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r : {&a->q, &a->k, &a->y_q, &a->y_k, &a->dy_q, &a->dy_k, &a->dq, &a->dk})
    if (!pitch_fits(a->rows, r->row_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  return TCU_DFT_OK;
}

bool any_rows(const tcu_norm_rotate_args &a) {
  return a.rows > 0 && a.sequences + (a.offsets != nullptr) > 0;
}

bool inputs_ok(const tcu_norm_rotate_args &a) {
  const int sz = type_size(a.type);
  return f32_ok(a.rates) && opt_ok(a.q_weight, 4) && opt_ok(a.k_weight, 4) &&
         opt_ok(a.offsets, 4) && opt_ok(a.positions, 4) && row_ok(a.q, sz) && row_ok(a.k, sz);
}

int by_type(const tcu_norm_rotate_args &a, bool grad, void *stream) {
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (a.type) {
    case TCU_SEQ_F32: return run<float>(a, grad, st);
    case TCU_SEQ_BF16: return run<bf16>(a, grad, st);
    default: return run<f16>(a, grad, st);
  }
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_norm_rotate_grad_workspace(const tcu_norm_rotate_args *a) {
  if (check_sizes(a)) return -1;
  return a->dq_weight || a->dk_weight ? blocks_of(*a) * 2 * a->dim * 4 : 0;
}

extern "C" int tcu_norm_rotate(const tcu_norm_rotate_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (!any_rows(*a)) return TCU_DFT_OK;
  const int sz = type_size(a->type);
  if (!inputs_ok(*a) || !row_ok(a->y_q, sz) || !row_ok(a->y_k, sz)) return TCU_DFT_ERR_INVALID;
  return by_type(*a, false, stream);
}

extern "C" int tcu_norm_rotate_grad(const tcu_norm_rotate_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (!opt_ok(a->dq_weight, 4) || !opt_ok(a->dk_weight, 4)) return TCU_DFT_ERR_INVALID;
  const int sz = type_size(a->type);
  if (any_rows(*a)) {
    const int64_t bytes = tcu_norm_rotate_grad_workspace(a);
    if (!inputs_ok(*a) || !row_ok(a->dy_q, sz) || !row_ok(a->dy_k, sz) || !row_ok(a->dq, sz) ||
        !row_ok(a->dk, sz) || a->workspace_bytes < bytes || (bytes && !f32_ok(a->workspace)))
      return TCU_DFT_ERR_INVALID;
  }
  return by_type(*a, true, stream);
}
