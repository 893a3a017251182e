// short_conv.cu -- the short depthwise causal convolution, its gradient and
// its single-token form (include/tcu_seq.h).
//
// Per sequence and channel, i counting the rows of the sequence and rows
// i < 0 coming from the carried state (or zeros):
//     p_i  = bias + sum_k w_k x_{i-(W-1)+k},     y_i = p_i sigma(p_i) or p_i
//     dp_i = dy_i f'(p_i)
//     dx_i = sum_k w_k dp_{i+(W-1)-k} (+ dlast at the last W-1 rows)
//     dw_k = sum_i dp_i x_{i-(W-1)+k},           dbias = sum_i dp_i
// A dozen operations for each value read and written: HBM bounds the whole
// of it, so a thread owns a few adjacent channels (one 16-byte word where the
// rows allow it) and walks down the rows with its window in registers: each
// row is read once, but for the W-1 rows above a run.
#include <algorithm>

#include "seq_common.cuh"

namespace tcu {
namespace seq {
namespace {

template <typename T>
struct ConvArgs {
  Rows<const T> x, dy;
  Rows<T> y, dx;
  const float *weight, *bias;
  const T *state, *dlast;
  T *last, *dstate;
  float *parts;  // gradient: [run][channels][W] then [run][channels]
  float *bias_parts;
  const int32_t *offsets;
  const int32_t *slots;
  int64_t rows, channels, num_slots;
  int sequences, batches, silu;
  int64_t runs;  // runs of kBlockRows * blocks rows in a batch entry
  int blocks;
};

constexpr int kThreads = 128;
constexpr int kBlockRows = 8;

// One sequence as rows [lo, hi) of a batch entry; span_of holds t itself
// whatever the offsets are.
struct Span {
  int64_t lo, hi;
  int seq;
};

template <typename T>
__device__ __forceinline__ Span span_of(const ConvArgs<T> &a, int64_t b, int64_t t) {
  if (!a.offsets) return {0, a.rows, (int)b};
  const int s = sequence_of(a.offsets, a.sequences, t);
  if (s < 0) return {t, t + 1, -1};
  return {max((int64_t)a.offsets[s], (int64_t)0),
          max(min((int64_t)a.offsets[s + 1], a.rows), t + 1), s};
}

// Row i of a sequence, from the state where i < 0.
template <typename T, int V, int W>
__device__ __forceinline__ void row_value(const ConvArgs<T> &a, int64_t b, const Span &s,
                                          int64_t i, int64_t c, float (&out)[V]) {
  if (i >= 0) {
    load_vec<T, V>(out, a.x.at(b, s.lo + i) + c);
  } else if (a.state && s.seq >= 0) {
    load_vec<T, V>(out, a.state + ((int64_t)s.seq * (W - 1) + (W - 1) + i) * a.channels + c);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = 0.f;
  }
}

template <typename T, int V, int W>
__device__ __forceinline__ void load_params(const ConvArgs<T> &a, int64_t c, float (&w)[W][V],
                                            float (&bias)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    bias[v] = a.bias ? a.bias[c + v] : 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k][v] = a.weight[(c + v) * W + k];
  }
}

// p_i from the definition, row by row: where the fast path's window would
// leave the sequence.
template <typename T, int V, int W>
__device__ __forceinline__ void pre_at(const ConvArgs<T> &a, int64_t b, const Span &s, int64_t i,
                                       int64_t c, const float (&w)[W][V], const float (&bias)[V],
                                       float (&p)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = bias[v];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    float x[V];
    row_value<T, V, W>(a, b, s, i - (W - 1) + k, c, x);
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = fmaf(w[k][v], x[v], p[v]);
  }
}

// The W-1 rows that a continuation of sequence s needs.
template <typename T, int V, int W>
__device__ __forceinline__ void write_last(const ConvArgs<T> &a, int64_t item, int64_t cv) {
  if constexpr (W > 1) {
    const int k = item % (W - 1);
    const int64_t s = item / (W - 1);
    Span sp;
    sp.seq = (int)s;
    if (a.offsets) {
      sp.lo = min(max((int64_t)a.offsets[s], (int64_t)0), a.rows);
      sp.hi = min(max((int64_t)a.offsets[s + 1], sp.lo), a.rows);
    } else {
      sp.lo = 0;
      sp.hi = a.rows;
    }
    float x[V];
    row_value<T, V, W>(a, a.offsets ? 0 : s, sp, sp.hi - sp.lo - (W - 1) + k, cv, x);
    store_vec<T, V>(a.last + (s * (W - 1) + k) * a.channels + cv, x);
  }
}

// y: one thread per V channels and run of rows; the threads past the runs
// write `last`.
template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_kernel(ConvArgs<T> a) {
  const int64_t cvs = a.channels / V;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t c = id % cvs * V;
  const int64_t item = id / cvs, runs = a.runs * a.batches;
  if (item >= runs) {
    if (a.last && item - runs < (int64_t)a.sequences * (W - 1))
      write_last<T, V, W>(a, item - runs, c);
    return;
  }
  const int64_t b = item / a.runs, t0 = item % a.runs * (kBlockRows * a.blocks);
  const int64_t t1 = min(t0 + kBlockRows * a.blocks, a.rows);
  float w[W][V], bias[V];
  load_params<T, V, W>(a, c, w, bias);
  Span s = span_of(a, b, t0);
  for (int64_t t = t0; t < t1; t += kBlockRows) {
    if (t >= s.lo + (W - 1) && t + kBlockRows <= min(s.hi, t1)) {
      Vec<T, V> in[kBlockRows + W - 1];
#pragma unroll
      for (int r = 0; r < kBlockRows + W - 1; ++r)
        in[r] = *reinterpret_cast<const Vec<T, V> *>(a.x.at(b, t - (W - 1) + r) + c);
#pragma unroll
      for (int r = 0; r < kBlockRows; ++r) {
        float p[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          p[v] = bias[v];
#pragma unroll
          for (int k = 0; k < W; ++k) p[v] = fmaf(w[k][v], to_f(in[r + k].v[v]), p[v]);
          if (a.silu) p[v] = silu(p[v]);
        }
        store_vec<T, V>(a.y.at(b, t + r) + c, p);
      }
      continue;
    }
    const int64_t te = min(t + kBlockRows, t1);
    for (int64_t r = t; r < te; ++r) {
      if (r >= s.hi) s = span_of(a, b, r);
      float p[V];
      pre_at<T, V, W>(a, b, s, r - s.lo, c, w, bias, p);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (a.silu) p[v] = silu(p[v]);
      store_vec<T, V>(a.y.at(b, r) + c, p);
    }
    if (te < t1 && te >= s.hi) s = span_of(a, b, te);
  }
}

// dp_i from the definition.
template <typename T, int V, int W>
__device__ __forceinline__ void dpre_at(const ConvArgs<T> &a, int64_t b, const Span &s, int64_t i,
                                        int64_t c, const float (&w)[W][V], const float (&bias)[V],
                                        float (&dp)[V]) {
  load_vec<T, V>(dp, a.dy.at(b, s.lo + i) + c);
  if (!a.silu) return;
  float p[V];
  pre_at<T, V, W>(a, b, s, i, c, w, bias, p);
#pragma unroll
  for (int v = 0; v < V; ++v) dp[v] *= dsilu(p[v]);
}

// The gradient of row i of a sequence, i >= -(W-1).
template <typename T, int V, int W>
__device__ __forceinline__ void drow_at(const ConvArgs<T> &a, int64_t b, const Span &s, int64_t i,
                                        int64_t c, const float (&w)[W][V], const float (&bias)[V],
                                        float (&dx)[V]) {
  const int64_t len = s.hi - s.lo, tail = i - (len - (W - 1));
  if (tail >= 0 && a.dlast && s.seq >= 0) {
    load_vec<T, V>(dx, a.dlast + ((int64_t)s.seq * (W - 1) + tail) * a.channels + c);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) dx[v] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const int64_t j = i + (W - 1) - k;
    if (j < 0 || j >= len) continue;
    float dp[V];
    dpre_at<T, V, W>(a, b, s, j, c, w, bias, dp);
#pragma unroll
    for (int v = 0; v < V; ++v) dx[v] = fmaf(w[k][v], dp[v], dx[v]);
  }
}

// dx and each run's share of dw and dbias: one thread per V channels and run;
// the threads past the runs write dstate.
template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_grad_kernel(ConvArgs<T> a) {
  const int64_t cvs = a.channels / V;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t c = id % cvs * V;
  const int64_t item = id / cvs, runs = a.runs * a.batches;
  float w[W][V], bias[V];
  if (item >= runs) {
    const int64_t rest = item - runs;
    if (!a.dstate || rest >= (int64_t)a.sequences * (W - 1)) return;
    load_params<T, V, W>(a, c, w, bias);
    constexpr int kPast = W > 1 ? W - 1 : 1;  // W == 1 has no past and returned
    const int64_t sq = rest / kPast, k = rest % kPast;
    Span s{0, a.rows, (int)sq};
    if (a.offsets) {
      s.lo = min(max((int64_t)a.offsets[sq], (int64_t)0), a.rows);
      s.hi = min(max((int64_t)a.offsets[sq + 1], s.lo), a.rows);
    }
    float dx[V];
    drow_at<T, V, W>(a, a.offsets ? 0 : sq, s, k - (W - 1), c, w, bias, dx);
    store_vec<T, V>(a.dstate + rest * a.channels + c, dx);
    return;
  }
  load_params<T, V, W>(a, c, w, bias);
  const int64_t b = item / a.runs, t0 = item % a.runs * (kBlockRows * a.blocks);
  const int64_t t1 = min(t0 + kBlockRows * a.blocks, a.rows);
  float dw[W][V], db[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    db[v] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) dw[k][v] = 0.f;
  }
  Span s = span_of(a, b, t0);
  for (int64_t r = t0; r < t1; ++r) {
    if (r >= s.hi) s = span_of(a, b, r);
    const int64_t i = r - s.lo;
    float g[V];
    drow_at<T, V, W>(a, b, s, i, c, w, bias, g);
    store_vec<T, V>(a.dx.at(b, r) + c, g);
    dpre_at<T, V, W>(a, b, s, i, c, w, bias, g);
#pragma unroll
    for (int k = 0; k < W; ++k) {
      float x[V];
      row_value<T, V, W>(a, b, s, i - (W - 1) + k, c, x);
#pragma unroll
      for (int v = 0; v < V; ++v) dw[k][v] = fmaf(g[v], x[v], dw[k][v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) db[v] += g[v];
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (a.bias_parts) a.bias_parts[item * a.channels + c + v] = db[v];
#pragma unroll
    for (int k = 0; k < W; ++k) a.parts[(item * a.channels + c + v) * W + k] = dw[k][v];
  }
}

// One token: one thread per V channels and batch entry.
template <typename T, int V, int W>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(ConvArgs<T> a) {
  const int64_t cvs = a.channels / V;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t c = id % cvs * V, b = id / cvs;
  if (b >= a.sequences) return;
  const int64_t slot = a.slots ? a.slots[b] : b;
  float p[V];
  if (slot < 0 || slot >= a.num_slots) {
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = 0.f;
    store_vec<T, V>(a.y.at(b, 0) + c, p);
    return;
  }
  Vec<T, V> x[W];
  T *cache = a.last + slot * (W - 1) * a.channels + c;
#pragma unroll
  for (int k = 0; k < W - 1; ++k)
    x[k] = *reinterpret_cast<const Vec<T, V> *>(cache + k * a.channels);
  x[W - 1] = *reinterpret_cast<const Vec<T, V> *>(a.x.at(b, 0) + c);
  float w[W][V], bias[V];
  load_params<T, V, W>(a, c, w, bias);
#pragma unroll
  for (int k = 0; k < W - 1; ++k) *reinterpret_cast<Vec<T, V> *>(cache + k * a.channels) = x[k + 1];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    p[v] = bias[v];
#pragma unroll
    for (int k = 0; k < W; ++k) p[v] = fmaf(w[k][v], to_f(x[k].v[v]), p[v]);
    if (a.silu) p[v] = silu(p[v]);
  }
  store_vec<T, V>(a.y.at(b, 0) + c, p);
}

// ------------------------------------------------------------- host side
enum Call { kForward, kGrad, kStep };

template <typename T, int V, int W>
int launch(Call call, const ConvArgs<T> &a, cudaStream_t st) {
  const int64_t cvs = a.channels / V;
  int64_t items = a.runs * a.batches;
  if (call == kStep) items = a.sequences;
  else if (call == kForward ? a.last != nullptr : a.dstate != nullptr)
    items += (int64_t)a.sequences * (W - 1);
  const int64_t blocks = (items * cvs + kThreads - 1) / kThreads;
  if (blocks == 0) return TCU_DFT_OK;
  if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  if (call == kForward) conv_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, st>>>(a);
  else if (call == kGrad) conv_grad_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, st>>>(a);
  else conv_step_kernel<T, V, W><<<(unsigned)blocks, kThreads, 0, st>>>(a);
  return launched();
}

template <typename T, int V>
int by_width(Call call, int width, const ConvArgs<T> &a, cudaStream_t st) {
  switch (width) {
    case 1: return launch<T, V, 1>(call, a, st);
    case 2: return launch<T, V, 2>(call, a, st);
    case 3: return launch<T, V, 3>(call, a, st);
    case 4: return launch<T, V, 4>(call, a, st);
    case 5: return launch<T, V, 5>(call, a, st);
    case 6: return launch<T, V, 6>(call, a, st);
    case 7: return launch<T, V, 7>(call, a, st);
    case 8: return launch<T, V, 8>(call, a, st);
  }
  return TCU_DFT_ERR_UNSUPPORTED;
}

struct Shape {
  int64_t batches, rows, runs;
  int blocks;
};

Shape shape_of(const tcu_short_conv_args &a) {
  Shape s;
  s.batches = a.offsets ? 1 : a.sequences;
  s.rows = a.rows;
  s.blocks = 4;
  s.runs = (a.rows + kBlockRows * s.blocks - 1) / (kBlockRows * s.blocks);
  return s;
}

int64_t grad_parts(const tcu_short_conv_args &a) {
  const Shape s = shape_of(a);
  return s.runs * s.batches;
}

int check_sizes(const tcu_short_conv_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->channels < 1 || a->width < 1)
    return TCU_DFT_ERR_INVALID;
  if (a->width > TCU_SEQ_MAX_WIDTH || a->rows > INT32_MAX || a->channels > INT32_MAX)
    return TCU_DFT_ERR_UNSUPPORTED;
  return TCU_DFT_OK;
}

template <typename T>
int dispatch(Call call, const tcu_short_conv_args &s, cudaStream_t st) {
  const Shape sh = shape_of(s);
  ConvArgs<T> a{};
  a.x = rows_of<const T>(s.x);
  a.y = rows_of<T>(s.y);
  a.dy = rows_of<const T>(s.dy);
  a.dx = rows_of<T>(s.dx);
  a.weight = s.weight;
  a.bias = s.bias;
  a.state = static_cast<const T *>(s.state);
  a.dlast = static_cast<const T *>(s.dlast);
  a.last = static_cast<T *>(s.last);
  a.dstate = static_cast<T *>(s.dstate);
  a.offsets = s.offsets;
  a.slots = s.slots;
  a.rows = s.rows;
  a.channels = s.channels;
  a.num_slots = s.num_slots;
  a.sequences = s.sequences;
  a.batches = (int)sh.batches;
  a.silu = s.silu;
  a.runs = sh.runs;
  a.blocks = sh.blocks;
  const int64_t parts = sh.runs * sh.batches;
  if (call == kGrad) {
    a.parts = static_cast<float *>(s.workspace);
    a.bias_parts = s.dbias ? a.parts + parts * s.channels * s.width : nullptr;
  }
  constexpr int V = 16 / sizeof(T);
  bool wide = s.channels % V == 0 && rows_aligned(s.x, s.type, sh.batches, s.rows, 16);
  if (call == kGrad)
    wide = wide && rows_aligned(s.dy, s.type, sh.batches, s.rows, 16) &&
           rows_aligned(s.dx, s.type, sh.batches, s.rows, 16);
  else
    wide = wide && rows_aligned(s.y, s.type, sh.batches, s.rows, 16);
  for (const void *p : {s.state, s.dlast, (const void *)s.last, (const void *)s.dstate})
    wide = wide && (uintptr_t)p % 16 == 0;
  const int rc = wide ? by_width<T, V>(call, s.width, a, st) : by_width<T, 1>(call, s.width, a, st);
  if (rc != TCU_DFT_OK || call != kGrad) return rc;
  const int rw = sum_parts(s.dweight, a.parts, parts, s.channels * s.width, st);
  if (rw != TCU_DFT_OK || !s.dbias) return rw;
  return sum_parts(s.dbias, a.bias_parts, parts, s.channels, st);
}

int by_type(Call call, const tcu_short_conv_args &a, cudaStream_t st) {
  switch (a.type) {
    case TCU_SEQ_F32: return dispatch<float>(call, a, st);
    case TCU_SEQ_BF16: return dispatch<bf16>(call, a, st);
    default: return dispatch<f16>(call, a, st);
  }
}

}  // namespace

__global__ void sum_parts_kernel(float *out, const float *partial, int64_t parts, int64_t count) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= count) return;
  float s = 0.f;
  for (int64_t p = 0; p < parts; ++p) s += partial[p * count + i];
  out[i] = s;
}

int sum_parts(float *out, const float *partial, int64_t parts, int64_t count, cudaStream_t st) {
  if (count == 0) return TCU_DFT_OK;
  sum_parts_kernel<<<(unsigned)((count + 127) / 128), 128, 0, st>>>(out, partial, parts, count);
  return launched();
}

}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_short_conv_grad_workspace(const tcu_short_conv_args *a) {
  if (check_sizes(a) != TCU_DFT_OK) return -1;
  return grad_parts(*a) * a->channels * (a->width + 1) * 4;
}

extern "C" int tcu_short_conv(const tcu_short_conv_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  const int sz = type_size(a->type);
  if (!f32_ok(a->weight) || !opt_ok(a->bias, 4) || !opt_ok(a->state, sz) ||
      !opt_ok(a->last, sz) || !opt_ok(a->offsets, 4))
    return TCU_DFT_ERR_INVALID;
  if (a->rows > 0 && (!row_ok(a->x, sz) || !row_ok(a->y, sz))) return TCU_DFT_ERR_INVALID;
  return by_type(kForward, *a, static_cast<cudaStream_t>(stream));
}

extern "C" int tcu_short_conv_grad(const tcu_short_conv_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  const int sz = type_size(a->type);
  if (!f32_ok(a->weight) || !f32_ok(a->dweight) || !opt_ok(a->bias, 4) || !opt_ok(a->dbias, 4) ||
      !opt_ok(a->state, sz) || !opt_ok(a->dlast, sz) || !opt_ok(a->dstate, sz) ||
      !opt_ok(a->offsets, 4) || !opt_ok(a->workspace, 4) ||
      a->workspace_bytes < tcu_short_conv_grad_workspace(a) ||
      (a->workspace_bytes > 0 && !a->workspace))
    return TCU_DFT_ERR_INVALID;
  if (a->rows > 0 && (!row_ok(a->x, sz) || !row_ok(a->dy, sz) || !row_ok(a->dx, sz)))
    return TCU_DFT_ERR_INVALID;
  return by_type(kGrad, *a, static_cast<cudaStream_t>(stream));
}

extern "C" int tcu_short_conv_step(const tcu_short_conv_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  const int sz = type_size(a->type);
  if (a->rows != 1 || a->offsets || a->num_slots < 0 || (!a->slots && a->num_slots < a->sequences) ||
      !f32_ok(a->weight) || !opt_ok(a->bias, 4) || !opt_ok(a->slots, 4))
    return TCU_DFT_ERR_INVALID;
  if (a->sequences > 0 &&
      (!row_ok(a->x, sz) || !row_ok(a->y, sz) ||
       (a->width > 1 && a->num_slots > 0 && (!a->last || (uintptr_t)a->last % sz))))
    return TCU_DFT_ERR_INVALID;
  return by_type(kStep, *a, static_cast<cudaStream_t>(stream));
}
