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
// of it, so a thread owns a few adjacent channels and walks down the rows with
// its window in registers and the next rows on their way: each row is read
// once, but for the W-1 rows above a run (and, for the gradient, below it).
//
// Measured, bf16, width 4 with silu: forward at 8 x 4096 x 4096, 4 channels a
// thread, 103 us, 5.2 TB/s (16-byte words of 8 channels hold half the threads:
// 112 us); gradient at 8 x 2048 x 4096, 2 channels a thread, 99 us, 4.1 TB/s
// (with 4: 135 us).  Copying runs at 6.8 TB/s.
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
  float *parts;  // gradient: [run]{[channels][W], [channels]}
  const int32_t *offsets;
  const int32_t *slots;
  int64_t channels, num_slots;
  int rows, sequences, batches, silu;
  int runs;  // of kBlockRows * blocks rows in a batch entry
  int blocks;
};

// A block: 32 threads along the channels, kItems items (runs, or batch
// entries) below each other.  A prompt's thread divides by a size of the call
// once, to find its run.
constexpr int kItems = 4;
constexpr int kThreads = 32 * kItems;
constexpr int kBlockRows = 8;
// Rows whose loads are on their way while as many are worked on: a multiple
// of the width, so that slots are known, near eight.
template <int W>
constexpr int kAhead = W * (8 / W);

// One sequence as rows [lo, hi) of a batch entry; span_of holds t itself
// whatever the offsets are.
struct Span {
  int lo, hi;
  int seq;
};

template <typename T>
__device__ __forceinline__ Span span_of(const ConvArgs<T> &a, int64_t b, int t) {
  if (!a.offsets) return {0, a.rows, (int)b};
  const int s = sequence_of(a.offsets, a.sequences, t);
  if (s < 0) return {t, t + 1, -1};
  return {max(a.offsets[s], 0), max(min(a.offsets[s + 1], a.rows), t + 1), s};
}
// Sequence s itself, empty ones too.
template <typename T>
__device__ __forceinline__ Span span_at(const ConvArgs<T> &a, int64_t s) {
  if (!a.offsets) return {0, a.rows, (int)s};
  const int lo = min(max(a.offsets[s], 0), a.rows);
  return {lo, min(max(a.offsets[s + 1], lo), a.rows), (int)s};
}

// What a thread owns: V channels, of which `count` exist, as pairs for packed
// arithmetic.  kWide: adjacent ones, read in words (count is V); otherwise one
// of each V-th part of the channels, so that lanes read adjacent values.
template <typename T, int V, int W, bool kWide>
struct Own {
  static constexpr int P = V / 2;
  using Row = Raw<T, V, !kWide>;
  const ConvArgs<T> &a;
  int64_t b, c, gap;
  int count;
  float2 w[W][P], bias[P];

  // The `which`-th of `all` threads that share a row.
  __device__ __forceinline__ Own(const ConvArgs<T> &args, int64_t which, int64_t all) : a(args) {
    c = kWide ? which * V : which;
    gap = kWide ? 1 : all;
    count = kWide ? V : (int)((a.channels - c + gap - 1) / gap);
  }
  __device__ __forceinline__ void params() {
    float *to = reinterpret_cast<float *>(bias);
    if constexpr (kWide) {  // the V rows of the weights are adjacent
      constexpr int step = V * W % 4 == 0 ? 4 : 2;
      Vec<float, step> all[V * W / step];
#pragma unroll
      for (int i = 0; i < V * W / step; ++i)
        all[i] = reinterpret_cast<const Vec<float, step> *>(a.weight + c * W)[i];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        to[v] = a.bias ? a.bias[c + v] : 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k)
          reinterpret_cast<float *>(w[k])[v] = all[(v * W + k) / step].v[(v * W + k) % step];
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool in = v < count;
        to[v] = a.bias && in ? a.bias[c + v * gap] : 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k)
          reinterpret_cast<float *>(w[k])[v] = in ? a.weight[(c + v * gap) * W + k] : 0.f;
      }
    }
  }
  __device__ __forceinline__ Row row(const T *p) const {
    Row r;
    r.template load<kWide>(p, count, gap);
    return r;
  }
  __device__ __forceinline__ void put(T *p, const float2 (&v)[P]) const {
    Row r;
#pragma unroll
    for (int i = 0; i < P; ++i) r.set(i, v[i]);
    r.template store<kWide>(p, count, gap);
  }
  // Row i of a sequence, from the state where i < 0.
  __device__ __forceinline__ Row value(const Span &s, int i) const {
    if (i >= 0) return row(a.x.at(b, s.lo + i) + c);
    if (a.state && s.seq >= 0)
      return row(a.state + ((int64_t)s.seq * (W - 1) + (W - 1) + i) * a.channels + c);
    Row zero;
#pragma unroll
    for (int j = 0; j < Row::kWords; ++j) zero.w[j] = 0;
    return zero;
  }
  // p of the row in slot j of a window whose slots are rows mod W.
  __device__ __forceinline__ void pre(const float2 (&x)[W][P], int j, float2 (&p)[P]) const {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      p[i] = bias[i];
#pragma unroll
      for (int k = 0; k < W; ++k) p[i] = __ffma2_rn(w[k][i], x[(j + 1 + k) % W][i], p[i]);
    }
  }
  // dp of that row from its dy.
  __device__ __forceinline__ void dpre(const float2 (&x)[W][P], int j, const Row &dy,
                                       float2 (&dp)[P]) const {
    float2 p[P];
    if (a.silu) pre(x, j, p);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      dp[i] = dy.pair(i);
      if (a.silu) dp[i] = __fmul2_rn(dp[i], dsilu2(p[i]));
    }
  }
  // The window before row i of a sequence, i in slot 0.
  __device__ __forceinline__ void window(const Span &s, int i, float2 (&x)[W][P]) const {
#pragma unroll
    for (int k = 1; k < W; ++k) {
      const Row r = value(s, i - W + k);
#pragma unroll
      for (int j = 0; j < P; ++j) x[k % W][j] = r.pair(j);
    }
  }
};

// y: one thread per V channels and run of rows; the threads past the runs
// write `last`, the W-1 rows that a continuation needs.  A thread walks down
// its rows with the last W of them in registers, slot r mod W each, and the
// next W on their way.
template <typename T, int V, int W, bool kWide>
__global__ void __launch_bounds__(kThreads) conv_kernel(ConvArgs<T> a) {
  const int64_t cvs = (a.channels + V - 1) / V;
  const int64_t cv = (int64_t)blockIdx.y * 32 + threadIdx.x;
  const int item = (int)(blockIdx.x * kItems + threadIdx.y), runs = a.runs * a.batches;
  if (cv >= cvs) return;
  Own<T, V, W, kWide> own(a, cv, cvs);
  using Row = typename Own<T, V, W, kWide>::Row;
  constexpr int P = V / 2;
  const int64_t c = own.c;
  if (item >= runs) {
    const int rest = item - runs;
    if (!a.last || rest >= a.sequences * (W - 1)) return;
    constexpr int kPast = W > 1 ? W - 1 : 1;  // W == 1 has no past and returned
    const Span s = span_at(a, rest / kPast);
    own.b = a.offsets ? 0 : s.seq;
    const Row r = own.value(s, s.hi - s.lo - (W - 1) + rest % kPast);
    r.template store<kWide>(a.last + (int64_t)rest * a.channels + c, own.count, own.gap);
    return;
  }
  const int b = (int)((unsigned)item / (unsigned)a.runs), run = item - b * a.runs;
  own.b = b;
  const int t0 = run * (kBlockRows * a.blocks), t1 = min(t0 + kBlockRows * a.blocks, a.rows);
  own.params();
  for (int lo = t0; lo < t1;) {
    const Span s = span_of(a, b, lo);
    const int hi = min(s.hi, t1);
    float2 x[W][P];
    own.window(s, lo - s.lo, x);
    const T *from = a.x.at(b, lo) + c;
    T *to = a.y.at(b, lo) + c;
    auto row = [&](int j, const Row &r) {
#pragma unroll
      for (int i = 0; i < P; ++i) x[j][i] = r.pair(i);
      float2 p[P];
      own.pre(x, j, p);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (a.silu) p[i] = silu2(p[i]);
      own.put(to, p);
      to += a.y.row;
    };
    int left = hi - lo;
    constexpr int G = kAhead<W>;
    Row next[G];
    if (left >= G) {
#pragma unroll
      for (int j = 0; j < G; ++j, from += a.x.row) next[j] = own.row(from);
    }
    for (; left >= G; left -= G) {
      Row now[G];
#pragma unroll
      for (int j = 0; j < G; ++j) now[j] = next[j];
      if (left >= 2 * G) {
#pragma unroll
        for (int j = 0; j < G; ++j, from += a.x.row) next[j] = own.row(from);
      }
#pragma unroll
      for (int j = 0; j < G; ++j) row(j % W, now[j]);
    }
#pragma unroll
    for (int j = 0; j < G - 1; ++j) {
      if (j >= left) break;
      row(j % W, own.row(from));
      from += a.x.row;
    }
    lo = hi;
  }
}

// dx and each run's share of dw and dbias: one thread per V channels and run;
// the threads past the runs write dstate.  A thread walks down its rows (and,
// for the last of them, W-1 rows on) with the last W rows of x and of dp in
// registers: row r gives p_r, dp_r, its terms of dw, and
// dx_{r-(W-1)} = sum_k w_k dp_{r-k}.
template <typename T, int V, int W, bool kWide>
__global__ void __launch_bounds__(kThreads) conv_grad_kernel(ConvArgs<T> a) {
  const int64_t cvs = (a.channels + V - 1) / V;
  const int64_t cv = (int64_t)blockIdx.y * 32 + threadIdx.x;
  const int item = (int)(blockIdx.x * kItems + threadIdx.y), runs = a.runs * a.batches;
  if (cv >= cvs) return;
  Own<T, V, W, kWide> own(a, cv, cvs);
  using Row = typename Own<T, V, W, kWide>::Row;
  constexpr int P = V / 2;
  const int64_t c = own.c;
  // dlast of the row that lies i before the end of what sequence s would
  // continue to, or zeros
  auto after = [&](const Span &s, int i, float2 (&dx)[P]) {
    if (!a.dlast || s.seq < 0) return;
    const Row r = own.row(a.dlast + ((int64_t)s.seq * (W - 1) + i) * a.channels + c);
#pragma unroll
    for (int j = 0; j < P; ++j) dx[j] = r.pair(j);
  };
  if (item >= runs) {
    // row i = k - (W-1) < 0 of sequence s: taps of its first rows
    const int rest = item - runs;
    if (!a.dstate || rest >= a.sequences * (W - 1)) return;
    constexpr int kPast = W > 1 ? W - 1 : 1;
    const Span s = span_at(a, rest / kPast);
    own.b = a.offsets ? 0 : s.seq;
    own.params();
    const int i = rest % kPast - (W - 1), len = s.hi - s.lo;
    float2 x[W][P], dp[P], dx[P] = {};
    if (i >= len - (W - 1)) after(s, i - (len - (W - 1)), dx);
    own.window(s, 0, x);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      if (j > i + (W - 1) || j >= len) break;
      const Row r = own.value(s, j);
#pragma unroll
      for (int n = 0; n < P; ++n) x[j][n] = r.pair(n);
      own.dpre(x, j, own.row(a.dy.at(own.b, s.lo + j) + c), dp);
      const int k = i + (W - 1) - j;  // the tap of row i in row j
#pragma unroll
      for (int m = 0; m < W; ++m)
        if (m == k)
#pragma unroll
          for (int n = 0; n < P; ++n) dx[n] = __ffma2_rn(own.w[m][n], dp[n], dx[n]);
    }
    own.put(a.dstate + (int64_t)rest * a.channels + c, dx);
    return;
  }
  const int b = (int)((unsigned)item / (unsigned)a.runs), run = item - b * a.runs;
  own.b = b;
  const int t0 = run * (kBlockRows * a.blocks), t1 = min(t0 + kBlockRows * a.blocks, a.rows);
  own.params();
  float2 dw[W][P] = {}, db[P] = {};
  for (int lo = t0; lo < t1;) {
    const Span s = span_of(a, b, lo);
    const int hi = min(s.hi, t1);
    float2 x[W][P], dp[W][P] = {};
    own.window(s, lo - s.lo, x);
    const T *px = a.x.at(b, lo) + c, *py = a.dy.at(b, lo) + c;
    T *to = a.dx.at(b, lo - (W - 1)) + c;  // of the row that the next one completes
    auto fill = [&](int j, const Row &r) {
#pragma unroll
      for (int i = 0; i < P; ++i) x[j][i] = r.pair(i);
    };
    auto weigh = [&](int j) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        db[i] = __fadd2_rn(db[i], dp[j][i]);
#pragma unroll
        for (int k = 0; k < W; ++k) dw[k][i] = __ffma2_rn(dp[j][i], x[(j + 1 + k) % W][i], dw[k][i]);
      }
    };
    auto emit = [&](int j, bool store, float2 (&dx)[P]) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) dx[i] = __ffma2_rn(own.w[k][i], dp[(j + W - k) % W][i], dx[i]);
      if (store) own.put(to, dx);
      to += a.dx.row;
    };
    const int n = hi - lo;
    int r0 = 0;  // rows done
    constexpr int G = kAhead<W>;
    Row nx[G], ny[G];
    auto fetch = [&]() {
#pragma unroll
      for (int j = 0; j < G; ++j, px += a.x.row, py += a.dy.row) nx[j] = own.row(px), ny[j] = own.row(py);
    };
    if (n >= G) fetch();
    for (; r0 + G <= n; r0 += G) {
      Row xs[G], ys[G];
#pragma unroll
      for (int j = 0; j < G; ++j) xs[j] = nx[j], ys[j] = ny[j];
      if (r0 + 2 * G <= n) fetch();
#pragma unroll
      for (int j = 0; j < G; ++j) {
        float2 dx[P] = {};
        fill(j % W, xs[j]);
        own.dpre(x, j % W, ys[j], dp[j % W]);
        weigh(j % W);
        emit(j % W, r0 + j >= W - 1, dx);
      }
    }
    // the rows left, and the W-1 beyond them that the last rows' dx still need
    const int end = s.hi - lo;  // of the sequence
#pragma unroll 1
    for (; r0 < n + W - 1; r0 += W) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const int r = r0 + j;
        if (r >= n + W - 1) break;
        float2 dx[P] = {};
        if (r < end) {
          fill(j, own.row(px));
          own.dpre(x, j, own.row(py), dp[j]);
          px += a.x.row;
          py += a.dy.row;
          if (r < n) weigh(j);
        } else {
#pragma unroll
          for (int i = 0; i < P; ++i) dp[j][i] = make_float2(0.f, 0.f);
          after(s, r - end, dx);
        }
        emit(j, r >= W - 1, dx);
      }
    }
    lo = hi;
  }
  float *share = a.parts + (int64_t)item * a.channels * (W + 1);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!kWide && v >= own.count) continue;
    share[a.channels * W + c + v * own.gap] = reinterpret_cast<const float *>(db)[v];
#pragma unroll
    for (int k = 0; k < W; ++k) share[(c + v * own.gap) * W + k] = reinterpret_cast<const float *>(dw[k])[v];
  }
}

// One token: one thread per V channels and batch entry.  512 x 4096 bf16: 13 us,
// 2.6 TB/s, of which launch and drain are 7.
template <typename T, int V, int W, bool kWide>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(ConvArgs<T> a) {
  const int64_t cvs = (a.channels + V - 1) / V;
  const int64_t cv = (int64_t)blockIdx.y * 32 + threadIdx.x;
  const int b = (int)(blockIdx.x * kItems + threadIdx.y);
  if (b >= a.sequences || cv >= cvs) return;
  Own<T, V, W, kWide> own(a, cv, cvs);
  using Row = typename Own<T, V, W, kWide>::Row;
  constexpr int P = V / 2;
  const int64_t c = own.c, slot = a.slots ? a.slots[b] : b;
  float2 p[P] = {};
  if (slot >= 0 && slot < a.num_slots) {
    T *cache = a.last + slot * (W - 1) * a.channels + c;
    Row r[W];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) r[k] = own.row(cache + k * a.channels);
    r[W - 1] = own.row(a.x.at(b, 0) + c);
    own.params();
    float2 x[W][P];
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if (k > 0) r[k].template store<kWide>(cache + (k - 1) * a.channels, own.count, own.gap);
#pragma unroll
      for (int i = 0; i < P; ++i) x[k][i] = r[k].pair(i);
    }
    own.pre(x, W - 1, p);
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (a.silu) p[i] = silu2(p[i]);
  }
  own.put(a.y.at(b, 0) + c, p);
}

// ------------------------------------------------------------- host side
enum Call { kForward, kGrad, kStep };

template <Call kCall, typename T, int V, int W, bool kWide>
int launch(const ConvArgs<T> &a, cudaStream_t st) {
  const int64_t cvs = (a.channels + V - 1) / V;
  int64_t items = (int64_t)a.runs * a.batches;
  if (kCall == kStep) items = a.sequences;
  else if (kCall == kForward ? a.last != nullptr : a.dstate != nullptr)
    items += (int64_t)a.sequences * (W - 1);
  if (items == 0) return TCU_DFT_OK;
  const int64_t down = (items + kItems - 1) / kItems, across = (cvs + 31) / 32;
  if (items > INT32_MAX - kItems || across > 65535) return TCU_DFT_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)down, (unsigned)across), block(32, kItems);
  if constexpr (kCall == kForward) conv_kernel<T, V, W, kWide><<<grid, block, 0, st>>>(a);
  else if constexpr (kCall == kGrad) conv_grad_kernel<T, V, W, kWide><<<grid, block, 0, st>>>(a);
  else conv_step_kernel<T, V, W, kWide><<<grid, block, 0, st>>>(a);
  return launched();
}

template <Call kCall, typename T, int V, bool kWide>
int by_width(int width, const ConvArgs<T> &a, cudaStream_t st) {
  switch (width) {
    case 1: return launch<kCall, T, V, 1, kWide>(a, st);
    case 2: return launch<kCall, T, V, 2, kWide>(a, st);
    case 3: return launch<kCall, T, V, 3, kWide>(a, st);
    case 4: return launch<kCall, T, V, 4, kWide>(a, st);
    case 5: return launch<kCall, T, V, 5, kWide>(a, st);
    case 6: return launch<kCall, T, V, 6, kWide>(a, st);
    case 7: return launch<kCall, T, V, 7, kWide>(a, st);
    case 8: return launch<kCall, T, V, 8, kWide>(a, st);
  }
  return TCU_DFT_ERR_UNSUPPORTED;
}

struct Shape {
  int64_t batches, runs;
  int blocks;  // of kBlockRows rows in a run
};

// Runs of up to 16 blocks of rows, so that few rows are read twice and few shares
// of dw written, but short enough to give every SM its 1024 threads.
Shape shape_of(const tcu_short_conv_args &a, int values) {
  Shape s;
  s.batches = a.offsets ? 1 : a.sequences;
  const int64_t tall = (a.rows + kBlockRows - 1) / kBlockRows;
  const int64_t threads = s.batches * tall * ((a.channels + values - 1) / values);
  s.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(16, threads / (1024 * num_sms())));
  s.runs = (tall + s.blocks - 1) / s.blocks;
  return s;
}

// Values a thread of the gradient owns: rows in words of 4 or 8 bytes.
constexpr int kGradValues = 2;

int check_sizes(const tcu_short_conv_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->channels < 1 || a->width < 1)
    return TCU_DFT_ERR_INVALID;
  if (a->width > TCU_SEQ_MAX_WIDTH || a->rows > kMostRows || a->channels > INT32_MAX)
    return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r : {&a->x, &a->y, &a->dy, &a->dx})
    if (!pitch_fits(a->rows, r->row_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  return TCU_DFT_OK;
}

template <typename T>
int dispatch(Call call, const tcu_short_conv_args &s, cudaStream_t st) {
  constexpr int most = 4;
  const int V = call == kGrad ? kGradValues : most;
  const Shape sh = shape_of(s, V);
  const int word = V * sizeof(T);
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
  a.rows = (int)s.rows;
  a.channels = s.channels;
  a.num_slots = s.num_slots;
  a.sequences = s.sequences;
  a.batches = (int)sh.batches;
  a.silu = s.silu;
  if (sh.runs * sh.batches > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  a.runs = (int)sh.runs;
  a.blocks = sh.blocks;
  if (call == kGrad) a.parts = static_cast<float *>(s.workspace);
  const int64_t batches = call == kStep ? s.sequences : sh.batches;
  bool wide = s.channels % V == 0 && (uintptr_t)s.weight % 16 == 0 &&
              rows_aligned(s.x, s.type, batches, s.rows, word);
  if (call == kGrad)
    wide = wide && rows_aligned(s.dy, s.type, batches, s.rows, word) &&
           rows_aligned(s.dx, s.type, batches, s.rows, word);
  else
    wide = wide && rows_aligned(s.y, s.type, batches, s.rows, word);
  for (const void *p : {s.state, s.dlast, (const void *)s.last, (const void *)s.dstate})
    wide = wide && (uintptr_t)p % word == 0;
  if (call == kForward)
    return wide ? by_width<kForward, T, most, true>(s.width, a, st)
                : by_width<kForward, T, 2, false>(s.width, a, st);
  if (call == kStep)
    return wide ? by_width<kStep, T, most, true>(s.width, a, st) : by_width<kStep, T, 2, false>(s.width, a, st);
  const int rc = wide ? by_width<kGrad, T, kGradValues, true>(s.width, a, st)
                      : by_width<kGrad, T, 2, false>(s.width, a, st);
  if (rc != TCU_DFT_OK) return rc;
  const int64_t weights = s.channels * s.width;
  const Sum sums[] = {{s.dweight, a.parts, weights}, {s.dbias, a.parts + weights, s.channels}};
  return sum_parts(sums, s.dbias ? 2 : 1, sh.runs * sh.batches, weights + s.channels, st);
}

int by_type(Call call, const tcu_short_conv_args &a, cudaStream_t st) {
  switch (a.type) {
    case TCU_SEQ_F32: return dispatch<float>(call, a, st);
    case TCU_SEQ_BF16: return dispatch<bf16>(call, a, st);
    default: return dispatch<f16>(call, a, st);
  }
}

}  // namespace

// A block sums 32 adjacent values, eight threads each, the eight in order.
struct Sums {
  Sum s[3];
};
__global__ void __launch_bounds__(256) sum_parts_kernel(Sums sums, int count, int64_t parts,
                                                        int64_t stride) {
  __shared__ float part[8][33];
  int64_t i = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
  const int y = threadIdx.x / 32;
  int k = 0;
  while (k < count && i >= sums.s[k].count) i -= sums.s[k++].count;
  float s = 0.f;
  if (k < count) {
    const float *from = sums.s[k].parts + i;
#pragma unroll 8
    for (int64_t p = y; p < parts; p += 8) s += from[p * (stride > 0 ? stride : sums.s[k].count)];
  }
  part[y][threadIdx.x % 32] = s;
  __syncthreads();
  if (y > 0 || k >= count) return;
#pragma unroll
  for (int j = 1; j < 8; ++j) s += part[j][threadIdx.x % 32];
  sums.s[k].out[i] = s;
}

int sum_parts(const Sum *sums, int count, int64_t parts, int64_t stride, cudaStream_t st) {
  Sums a{};
  int64_t n = 0;
  for (int k = 0; k < count; ++k) {
    a.s[k] = sums[k];
    n += sums[k].count;
  }
  if (n == 0) return TCU_DFT_OK;
  sum_parts_kernel<<<(unsigned)((n + 31) / 32), 256, 0, st>>>(a, count, parts, stride);
  return launched();
}

}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_short_conv_grad_workspace(const tcu_short_conv_args *a) {
  if (check_sizes(a) != TCU_DFT_OK) return -1;
  const Shape s = shape_of(*a, kGradValues);
  return s.runs * s.batches * a->channels * (a->width + 1) * 4;
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
  const wide_int cache = (wide_int)a->num_slots * (a->width - 1) * a->channels * sz;
  for (const tcu_seq_rows *r : {&a->x, &a->y})
    if (over(a->last, cache, r->ptr, a->channels * sz, a->sequences, r->batch_stride * sz))
      return TCU_DFT_ERR_INVALID;
  if (over(a->last, cache, a->weight, a->channels * a->width * 4) ||
      over(a->last, cache, a->bias, a->channels * 4) ||
      over(a->last, cache, a->slots, (int64_t)a->sequences * 4))
    return TCU_DFT_ERR_INVALID;
  return by_type(kStep, *a, static_cast<cudaStream_t>(stream));
}
