// state_scan.cuh -- kernels of the selective state-space scan, its gradient
// and its single-token form (include/tcu_seq.h), as templates on the element
// type; state_scan_{f32,bf16,f16}.cu instantiate them.
//
// Per sequence and channel, with N states n:
//     d_t = softplus(dt_t + dt_bias),   a_t[n] = exp(d_t A[n])
//     h_t[n] = a_t[n] h_{t-1}[n] + d_t u_t B_t[n]
//     o_t = sum_n C_t[n] h_t[n] + skip u_t,   y_t = o_t g_t sigma(g_t)
// and, with q_t = dy_t g_t sigma(g_t), the adjoint state
//     e_t[n] = C_t[n] q_t + a_{t+1}[n] e_{t+1}[n]   (+ dlast at the last row)
//     dC_t[n] = sum_c q_t h_t[n],           dB_t[n] = sum_c d_t u_t e_t[n]
//     r_t = sum_n e_t[n] B_t[n],            v_t[n] = a_t[n] e_t[n] h_{t-1}[n]
//     dA[n] = sum_t v_t[n] d_t,             dd_t = sum_n v_t[n] A[n] + r_t u_t
//     du_t = r_t d_t + skip q_t,            ddt_t = dd_t sigma(dt_t + dt_bias)
//     dg_t = dy_t o_t (g sigma(g))',        dskip = sum_t q_t u_t
// (dB, dC over the channels of the group; dA, dskip over batch and rows).
//
// Layout.  A thread owns CH channels x 4 states in registers; LS adjacent
// lanes cover a channel's states, the other lanes further channels, so a row
// costs a thread CH * 4 independent recurrence steps for one 16-byte load
// each of B, C (4 states), d and d u (CH channels) from shared memory, the
// sums over states are a shuffle reduction over LS lanes, and those over
// channels (gradients of B and C) one over the other 32 / LS.  A block is 4
// warps of adjacent channels of one group; it walks down its rows in tiles of
// kTile, first turning u, dt (and gate, dy) into d, d u, q once per value.
//
// Time is split into chunks where batch x channels alone do not fill the
// card: a first kernel leaves each chunk's final state from a zero start and
// its sum of d, a second carries states over the chunks (a chunk multiplies
// by exp(A sum d)), and the main kernel starts every chunk from its true
// state.  The gradient does the same from the other end.
//
// Packed sequences: row_sequence_kernel writes the sequence of every row; a
// sequence opens where that changes, which the kernels keep as a bit mask per
// tile and test per row.
#pragma once
#include <algorithm>

#include "seq_common.cuh"

namespace tcu {
namespace seq {

constexpr int kWarps = 4;
constexpr int kScanThreads = 32 * kWarps;
constexpr int kTile = TCU_SEQ_MARK;  // rows of a tile: a warp's ballot covers it
constexpr int kSub = 4;              // rows whose states a gradient thread holds
static_assert(kTile == 32, "masks of a tile's rows are 32-bit");

template <typename T>
struct ScanArgs {
  Rows<const T> u, dt, gate, B, C, dy;
  Rows<T> y, du, ddt, dgate, dB, dC;
  const float *A, *skip, *dt_bias, *state, *dlast;
  float *last, *dstate, *marks;
  // workspace
  float *carry;    // [batch][chunk][channels][states]: state that enters a chunk
  float *sum_d;    // [batch][chunk][channels]
  int32_t *row_seq;
  float *bc_parts;  // [channel block of a group][batch][row][group][dB, dC][states]
  float *A_parts;   // [batch][chunk][channels][states]
  float *skip_parts, *bias_parts;  // [batch][chunk][channels]
  const int32_t *offsets, *slots;
  int64_t rows, channels, num_slots;
  int64_t chunk_rows;
  int states, groups, per_group, group_blocks;
  int sequences, batches, chunks, softplus;
};

// The channels a block of the given kernel covers, and its rows.
template <int DB, typename T>
struct Place {
  int64_t b, k, r0, r1;
  int g, cb;
  int64_t c0;
  int nc;
  __device__ __forceinline__ explicit Place(const ScanArgs<T> &a) {
    const int blocks = a.groups * a.group_blocks;
    const int64_t id = blockIdx.x;
    const int blk = (int)(id % blocks);
    const int64_t bk = id / blocks;
    k = bk % a.chunks;
    b = bk / a.chunks;
    g = blk / a.group_blocks;
    cb = blk % a.group_blocks;
    c0 = (int64_t)g * a.per_group + cb * DB;
    nc = min(DB, a.per_group - cb * DB);
    r0 = k * a.chunk_rows;
    r1 = min(r0 + a.chunk_rows, a.rows);
  }
};

__device__ __forceinline__ float softplus(float v) {
  return fmaxf(v, 0.f) + log1pf(exp2_fast(-kLog2e * fabsf(v)));
}

// Four states of one channel, from / to an array [..][states].
__device__ __forceinline__ void load4(float (&h)[4], const float *p, int n, int states) {
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = n + i < states ? p[n + i] : 0.f;
}
__device__ __forceinline__ void store4(float *p, const float (&h)[4], int n, int states) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < states) p[n + i] = h[i];
}

// Sums v[i] over groups of L lanes at stride S (L * S <= 32, powers of two).
// Halves the values at every step while there are several: afterwards the
// lane of rank q within its group holds the sums of values first(q) ..
// first(q) + max(1, V / L), in v[0 ..].
template <int V, int L, int S>
__device__ __forceinline__ void reduce_scatter(float *v, int lane) {
  if constexpr (L > 1) {
    constexpr int half = L / 2 * S;
    if constexpr (V > 1) {
      const bool up = lane & half;
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float send = up ? v[i] : v[i + V / 2];
        const float keep = up ? v[i + V / 2] : v[i];
        v[i] = keep + __shfl_xor_sync(~0u, send, half);
      }
      reduce_scatter<V / 2, L / 2, S>(v, lane);
    } else {
      v[0] += __shfl_xor_sync(~0u, v[0], half);
      reduce_scatter<1, L / 2, S>(v, lane);
    }
  }
}
// Which values a lane of rank q holds after reduce_scatter<V, L, S>.
template <int V, int L>
__device__ __forceinline__ int first_of(int q) {
  if constexpr (L == 1 || V == 1) return 0;
  else return (q >= L / 2 ? V / 2 : 0) + first_of<V / 2, L / 2>(q % (L / 2));
}
// Whether the lane is the first of those that hold the same sums.
template <int V, int L>
__device__ __forceinline__ bool owner_of(int q) {
  return V >= L || q % (L / (V < L ? V : L)) == 0;
}

// Bits of the tile's rows that open (or, closes, end) a sequence.
template <typename T>
__device__ __forceinline__ uint32_t opens_mask(const ScanArgs<T> &a, int64_t row0, int lane) {
  const int64_t r = row0 + lane;
  const bool o = r < a.rows && (r == 0 || a.row_seq[r] != a.row_seq[r - 1]);
  return __ballot_sync(~0u, o);
}
template <typename T>
__device__ __forceinline__ uint32_t closes_mask(const ScanArgs<T> &a, int64_t row0, int lane) {
  const int64_t r = row0 + lane;
  const bool c = r < a.rows && (r + 1 == a.rows || a.row_seq[r] != a.row_seq[r + 1]);
  return __ballot_sync(~0u, c);
}

__global__ void row_sequence_kernel(int32_t *row_seq, const int32_t *offsets, int count,
                                    int64_t rows);

// Shape of a kernel: LS lanes over the states, CH channels a thread.
template <int LS_, int CH_>
struct Shape {
  static constexpr int LS = LS_, CH = CH_;
  static constexpr int kStates = 4 * LS;            // states, padded
  static constexpr int kWarpChannels = 32 / LS * CH;
  static constexpr int kChannels = kWarps * kWarpChannels;
};

// Stages a tile of B and C ([row][padded states], zeros past the end).
template <int NP, typename T>
__device__ __forceinline__ void stage_bc(const ScanArgs<T> &a, int64_t b, int g, int64_t row0,
                                         int rows, float *sB, float *sC) {
  for (int e = threadIdx.x; e < kTile * NP; e += kScanThreads) {
    const int t = e / NP, n = e % NP;
    float vb = 0.f, vc = 0.f;
    if (t < rows && n < a.states) {
      vb = to_f(a.B.at(b, row0 + t)[(int64_t)g * a.states + n]);
      if (sC) vc = to_f(a.C.at(b, row0 + t)[(int64_t)g * a.states + n]);
    }
    sB[e] = vb;
    if (sC) sC[e] = vc;
  }
}

// d of one value.
template <typename T>
__device__ __forceinline__ float step_of(const ScanArgs<T> &a, float dt, float bias) {
  const float v = dt + bias;
  return a.softplus ? softplus(v) : v;
}

// The scan of a chunk.  kLocal: from a zero start, leaving its final state
// and sum of d for the carry; otherwise from the carried state, with outputs.
template <typename T, class P, bool kPacked, bool kLocal>
__global__ void __launch_bounds__(kScanThreads) scan_kernel(ScanArgs<T> a) {
  constexpr int LS = P::LS, CH = P::CH, NP = P::kStates, DB = P::kChannels;
  extern __shared__ __align__(16) float smem[];
  float *sd = smem, *sx = sd + kTile * DB, *sB = sx + kTile * DB, *sC = sB + kTile * NP;
  const Place<DB, T> w(a);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int sl = lane % LS, n0 = sl * 4;
  const int ch0 = warp * P::kWarpChannels + lane / LS * CH;  // of the block
  float A2[CH][4], h[CH][4], dsum[CH];
  const int64_t state0 = (w.b * a.chunks + w.k) * a.channels + w.c0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const bool in = ch0 + c < w.nc;
    dsum[c] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] = h[c][i] = 0.f;
    if (!in) continue;
    load4(A2[c], a.A + (w.c0 + ch0 + c) * a.states, n0, a.states);
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] *= kLog2e;
    if (!kPacked && w.k == 0) {
      if (a.state)
        load4(h[c], a.state + (w.b * a.channels + w.c0 + ch0 + c) * a.states, n0, a.states);
    } else if (!kLocal && w.k > 0) {
      load4(h[c], a.carry + (state0 + ch0 + c) * a.states, n0, a.states);
    }
  }
  for (int64_t row0 = w.r0; row0 < w.r1; row0 += kTile) {
    const int rows = (int)min((int64_t)kTile, w.r1 - row0);
    __syncthreads();
    for (int e = threadIdx.x; e < kTile * DB; e += kScanThreads) {
      const int t = e / DB, c = e % DB;
      float d = 0.f, x = 0.f;
      if (t < rows && c < w.nc) {
        const float bias = a.dt_bias ? a.dt_bias[w.c0 + c] : 0.f;
        d = step_of(a, to_f(a.dt.at(w.b, row0 + t)[w.c0 + c]), bias);
        x = d * to_f(a.u.at(w.b, row0 + t)[w.c0 + c]);
      }
      sd[e] = d;
      sx[e] = x;
    }
    stage_bc<NP>(a, w.b, w.g, row0, rows, sB, kLocal ? nullptr : sC);
    const uint32_t opens = kPacked ? opens_mask(a, row0, lane) : 0;
    __syncthreads();
    if (!kLocal && a.marks) {
      const int64_t marks = (a.rows + kTile - 1) / kTile;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (ch0 + c < w.nc)
          store4(a.marks + ((w.b * marks + row0 / kTile) * a.channels + w.c0 + ch0 + c) * a.states,
                 h[c], n0, a.states);
    }
    for (int t = 0; t < rows; ++t) {
      if (kPacked && (opens >> t & 1)) {
        const int64_t r = row0 + t;
        const int s = a.row_seq[r], before = r > 0 ? a.row_seq[r - 1] : -1;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (ch0 + c >= w.nc) continue;
          const int64_t at = w.c0 + ch0 + c;
          if (!kLocal && a.last && before >= 0)
            store4(a.last + (before * a.channels + at) * a.states, h[c], n0, a.states);
          dsum[c] = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) h[c][i] = 0.f;
          if (a.state && s >= 0)
            load4(h[c], a.state + (s * a.channels + at) * a.states, n0, a.states);
        }
      }
      float y[CH];
      const float4 B4 = *reinterpret_cast<const float4 *>(sB + t * NP + n0);
      const float B[4] = {B4.x, B4.y, B4.z, B4.w};
      float C[4] = {};
      if (!kLocal) {
        const float4 C4 = *reinterpret_cast<const float4 *>(sC + t * NP + n0);
        C[0] = C4.x, C[1] = C4.y, C[2] = C4.z, C[3] = C4.w;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const float d = sd[t * DB + ch0 + c], x = sx[t * DB + ch0 + c];
        y[c] = 0.f;
        if (kLocal) dsum[c] += d;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[c][i] = fmaf(exp2_fast(d * A2[c][i]), h[c][i], x * B[i]);
          if (!kLocal) y[c] = fmaf(C[i], h[c][i], y[c]);
        }
      }
      if (!kLocal) {
        reduce_scatter<CH, LS, 1>(y, lane);
        __syncwarp();
        constexpr int held = CH > LS ? CH / LS : 1;
        if (owner_of<CH, LS>(sl)) {
          const int at = t * DB + ch0 + first_of<CH, LS>(sl);
#pragma unroll
          for (int i = 0; i < held; ++i) sx[at + i] = y[i];
        }
      }
    }
    if (kLocal) continue;
    __syncthreads();
    for (int e = threadIdx.x; e < rows * DB; e += kScanThreads) {
      const int t = e / DB, c = e % DB;
      if (c >= w.nc) continue;
      float o = sx[e];
      if (a.skip) o = fmaf(a.skip[w.c0 + c], to_f(a.u.at(w.b, row0 + t)[w.c0 + c]), o);
      if (a.gate.p) o *= silu(to_f(a.gate.at(w.b, row0 + t)[w.c0 + c]));
      a.y.at(w.b, row0 + t)[w.c0 + c] = from_f<T>(o);
    }
  }
  if (kLocal) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (ch0 + c >= w.nc) continue;
      store4(a.carry + (state0 + ch0 + c) * a.states, h[c], n0, a.states);
      if (sl == 0) a.sum_d[state0 + ch0 + c] = dsum[c];
    }
  } else if (a.last && w.r1 == a.rows) {
    const int s = kPacked ? a.row_seq[a.rows - 1] : (int)w.b;
    if (s >= 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (ch0 + c < w.nc)
          store4(a.last + (s * a.channels + w.c0 + ch0 + c) * a.states, h[c], n0, a.states);
    }
  }
}

// carry[k] <- the state that enters chunk k (kBack: the adjoint that enters
// it from below), from each chunk's own contribution in carry[k].
template <typename T, bool kBack>
__global__ void carry_kernel(ScanArgs<T> a) {
  const int64_t per = a.channels * a.states;
  const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (id >= per * a.batches) return;
  const int64_t b = id / per, at = id % per, c = at / a.states;
  const float A2 = a.A[at] * kLog2e;
  float h = 0.f;
  for (int j = 0; j < a.chunks; ++j) {
    const int k = kBack ? a.chunks - 1 - j : j;
    const int64_t r0 = k * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
    float *p = a.carry + (b * a.chunks + k) * per + at;
    const float own = *p, decay = exp2_fast(A2 * a.sum_d[(b * a.chunks + k) * a.channels + c]);
    // does a sequence open (close, going back) within the chunk?
    bool cut;
    if (kBack) cut = r1 == a.rows || (a.row_seq && a.row_seq[r0] != a.row_seq[r1]);
    else cut = r0 == 0 || (a.row_seq && a.row_seq[r0 - 1] != a.row_seq[r1 - 1]);
    *p = h;
    h = cut || h == 0.f ? own : fmaf(decay, h, own);
  }
}

// One token: LS lanes per channel, 4 states each, the cache in place.
template <typename T, int LS>
__global__ void __launch_bounds__(kScanThreads) scan_step_kernel(ScanArgs<T> a) {
  const int64_t id = ((int64_t)blockIdx.x * kScanThreads + threadIdx.x) / LS;
  const int sl = threadIdx.x % LS, n0 = sl * 4;
  const bool in = id < a.channels * a.sequences;
  const int64_t b = in ? id / a.channels : 0, c = in ? id % a.channels : 0;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool live = in && slot >= 0 && slot < a.num_slots;
  float o = 0.f, u = 0.f;
  if (live) {
    u = to_f(a.u.at(b, 0)[c]);
    const float d = step_of(a, to_f(a.dt.at(b, 0)[c]), a.dt_bias ? a.dt_bias[c] : 0.f);
    const float x = d * u;
    float A[4], h[4];
    load4(A, a.A + c * a.states, n0, a.states);
    float *cache = a.last + (slot * a.channels + c) * a.states;
    load4(h, cache, n0, a.states);
    const int64_t g = c / a.per_group * a.states;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n0 + i >= a.states) continue;
      h[i] = fmaf(exp2_fast(d * (A[i] * kLog2e)), h[i], x * to_f(a.B.at(b, 0)[g + n0 + i]));
      o = fmaf(to_f(a.C.at(b, 0)[g + n0 + i]), h[i], o);
    }
    store4(cache, h, n0, a.states);
  }
#pragma unroll
  for (int s = LS / 2; s > 0; s /= 2) o += __shfl_xor_sync(~0u, o, s);
  if (!in || sl != 0) return;
  if (live) {
    if (a.skip) o = fmaf(a.skip[c], u, o);
    if (a.gate.p) o *= silu(to_f(a.gate.at(b, 0)[c]));
  }
  a.y.at(b, 0)[c] = from_f<T>(live ? o : 0.f);
}

// ---------------------------------------------------------------- gradient
// The adjoint of a chunk from a zero start below it: its contribution to the
// adjoint above it and its sum of d.
template <typename T, class P, bool kPacked>
__global__ void __launch_bounds__(kScanThreads) adjoint_kernel(ScanArgs<T> a) {
  constexpr int LS = P::LS, CH = P::CH, NP = P::kStates, DB = P::kChannels;
  extern __shared__ __align__(16) float smem[];
  float *sd = smem, *sq = sd + kTile * DB, *sC = sq + kTile * DB;
  const Place<DB, T> w(a);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int sl = lane % LS, n0 = sl * 4;
  const int ch0 = warp * P::kWarpChannels + lane / LS * CH;
  float A2[CH][4], e[CH][4], dsum[CH];
  const int64_t state0 = (w.b * a.chunks + w.k) * a.channels + w.c0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    dsum[c] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] = e[c][i] = 0.f;
    if (ch0 + c >= w.nc) continue;
    const int64_t at = w.c0 + ch0 + c;
    load4(A2[c], a.A + at * a.states, n0, a.states);
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] *= kLog2e;
    if (!kPacked && w.r1 == a.rows && a.dlast)
      load4(e[c], a.dlast + (w.b * a.channels + at) * a.states, n0, a.states);
  }
  const int64_t tiles = (w.r1 - w.r0 + kTile - 1) / kTile;
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t row0 = w.r0 + tile * kTile;
    const int rows = (int)min((int64_t)kTile, w.r1 - row0);
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * DB; i += kScanThreads) {
      const int t = i / DB, c = i % DB;
      float d = 0.f, q = 0.f;
      if (t < rows && c < w.nc) {
        d = step_of(a, to_f(a.dt.at(w.b, row0 + t)[w.c0 + c]),
                    a.dt_bias ? a.dt_bias[w.c0 + c] : 0.f);
        q = to_f(a.dy.at(w.b, row0 + t)[w.c0 + c]);
        if (a.gate.p) q *= silu(to_f(a.gate.at(w.b, row0 + t)[w.c0 + c]));
      }
      sd[i] = d;
      sq[i] = q;
    }
    for (int i = threadIdx.x; i < kTile * NP; i += kScanThreads) {
      const int t = i / NP, n = i % NP;
      sC[i] = t < rows && n < a.states
                  ? to_f(a.C.at(w.b, row0 + t)[(int64_t)w.g * a.states + n])
                  : 0.f;
    }
    const uint32_t closes = kPacked ? closes_mask(a, row0, lane) : 0;
    __syncthreads();
    for (int t = rows - 1; t >= 0; --t) {
      if (kPacked && (closes >> t & 1)) {
        const int s = a.row_seq[row0 + t];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
          for (int i = 0; i < 4; ++i) e[c][i] = 0.f;
          if (ch0 + c < w.nc && a.dlast && s >= 0)
            load4(e[c], a.dlast + (s * a.channels + w.c0 + ch0 + c) * a.states, n0, a.states);
        }
      }
      const float4 C4 = *reinterpret_cast<const float4 *>(sC + t * NP + n0);
      const float C[4] = {C4.x, C4.y, C4.z, C4.w};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const float d = sd[t * DB + ch0 + c], q = sq[t * DB + ch0 + c];
        dsum[c] += d;
#pragma unroll
        for (int i = 0; i < 4; ++i) e[c][i] = exp2_fast(d * A2[c][i]) * fmaf(C[i], q, e[c][i]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (ch0 + c >= w.nc) continue;
    store4(a.carry + (state0 + ch0 + c) * a.states, e[c], n0, a.states);
    if (sl == 0) a.sum_d[state0 + ch0 + c] = dsum[c];
  }
}

// Shared memory of the gradient kernel, in floats.
template <class P>
constexpr int grad_floats() {
  return kTile * P::kChannels * 3 + kTile * P::kStates * 2 +
         kTile / kSub * P::CH * 4 * kScanThreads + kWarps * kTile * P::kStates * 2;
}

// The gradient over a chunk.  Tiles from the last to the first: the states of
// a tile are recomputed from its mark, keeping every kSub-th in shared memory
// (each thread its own); then kSub rows at a time from those, with states and
// decays in registers, the adjoint walks up.
template <typename T, class P, bool kPacked>
__global__ void __launch_bounds__(kScanThreads) scan_grad_kernel(ScanArgs<T> a) {
  constexpr int LS = P::LS, CH = P::CH, NP = P::kStates, DB = P::kChannels;
  constexpr int CL = 32 / LS, E = CH * 4;
  extern __shared__ __align__(16) float smem[];
  float *sd = smem, *sx = sd + kTile * DB, *sq = sx + kTile * DB, *sB = sq + kTile * DB,
        *sC = sB + kTile * NP, *snap = sC + kTile * NP, *sbc = snap + kTile / kSub * E * kScanThreads;
  const Place<DB, T> w(a);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int sl = lane % LS, n0 = sl * 4;
  const int ch0 = warp * P::kWarpChannels + lane / LS * CH;
  float A2[CH][4], dA[CH][4], e[CH][4];
  const int64_t part = w.b * a.chunks + w.k;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] = e[c][i] = dA[c][i] = 0.f;
    if (ch0 + c >= w.nc) continue;
    const int64_t at = w.c0 + ch0 + c;
    load4(A2[c], a.A + at * a.states, n0, a.states);
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[c][i] *= kLog2e;
    if (w.r1 < a.rows)
      load4(e[c], a.carry + (part * a.channels + at) * a.states, n0, a.states);
    else if (!kPacked && a.dlast)
      load4(e[c], a.dlast + (w.b * a.channels + at) * a.states, n0, a.states);
  }
  // the epilogue's thread owns one channel (or shares it with others, DB < threads)
  const int ec = threadIdx.x % DB;
  float dskip = 0.f, dbias = 0.f;
  const int64_t marks = (a.rows + kTile - 1) / kTile;
  const int64_t tiles = (w.r1 - w.r0 + kTile - 1) / kTile;
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t row0 = w.r0 + tile * kTile;
    const int rows = (int)min((int64_t)kTile, w.r1 - row0);
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * DB; i += kScanThreads) {
      const int t = i / DB, c = i % DB;
      float d = 0.f, x = 0.f, q = 0.f;
      if (t < rows && c < w.nc) {
        d = step_of(a, to_f(a.dt.at(w.b, row0 + t)[w.c0 + c]),
                    a.dt_bias ? a.dt_bias[w.c0 + c] : 0.f);
        x = d * to_f(a.u.at(w.b, row0 + t)[w.c0 + c]);
        q = to_f(a.dy.at(w.b, row0 + t)[w.c0 + c]);
        if (a.gate.p) q *= silu(to_f(a.gate.at(w.b, row0 + t)[w.c0 + c]));
      }
      sd[i] = d;
      sx[i] = x;
      sq[i] = q;
    }
    stage_bc<NP>(a, w.b, w.g, row0, rows, sB, sC);
    const uint32_t opens = kPacked ? opens_mask(a, row0, lane) : 0;
    const uint32_t closes = kPacked ? closes_mask(a, row0, lane) : 0;
    float h[CH][4];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) h[c][i] = 0.f;
      if (ch0 + c < w.nc)
        load4(h[c], a.marks + ((w.b * marks + row0 / kTile) * a.channels + w.c0 + ch0 + c) * a.states,
              n0, a.states);
    }
    __syncthreads();
    auto open = [&](int t) {  // the state a sequence starts from
      const int s = a.row_seq[row0 + t];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[c][i] = 0.f;
        if (a.state && s >= 0 && ch0 + c < w.nc)
          load4(h[c], a.state + (s * a.channels + w.c0 + ch0 + c) * a.states, n0, a.states);
      }
    };
    auto keep = [&](int sub) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          snap[(sub * E + c * 4 + i) * kScanThreads + threadIdx.x] = h[c][i];
    };
    const int subs = (rows + kSub - 1) / kSub;
    for (int sub = 0; sub < subs; ++sub) {
      keep(sub);
      if (sub == subs - 1) break;
#pragma unroll
      for (int j = 0; j < kSub; ++j) {
        const int t = sub * kSub + j;
        if (kPacked && (opens >> t & 1)) open(t);
        const float4 B4 = *reinterpret_cast<const float4 *>(sB + t * NP + n0);
        const float B[4] = {B4.x, B4.y, B4.z, B4.w};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const float d = sd[t * DB + ch0 + c], x = sx[t * DB + ch0 + c];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            h[c][i] = fmaf(exp2_fast(d * A2[c][i]), h[c][i], x * B[i]);
        }
      }
    }
    for (int sub = subs - 1; sub >= 0; --sub) {
      float hs[kSub][CH][4], as[kSub][CH][4];
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          h[c][i] = snap[(sub * E + c * 4 + i) * kScanThreads + threadIdx.x];
#pragma unroll
      for (int j = 0; j < kSub; ++j) {
        // rows past the end have d = x = 0: the state stays
        const int t = sub * kSub + j;
        if (kPacked && (opens >> t & 1)) open(t);
        const float4 B4 = *reinterpret_cast<const float4 *>(sB + t * NP + n0);
        const float B[4] = {B4.x, B4.y, B4.z, B4.w};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const float d = sd[t * DB + ch0 + c], x = sx[t * DB + ch0 + c];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            as[j][c][i] = exp2_fast(d * A2[c][i]);
            h[c][i] = fmaf(as[j][c][i], h[c][i], x * B[i]);
            hs[j][c][i] = h[c][i];
          }
        }
      }
#pragma unroll
      for (int j = kSub - 1; j >= 0; --j) {
        const int t = sub * kSub + j;
        if (kPacked && (closes >> t & 1)) {
          const int s = a.row_seq[row0 + t];
#pragma unroll
          for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) e[c][i] = 0.f;
            if (ch0 + c < w.nc && a.dlast && s >= 0)
              load4(e[c], a.dlast + (s * a.channels + w.c0 + ch0 + c) * a.states, n0, a.states);
          }
        }
        // h <- the state before row t
        if (kPacked && (opens >> t & 1)) {
          open(t);
        } else {
#pragma unroll
          for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              h[c][i] = j > 0 ? hs[j > 0 ? j - 1 : 0][c][i]
                              : snap[(sub * E + c * 4 + i) * kScanThreads + threadIdx.x];
        }
        const float4 B4 = *reinterpret_cast<const float4 *>(sB + t * NP + n0);
        const float4 C4 = *reinterpret_cast<const float4 *>(sC + t * NP + n0);
        const float B[4] = {B4.x, B4.y, B4.z, B4.w}, C[4] = {C4.x, C4.y, C4.z, C4.w};
        float bc[8] = {};
        float o[CH], r[CH], v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const float d = sd[t * DB + ch0 + c], x = sx[t * DB + ch0 + c], q = sq[t * DB + ch0 + c];
          o[c] = r[c] = v[c] = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float ee = fmaf(C[i], q, e[c][i]);
            bc[i] = fmaf(x, ee, bc[i]);
            bc[4 + i] = fmaf(q, hs[j][c][i], bc[4 + i]);
            r[c] = fmaf(ee, B[i], r[c]);
            o[c] = fmaf(hs[j][c][i], C[i], o[c]);
            e[c][i] = as[j][c][i] * ee;
            const float p = e[c][i] * h[c][i];
            v[c] = fmaf(p, A2[c][i], v[c]);
            dA[c][i] = fmaf(p, d, dA[c][i]);
          }
        }
        if (kPacked && (opens >> t & 1) && a.dstate && a.row_seq[row0 + t] >= 0) {
#pragma unroll
          for (int c = 0; c < CH; ++c)
            if (ch0 + c < w.nc)
              store4(a.dstate + (a.row_seq[row0 + t] * a.channels + w.c0 + ch0 + c) * a.states,
                     e[c], n0, a.states);
        }
        // sums over states: one channel's o, r, v to its owner, in place of
        // the row's x, q, d (read by this warp only, and for the last time)
        reduce_scatter<CH, LS, 1>(o, lane);
        reduce_scatter<CH, LS, 1>(r, lane);
        reduce_scatter<CH, LS, 1>(v, lane);
        __syncwarp();
        if (owner_of<CH, LS>(sl)) {
          constexpr int held = CH > LS ? CH / LS : 1;
          const int at = t * DB + ch0 + first_of<CH, LS>(sl);
#pragma unroll
          for (int i = 0; i < held; ++i) {
            sx[at + i] = o[i];
            sq[at + i] = r[i];
            sd[at + i] = v[i];
          }
        }
        // sums over the warp's channels
        reduce_scatter<8, CL, LS>(bc, lane);
        if (owner_of<8, CL>(lane / LS)) {
          constexpr int held = 8 > CL ? 8 / CL : 1;
          const int f = first_of<8, CL>(lane / LS);
#pragma unroll
          for (int i = 0; i < held; ++i) {
            const int which = (f + i) / 4, n = n0 + (f + i) % 4;
            sbc[((warp * kTile + t) * 2 + which) * NP + n] = bc[i];
          }
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * 2 * NP; i += kScanThreads) {
      const int n = i % NP;
      if (n >= a.states) continue;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) s += sbc[k * kTile * 2 * NP + i];
      const int t = i / (2 * NP), which = i / NP % 2;
      a.bc_parts[((((int64_t)w.cb * a.batches + w.b) * a.rows + row0 + t) * a.groups + w.g) * 2 *
                     a.states + which * a.states + n] = s;
    }
    if (ec < w.nc) {
      const int64_t c = w.c0 + ec;
      const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;
      for (int t = threadIdx.x / DB; t < rows; t += kScanThreads / DB) {
        const int64_t r = row0 + t;
        const float u = to_f(a.u.at(w.b, r)[c]), dt = to_f(a.dt.at(w.b, r)[c]) + bias;
        const float dy = to_f(a.dy.at(w.b, r)[c]);
        const float d = a.softplus ? softplus(dt) : dt;
        const float o = sx[t * DB + ec], rr = sq[t * DB + ec], v = sd[t * DB + ec] * kLn2;
        float q = dy;
        if (a.gate.p) {
          const float z = to_f(a.gate.at(w.b, r)[c]);
          q *= silu(z);
          if (a.dgate.p) a.dgate.at(w.b, r)[c] = from_f<T>(dy * fmaf(skip, u, o) * dsilu(z));
        }
        float g = fmaf(rr, u, v);
        if (a.softplus) g *= sigmoid(dt);
        a.du.at(w.b, r)[c] = from_f<T>(fmaf(rr, d, skip * q));
        a.ddt.at(w.b, r)[c] = from_f<T>(g);
        dskip = fmaf(q, u, dskip);
        dbias += g;
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (ch0 + c >= w.nc) continue;
    const int64_t at = w.c0 + ch0 + c;
    store4(a.A_parts + (part * a.channels + at) * a.states, dA[c], n0, a.states);
    if (!kPacked && a.dstate && w.k == 0)
      store4(a.dstate + (w.b * a.channels + at) * a.states, e[c], n0, a.states);
  }
  __syncthreads();
  sd[threadIdx.x] = dskip;
  sx[threadIdx.x] = dbias;
  __syncthreads();
  if (threadIdx.x < w.nc) {
    float s = 0.f, bsum = 0.f;
    for (int i = threadIdx.x; i < kScanThreads; i += DB) {
      s += sd[i];
      bsum += sx[i];
    }
    const int64_t at = part * a.channels + w.c0 + threadIdx.x;
    if (a.skip_parts) a.skip_parts[at] = s;
    if (a.bias_parts) a.bias_parts[at] = bsum;
  }
}

// dB and dC from the channel blocks' shares, in order.
template <typename T>
__global__ void sum_bc_kernel(ScanArgs<T> a) {
  const int64_t per = (int64_t)a.groups * 2 * a.states, count = a.batches * a.rows * per;
  const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (id >= count) return;
  float s = 0.f;
  for (int k = 0; k < a.group_blocks; ++k) s += a.bc_parts[k * count + id];
  const int64_t row = id / per, in = id % per;
  const int64_t b = row / a.rows, t = row % a.rows;
  const int g = (int)(in / (2 * a.states)), which = (int)(in / a.states % 2), n = (int)(in % a.states);
  const Rows<T> &out = which ? a.dC : a.dB;
  out.at(b, t)[(int64_t)g * a.states + n] = from_f<T>(s);
}

// ------------------------------------------------------------- host side
enum ScanCall { kScan, kScanGrad, kScanStep };

// The channels of a block by the lanes over the states: forward and gradient.
constexpr int scan_ch(int ls) { return ls < 4 ? ls : 4; }
constexpr int grad_ch(int ls) { return ls < 2 ? 1 : 2; }
constexpr int block_channels(int ls, int ch) { return kWarps * (32 / ls) * ch; }

inline int lanes_of(int64_t states) {
  int ls = 1;
  while (ls * 4 < states) ls *= 2;
  return ls;
}

// How rows are split into chunks, and the workspace that takes.
struct ScanPlan {
  int64_t batches, chunk_rows;
  int ls, db, per_group, group_blocks, chunks;
  // floats
  int64_t carry, sum_d, row_seq, bc_parts, A_parts, vec_parts;
  int64_t total() const { return carry + sum_d + row_seq + bc_parts + A_parts + 2 * vec_parts; }
};
ScanPlan plan_of(const tcu_state_scan_args &a, bool grad);

template <typename T>
int run_scan(ScanCall call, const tcu_state_scan_args &s, cudaStream_t st);

}  // namespace seq
}  // namespace tcu
