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
// What bounds it.  At 16 states a (row, channel) is 8 bytes of 16-bit rows in
// and out, 16 exponentials and 64 fp32 operations forward: on this card 32
// exponentials and 128 fp32 operations a clock and SM, so the special function
// unit and the FMA pipe both need 1.4 times HBM's time, the gradient's 200
// operations three times.  The kernels are made for those pipes: packed fp32
// (fma.rn.f32x2, half the issue slots), recurrences in registers, and few words
// drawn from shared memory, whose pipe returns 32 a clock however few of them
// differ.
//
// Layout.  A thread owns CH channels x 4 states, in pairs of channels; LS
// adjacent lanes cover a channel's states, the other lanes further channels.  A
// row then costs it CH * 4 independent recurrence steps for one 16-byte load
// each of B, C (4 states), d and d u (CH channels).  Sums over states go over LS
// lanes, sums over channels (gradients of B and C) over the other 32 / LS.
//
// Time is split into chunks where batch x channels alone do not fill the
// card: a first kernel leaves each chunk's final state from a zero start and
// its sum of d, a second carries states over the chunks (a chunk multiplies
// by exp(A sum d)), and the main kernel starts every chunk from its true
// state.  The gradient does the same from the other end.
//
// Packed sequences: row_sequence_kernel writes the sequence of every row; a
// sequence opens where that changes, which the kernels keep as a bit mask of
// the rows at hand and test per row only where one is set.
#pragma once
#include <algorithm>

#include "seq_common.cuh"
#include "tcgen05.cuh"

namespace tcu {
namespace seq {

constexpr int kScanThreads = 128;     // of the single-token kernel
constexpr int kTile = 32;             // rows of a forward tile: a warp's ballot
constexpr int kMark = TCU_SEQ_MARK;   // rows of a gradient tile

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
  float *bc_parts;  // [block of a group's channels][batch][row][group][dB, dC][states]
  float *A_parts;   // [batch][chunk][channels][states]
  float *skip_parts, *bias_parts;  // [batch][chunk][channels]
  const int32_t *offsets, *slots;
  int64_t channels, num_slots;
  int rows, chunk_rows;
  int states, groups, per_group, group_blocks;
  int sequences, batches, chunks, softplus;
  // whether states, and B and C, are read in words of four values
  int wide_states, wide_bc;
  int wide;  // whether rows are, in words of 16 bytes
};

// The channels a block of the given kernel covers, and its rows.
template <int DB, typename T>
struct Place {
  int64_t b, k, c0;
  int r0, r1;  // rows
  int g, cb, nc;
  // of `chunks` chunks from `first` on
  __device__ __forceinline__ explicit Place(const ScanArgs<T> &a, int chunks, int first) {
    const unsigned blocks = a.groups * a.group_blocks, bk = blockIdx.x / blocks;
    const unsigned blk = blockIdx.x - bk * blocks;
    b = bk / (unsigned)chunks;
    k = first + (int)(bk - (unsigned)b * chunks);
    g = (int)(blk / (unsigned)a.group_blocks);
    cb = (int)blk - g * a.group_blocks;
    c0 = (int64_t)g * a.per_group + cb * DB;
    nc = min(DB, a.per_group - cb * DB);
    r0 = (int)k * a.chunk_rows;
    r1 = chunk_end(r0, a.chunk_rows, a.rows);
  }
};

__device__ __forceinline__ float softplus(float v) { return softplus2(make_float2(v, v)).x; }

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
__device__ __forceinline__ uint32_t opens_mask(const ScanArgs<T> &a, int row0, int lane) {
  const int r = row0 + lane;
  const bool o = r < a.rows && (r == 0 || a.row_seq[r] != a.row_seq[r - 1]);
  return __ballot_sync(~0u, o);
}
template <typename T>
__device__ __forceinline__ uint32_t closes_mask(const ScanArgs<T> &a, int row0, int lane) {
  const int r = row0 + lane;
  const bool c = r < a.rows && (r + 1 == a.rows || a.row_seq[r] != a.row_seq[r + 1]);
  return __ballot_sync(~0u, c);
}

__global__ void row_sequence_kernel(int32_t *row_seq, const int32_t *offsets, int count,
                                    int rows);

// d of one value.
template <typename T>
__device__ __forceinline__ float step_of(const ScanArgs<T> &a, float dt, float bias) {
  const float v = dt + bias;
  return a.softplus ? softplus(v) : v;
}

// ------------------------------------------------------------------ forward
// How the forward kernels are laid out.  A block is pairs of warps over
// adjacent channels of one group, each pair by itself.  Its first warp runs
// the recurrence of WC channels, LS lanes over the states, CH channels a
// thread; the second turns the rows u, dt into d, d u for it one piece of RP
// rows ahead, and its sums into y one piece behind, a lane owning V adjacent
// channels of a row.  With 16 values a lane there are too few recurrences to
// hide each other's latencies, and the two halves are about equally long.
// The first warps come first, so that each SM quarter gets as many of either
// kind.  What the inner loop draws from shared memory, whose pipe returns 32
// words a clock whatever lanes share, is 2 CH + 2 * 4 words for CH * 4 states.
//
// Measured at 8 x 2048 rows x 4096 channels x 16 states, bf16: 360 us, 3.0e12
// state updates a second, 31 % of what the exponentials alone would allow;
// 119 instructions a row and warp at 66 % of the issue slots where two blocks
// share an SM (256 blocks leave 16 % of the slots empty).  One warp doing both
// halves: 516 us; with 2 channels a thread, twice the warps and words: 685 us;
// blocks of one or two pairs: 498 and 441 us.
constexpr int scan_ch(int ls) { return ls == 2 ? 2 : 4; }
constexpr int kPairs = 4;
constexpr int scan_channels(int ls) { return kPairs * (32 / ls) * scan_ch(ls); }
constexpr int kResident = 2;  // blocks that registers and shared memory let an SM hold
template <int LS_, typename T, bool kWide>
struct Lay {
  static constexpr int LS = LS_, CH = scan_ch(LS), NP = 4 * LS;
  static constexpr int kBlock = 64 * kPairs;
  static constexpr int WC = 32 / LS * CH, DB = kPairs * WC;
  static constexpr int RP = 8, V = WC >= 8 ? WC / 4 : 2;
  static constexpr int COLS = WC / V, kActive = RP * COLS;  // lanes that own values
  static constexpr int kRow = WC + 4;  // pitch of d, d u
  // pitches of the lanes' shares of o: 8 lanes' 16-byte accesses miss each
  // other's banks
  static constexpr int kYLane = LS == 2 ? 48 : LS == 4 ? 40 : LS == 32 ? 4 : WC + 4;
  static constexpr int kYRow = LS * kYLane + 4;
  static constexpr int kRaw = Raw<T, V, !kWide>::kWords;
  // pieces of raw rows: one behind, the current one, and two ahead, or one
  // where they would leave no room for a second block
  static constexpr int kRing = kRaw * V > 32 ? 3 : 4;
  // shared memory, in floats
  static constexpr int kBC = RP * NP;  // a piece of B or C
  static constexpr int kPairFloats =
      4 * kBC + 2 * WC + 2 * (2 * RP * kRow + RP * kYRow) + kRing * 3 * kActive * kRaw;
  static constexpr int kFloats = kPairs * kPairFloats;
};

// The two warps of a pair meet.
__device__ __forceinline__ void meet(int pair) {
  asm volatile("bar.sync %0, 64;" ::"r"(pair + 1) : "memory");
}

__device__ __forceinline__ void copy_async(uint32_t *to, const void *from, int bytes) {
  const uint32_t s = (uint32_t)__cvta_generic_to_shared(to);
  if (bytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
  else if (bytes == 8)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(s), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(from) : "memory");
}

// The exponent of a decay: d A (d times log2 e), and what the special function
// unit falls short of on the mean: 1.5e-8 to 2.7e-8 of its result for arguments
// from -1 to -2^-8 (2^23 arguments an octave against 64 bits), so a state that
// lives for a hundred rows would be a hundred times that off.  With it the
// gradient of A is 8.3e-7 off 64 bits at 8 x 2048 x 4096 x 16, 1.9e-6 without.
// 2^kShort rounds to 1: d = 0 leaves a state as it is.
constexpr float kShort = 2.2e-8f;
__device__ __forceinline__ float2 exponent(float2 d, float2 A) {
  return __ffma2_rn(d, A, make_float2(kShort, kShort));
}
// h <- 2^e h + b.  The decays come out of the special function unit one by one;
// packing them for one product costs more moves than two products do.
__device__ __forceinline__ float2 decay_add(float2 e, float2 h, float2 b) {
  return make_float2(fmaf(exp2_fast(e.x), h.x, b.x), fmaf(exp2_fast(e.y), h.y, b.y));
}
// 2^e h
__device__ __forceinline__ float2 decay(float2 e, float2 h) {
  return __fmul2_rn(make_float2(exp2_fast(e.x), exp2_fast(e.y)), h);
}

// Four states of CH channels (pairs of channels packed) from / to an array
// [channels][states], channels from c on of which `count` exist.
template <typename T, int PAIRS>
__device__ __forceinline__ void load_states(float2 (&h)[PAIRS][4], const ScanArgs<T> &a,
                                            const float *base, int n0, int count) {
#pragma unroll
  for (int p = 0; p < PAIRS; ++p) {
    float v[2][4] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (!base || 2 * p + j >= count) continue;
      const float *q = base + (int64_t)(2 * p + j) * a.states;
      if (a.wide_states) {
        const float4 w = n0 < a.states ? *reinterpret_cast<const float4 *>(q + n0)
                                       : make_float4(0.f, 0.f, 0.f, 0.f);
        v[j][0] = w.x, v[j][1] = w.y, v[j][2] = w.z, v[j][3] = w.w;
      } else {
        load4(v[j], q, n0, a.states);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) h[p][i] = make_float2(v[0][i], v[1][i]);
  }
}
template <typename T, int PAIRS>
__device__ __forceinline__ void store_states(const float2 (&h)[PAIRS][4], const ScanArgs<T> &a,
                                             float *base, int n0, int count) {
#pragma unroll
  for (int p = 0; p < PAIRS; ++p)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (2 * p + j >= count) continue;
      float *q = base + (int64_t)(2 * p + j) * a.states;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = j ? h[p][i].y : h[p][i].x;
      if (a.wide_states) {
        if (n0 < a.states) *reinterpret_cast<float4 *>(q + n0) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        store4(q, v, n0, a.states);
      }
    }
}

// The scan of a chunk.  kOutputs: from the carried state, with outputs.
// kState: from a zero start, leaving the chunk's final state and its sum of d
// for the carry.  kAdjoint: the same for the adjoint, whose recurrence is the
// scan's from the last row to the first, with q for d u and C for B, and the
// decay after the sum: c <- a (c + q C).  kWide: rows in words of V values.
enum ScanMode { kOutputs, kState, kAdjoint };
template <typename T, int LS, bool kPacked, ScanMode kMode, bool kWide>
__global__ void __launch_bounds__(64 * kPairs, kResident)
    scan_kernel(ScanArgs<T> a) {
  using L = Lay<LS, T, kWide>;
  using Row = Raw<T, L::V, !kWide>;
  constexpr int kRing = L::kRing, CH = L::CH, PAIRS = CH / 2, V = L::V, RP = L::RP;
  constexpr bool kLocal = kMode != kOutputs, kBack = kMode == kAdjoint;
  extern __shared__ __align__(16) float smem[];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int pair = warp % kPairs;
  float *sbc = smem + pair * L::kPairFloats;           // [2][B, C][RP][states]
  float *sbias = sbc + 4 * L::kBC, *sskip = sbias + L::WC;
  float *sdx = sskip + L::WC;                          // [2][d, x][RP][kRow]
  float *sy = sdx + 4 * RP * L::kRow;                  // [2][RP][kYRow]
  uint32_t *ring = reinterpret_cast<uint32_t *>(sy + 2 * RP * L::kYRow);
  // the last chunk's own final state (first, going back) is of no use
  const Place<L::DB, T> w(a, a.chunks - kLocal, kBack);
  const int64_t c0 = w.c0 + pair * L::WC;
  const int nc = w.nc - pair * L::WC;
  if (nc <= 0) return;  // both warps of the pair
  const int pieces = (w.r1 - w.r0 + RP - 1) / RP;
  // row t of piece i
  auto row_of = [&](int i, int t) {
    return kBack ? w.r1 - 1 - (i * RP + t) : w.r0 + i * RP + t;
  };

  if (warp >= kPairs) {
    // ---- rows into d, d u; sums into y
    const int vr = lane / L::COLS, vc = lane % L::COLS * V;
    const int vcount = lane < L::kActive ? min(V, nc - vc) : 0;
    for (int c = lane; c < L::WC; c += 32) {
      sbias[c] = a.dt_bias && c < nc ? a.dt_bias[c0 + c] : 0.f;
      sskip[c] = a.skip && c < nc ? a.skip[c0 + c] : 0.f;
    }
    __syncwarp();
    const float *bias = sbias + vc, *skip = sskip + vc;
    const Rows<const T> &ru = kBack ? a.dy : a.u;
    const int first = row_of(0, vr);
    const T *pu = ru.at(w.b, first) + c0 + vc, *pd = a.dt.at(w.b, first) + c0 + vc;
    const T *pz = a.gate.p && kMode != kState ? a.gate.at(w.b, first) + c0 + vc : nullptr;
    T *py = kLocal ? nullptr : a.y.at(w.b, first) + c0 + vc;
    constexpr int64_t way = kBack ? -RP : RP;
    const int64_t su = way * ru.row, sdt = way * a.dt.row, sz = way * a.gate.row, so = way * a.y.row;
    const int last = w.r1 - w.r0 - vr;  // this lane's row is in piece i if i RP < last
    auto slot = [&](int i, int which) { return ring + ((i % kRing * 3 + which) * L::kActive + lane) * L::kRaw; };
    // piece i of u, dt, gate on its way to the ring
    Row hold[3];
    auto fetch = [&](int i) {
      const bool in = i * RP < last && vcount > 0;
      if constexpr (kWide) {
        if (in) {
          constexpr int word = L::kRaw % 4 == 0 ? 4 : L::kRaw % 2 == 0 ? 2 : 1;
#pragma unroll
          for (int j = 0; j < L::kRaw; j += word) {
            copy_async(slot(i, 0) + j, reinterpret_cast<const uint32_t *>(pu) + j, word * 4);
            copy_async(slot(i, 1) + j, reinterpret_cast<const uint32_t *>(pd) + j, word * 4);
            if (pz) copy_async(slot(i, 2) + j, reinterpret_cast<const uint32_t *>(pz) + j, word * 4);
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      } else {
        hold[0].template load<false>(pu, in ? vcount : 0);
        hold[1].template load<false>(pd, in ? vcount : 0);
        if (pz) hold[2].template load<false>(pz, in ? vcount : 0);
      }
      pu += su;
      pd += sdt;
      if (pz) pz += sz;
    };
    auto landed = [&](int i) {  // what fetch(i) loaded by value
      if constexpr (!kWide) {
        if (lane >= L::kActive) return;
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int j = 0; j < L::kRaw; ++j) slot(i, k)[j] = hold[k].w[j];
      }
    };
    auto take = [&](int i, int which) {
      Row r;
#pragma unroll
      for (int j = 0; j < L::kRaw; ++j) r.w[j] = slot(i, which)[j];
      return r;
    };
    // B and C of a piece: quads of states, each of a lane's 32 / LS rows
    // further down than the one before
    constexpr int kItems = RP * LS, kBatch = kItems < 64 ? 1 : 2, kDown = 32 / LS;
    Raw<T, 4> qb[kBatch], qc[kBatch];
    const int qr = lane / LS, qn = lane % LS * 4, rows = w.r1 - w.r0;
    const int quad = lane < kItems ? min(4, a.states - qn) : 0;
    const int64_t of_group = (int64_t)w.g * a.states + qn;
    const Rows<const T> &rb = kBack ? a.C : a.B;
    const T *pb = rb.at(w.b, row_of(0, qr)) + of_group;
    const T *pc = kLocal ? nullptr : a.C.at(w.b, row_of(0, qr)) + of_group;
    const int64_t sb = way * rb.row, sc = way * a.C.row;
    // in order of i and base, so that the pointers follow
    auto load_bc = [&](int i, int base) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int down = (base / 32 + j) * kDown;
        const int count = i * RP + qr + down < rows ? quad : 0;
        const T *from = pb + (kBack ? -down : down) * (int64_t)rb.row;
        if (a.wide_bc) qb[j].template load<true>(from, count);
        else qb[j].template load<false>(from, count);
        if (kLocal) continue;
        from = pc + (kBack ? -down : down) * (int64_t)a.C.row;
        if (a.wide_bc) qc[j].template load<true>(from, count);
        else qc[j].template load<false>(from, count);
      }
      if (base + kBatch * 32 >= kItems) {
        pb += sb;
        if (!kLocal) pc += sc;
      }
    };
    auto store_bc = [&](int i, int base) {
      float4 *to = reinterpret_cast<float4 *>(sbc + i % 2 * 2 * L::kBC);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int item = base + j * 32 + lane;
        if (item >= kItems) continue;  // fewer than one a lane
        float2 v0 = qb[j].pair(0), v1 = qb[j].pair(1);
        to[item] = make_float4(v0.x, v0.y, v1.x, v1.y);
        if (kLocal) continue;
        v0 = qc[j].pair(0), v1 = qc[j].pair(1);
        to[kItems + item] = make_float4(v0.x, v0.y, v1.x, v1.y);
      }
    };
    auto stage = [&](int i) {
      if (lane >= L::kActive) return;
      const Row u = take(i, 0), dt = take(i, 1);
      float *od = sdx + i % 2 * 2 * RP * L::kRow + vr * L::kRow + vc, *ox = od + RP * L::kRow;
      float2 d[V / 2], x[V / 2];
#pragma unroll
      for (int v = 0; v < V / 2; ++v) {
        d[v] = __fadd2_rn(dt.pair(v), *reinterpret_cast<const float2 *>(bias + 2 * v));
        if (a.softplus) d[v] = softplus2(d[v]);
        x[v] = u.pair(v);
        if (!kBack) x[v] = __fmul2_rn(d[v], x[v]);
        else if (pz) x[v] = __fmul2_rn(x[v], silu2(take(i, 2).pair(v)));
        d[v] = __fmul2_rn(d[v], make_float2(kLog2e, kLog2e));
      }
#pragma unroll
      for (int v = 0; v < V / 2; ++v) {
        if constexpr (V == 2) {
          *reinterpret_cast<float2 *>(od) = d[0];
          *reinterpret_cast<float2 *>(ox) = x[0];
        } else if (v % 2 == 0) {
          *reinterpret_cast<float4 *>(od + 2 * v) = make_float4(d[v].x, d[v].y, d[v + 1].x, d[v + 1].y);
          *reinterpret_cast<float4 *>(ox + 2 * v) = make_float4(x[v].x, x[v].y, x[v + 1].x, x[v + 1].y);
        }
      }
    };
    auto finish = [&](int i) {
      if (lane >= L::kActive) return;
      const Row u = take(i, 0), z = take(i, 2);
      const float *from = sy + i % 2 * RP * L::kYRow + vr * L::kYRow + vc;
      float2 o[V / 2];
#pragma unroll
      for (int v = 0; v < V / 2; ++v)
        o[v] = __fmul2_rn(*reinterpret_cast<const float2 *>(skip + 2 * v), u.pair(v));
#pragma unroll
      for (int q = 0; q < LS; ++q)
#pragma unroll
        for (int v = 0; v < V / 2; ++v) {
          if constexpr (V == 2) {
            o[0] = __fadd2_rn(o[0], *reinterpret_cast<const float2 *>(from + q * L::kYLane));
          } else if (v % 2 == 0) {
            const float4 y4 = *reinterpret_cast<const float4 *>(from + q * L::kYLane + 2 * v);
            o[v] = __fadd2_rn(o[v], make_float2(y4.x, y4.y));
            o[v + 1] = __fadd2_rn(o[v + 1], make_float2(y4.z, y4.w));
          }
        }
      Row out;
#pragma unroll
      for (int v = 0; v < V / 2; ++v) {
        if (pz) o[v] = __fmul2_rn(o[v], silu2(z.pair(v)));
        out.set(v, o[v]);
      }
      out.template store<kWide>(py, i * RP < last ? vcount : 0);
      py += so;
    };
    auto ready = [&]() {
      if constexpr (kWide) asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
    };
#pragma unroll 1
    for (int i = 0; i < kRing - 1; ++i) {
      fetch(i);
      landed(i);
    }
    load_bc(0, 0);
    ready();
    stage(0);
#pragma unroll 1
    for (int base = 0; base < kItems; base += kBatch * 32) {
      if (base > 0) load_bc(0, base);
      store_bc(0, base);
    }
    meet(pair);
#pragma unroll 1
    for (int i = 0; i <= pieces; ++i) {
      const bool more = i + 1 < pieces;
      if (more) load_bc(i + 1, 0);
      if (!kLocal && i > 0) finish(i - 1);
      fetch(i + kRing - 1);
      if (more) {
        ready();
        stage(i + 1);
#pragma unroll 1
        for (int base = 0; base < kItems; base += kBatch * 32) {
          if (base > 0) load_bc(i + 1, base);
          store_bc(i + 1, base);
        }
      }
      landed(i + kRing - 1);
      meet(pair);
    }
    return;
  }

  // ---- the recurrence
  const int sl = lane % LS, n0 = sl * 4, ch0 = lane / LS * CH, count = nc - ch0;
  const int64_t at = c0 + ch0, state0 = (w.b * a.chunks + w.k) * a.channels + at;
  float2 A[PAIRS][4], h[PAIRS][4], dsum[PAIRS];
  load_states(A, a, a.A + at * a.states, n0, count);
#pragma unroll
  for (int p = 0; p < PAIRS; ++p) dsum[p] = make_float2(0.f, 0.f);
  const float *start = nullptr;
  const float *ends = kBack ? a.dlast : a.state;  // what sequences start from
  if (!kPacked && (kBack ? w.r1 == a.rows : w.k == 0))
    start = ends ? ends + (w.b * a.channels + at) * a.states : nullptr;
  else if (!kLocal && w.k > 0)
    start = a.carry + state0 * a.states;
  load_states(h, a, start, n0, count);
  meet(pair);
#pragma unroll 1
  for (int i = 0; i <= pieces; ++i) {
    if (i == pieces) {
      meet(pair);
      break;
    }
    const int row0 = row_of(i, 0);
    const int rows = min(RP, w.r1 - w.r0 - i * RP);
    uint32_t opens = 0;  // rows of the piece where a sequence opens (going back: ends)
    if (kPacked) {
      const int r = row_of(i, lane);
      bool o = lane < rows;
      if (kBack) o = o && (r + 1 == a.rows || a.row_seq[r] != a.row_seq[r + 1]);
      else o = o && (r == 0 || a.row_seq[r] != a.row_seq[r - 1]);
      opens = __ballot_sync(~0u, o);
    }
    const float *sd = sdx + i % 2 * 2 * RP * L::kRow + ch0, *sx = sd + RP * L::kRow;
    const float4 *sB = reinterpret_cast<const float4 *>(sbc + i % 2 * 2 * L::kBC) + sl,
                 *sC = sB + RP * LS;
    float *to = sy + i % 2 * RP * L::kYRow + sl * L::kYLane + ch0;
    auto mark = [&](int t) {
      if (kLocal || !a.marks || (uint32_t)(row0 + t) % kMark != 0) return;
      const int64_t marks = (a.rows + kMark - 1) / kMark, m = (uint32_t)(row0 + t) / kMark;
      store_states(h, a, a.marks + ((w.b * marks + m) * a.channels + at) * a.states, n0, count);
    };
    auto open = [&](int t) {
      const int r = row_of(i, t);
      const int s = a.row_seq[r], before = !kBack && r > 0 ? a.row_seq[r - 1] : -1;
      if (!kLocal && a.last && before >= 0)
        store_states(h, a, a.last + (before * a.channels + at) * a.states, n0, count);
      load_states(h, a, ends && s >= 0 ? ends + (s * a.channels + at) * a.states : nullptr, n0,
                  count);
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) dsum[p] = make_float2(0.f, 0.f);
    };
    auto step = [&](int t, float2 (&y)[PAIRS]) {
      float2 d[PAIRS], x[PAIRS];
      if constexpr (CH == 4) {
        const float4 d4 = *reinterpret_cast<const float4 *>(sd + t * L::kRow);
        const float4 x4 = *reinterpret_cast<const float4 *>(sx + t * L::kRow);
        d[0] = make_float2(d4.x, d4.y), d[PAIRS - 1] = make_float2(d4.z, d4.w);
        x[0] = make_float2(x4.x, x4.y), x[PAIRS - 1] = make_float2(x4.z, x4.w);
      } else {
        d[0] = *reinterpret_cast<const float2 *>(sd + t * L::kRow);
        x[0] = *reinterpret_cast<const float2 *>(sx + t * L::kRow);
      }
      const float4 B4 = sB[t * LS];
      const float B[4] = {B4.x, B4.y, B4.z, B4.w};
      float4 C4 = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!kLocal) C4 = sC[t * LS];
      const float C[4] = {C4.x, C4.y, C4.z, C4.w};
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        if (kLocal) dsum[p] = __fadd2_rn(dsum[p], d[p]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 e = exponent(d[p], A[p][j]);
          const float2 b = make_float2(B[j], B[j]);
          h[p][j] = kBack ? decay(e, __ffma2_rn(x[p], b, h[p][j]))
                          : decay_add(e, h[p][j], __fmul2_rn(x[p], b));
          if (kLocal) continue;
          const float2 c = make_float2(C[j], C[j]);
          y[p] = j == 0 ? __fmul2_rn(c, h[p][j]) : __ffma2_rn(c, h[p][j], y[p]);
        }
      }
    };
    auto share = [&](int t, const float2 (&y)[PAIRS]) {
      if constexpr (CH == 4)
        *reinterpret_cast<float4 *>(to + t * L::kYRow) =
            make_float4(y[0].x, y[0].y, y[PAIRS - 1].x, y[PAIRS - 1].y);
      else
        *reinterpret_cast<float2 *>(to + t * L::kYRow) = y[0];
    };
    if (rows < RP || opens != 0) {
      for (int t = 0; t < rows; ++t) {
        mark(t);
        if (kPacked && (opens >> t & 1)) open(t);
        float2 y[PAIRS];
        step(t, y);
        if (!kLocal) share(t, y);
      }
    } else {
      // a few rows at a time, their loads ahead of all stores
      constexpr int R = 4;
#pragma unroll
      for (int t = 0; t < RP; t += R) {
        mark(t);
        float2 y[R][PAIRS];
#pragma unroll
        for (int j = 0; j < R; ++j) step(t + j, y[j]);
        if constexpr (!kLocal) {
#pragma unroll
          for (int j = 0; j < R; ++j) share(t + j, y[j]);
        }
      }
    }
    meet(pair);
  }
  if (kLocal) {
    store_states(h, a, a.carry + state0 * a.states, n0, count);
    if (sl == 0)
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        if (2 * p < count) a.sum_d[state0 + 2 * p] = dsum[p].x;
        if (2 * p + 1 < count) a.sum_d[state0 + 2 * p + 1] = dsum[p].y;
      }
  } else if (a.last && w.r1 == a.rows) {
    const int s = kPacked ? a.row_seq[a.rows - 1] : (int)w.b;
    if (s >= 0) store_states(h, a, a.last + (s * a.channels + at) * a.states, n0, count);
  }
}

// A thousandth of the scan's work, but a chain: latency bounds it.
// carry[k] <- the state that enters chunk k (kBack: the adjoint that enters
// it from below), from each chunk's own contribution in carry[k].  One thread
// a state; the chunks' loads go ahead in fours of the chain that joins them.
template <typename T, bool kBack>
__global__ void carry_kernel(ScanArgs<T> a) {
  const int64_t per = a.channels * a.states;
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= per) return;
  const int64_t c = at / a.states;
  const float A = a.A[at];
  for (int64_t b = blockIdx.y; b < a.batches; b += gridDim.y) {
    float h = 0.f;
    for (int j0 = 0; j0 < a.chunks; j0 += 4) {
      float own[4], sum[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // the last chunk of the walk has left nothing, and nothing needs it
        const int k = kBack ? a.chunks - 1 - (j0 + j) : j0 + j;
        const bool in = j0 + j < a.chunks - 1;
        own[j] = in ? a.carry[(b * a.chunks + k) * per + at] : 0.f;
        sum[j] = in ? a.sum_d[(b * a.chunks + k) * a.channels + c] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j0 + j >= a.chunks) break;
        const int k = kBack ? a.chunks - 1 - (j0 + j) : j0 + j;
        const int r0 = k * a.chunk_rows, r1 = chunk_end(r0, a.chunk_rows, a.rows);
        // does a sequence open (close, going back) within the chunk?
        bool cut;
        if (kBack) cut = r1 == a.rows || (a.row_seq && a.row_seq[r0] != a.row_seq[r1]);
        else cut = r0 == 0 || (a.row_seq && a.row_seq[r0 - 1] != a.row_seq[r1 - 1]);
        a.carry[(b * a.chunks + k) * per + at] = h;
        h = cut || h == 0.f ? own[j] : fmaf(exp2_fast(A * sum[j]), h, own[j]);
      }
    }
  }
}

// One token: LS lanes per channel, 4 states each, the cache in place: 16
// bytes a lane read and written, nearly all that it does.  NB batch entries
// at once, on their way together; what is one value a row and channel (d, d u,
// the gate) is done for one entry by each NB-th part of the lanes.  512 entries x
// 4096 channels x 16 states: 53 us, 5.4 TB/s; one entry at a time, with that
// work in every lane, 83 us.
//
// Up to 65535 blocks below each other step by NB <= 4 entries each, counted in
// 32 bits: kMostEntries leaves room for the step past the last one.
constexpr int kMostEntries = INT32_MAX - 4 * 65535;
template <typename T, int LS, int NB, bool kWide>
__global__ void __launch_bounds__(kScanThreads) scan_step_kernel(ScanArgs<T> a) {
  constexpr int kShare = LS / NB;  // lanes of a channel for one entry's values
  const int64_t c = ((int64_t)blockIdx.x * kScanThreads + threadIdx.x) / LS;
  const int lane = threadIdx.x % 32, sl = lane % LS, n0 = sl * 4, first = lane - sl;
  const bool here = c < a.channels;
  const int n = here ? min(4, a.states - n0) : 0;
  const int64_t g = (unsigned)c / (unsigned)a.per_group * (int64_t)a.states + n0;
  const int64_t entry = a.channels * a.states;
  float *at = a.last + c * a.states + n0;
  Raw<float, 4> A;
  A.template load<kWide>(a.A + c * a.states + n0, n);
  const float bias = here && a.dt_bias ? a.dt_bias[c] : 0.f;
  const float skip = here && a.skip ? a.skip[c] : 0.f;
  for (int b0 = blockIdx.y * NB; b0 < a.sequences; b0 += gridDim.y * NB) {
    Raw<float, 4> h[NB];
    Raw<T, 4> B[NB], C[NB];
    float *cache[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int b = b0 + i;
      const int slot = b >= a.sequences ? -1 : a.slots ? a.slots[b] : b;
      const bool live = slot >= 0 && slot < a.num_slots;
      cache[i] = live ? at + slot * entry : nullptr;
      h[i].template load<kWide>(cache[i], live ? n : 0);
      B[i].template load<kWide>(a.B.at(0, b) + g, live ? n : 0);
      C[i].template load<kWide>(a.C.at(0, b) + g, live ? n : 0);
    }
    const int mine = sl / kShare, b = b0 + mine;  // this lane's entry
    const bool in = here && b < a.sequences;
    const float u = in ? to_f(a.u.at(0, b)[c]) : 0.f;
    const float z = in && a.gate.p ? to_f(a.gate.at(0, b)[c]) : 0.f;
    const float d = step_of(a, in ? to_f(a.dt.at(0, b)[c]) : 0.f, bias), x = d * u;
    float o[NB];
    bool live = false;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const float di = __shfl_sync(~0u, d, first + i * kShare) * kLog2e;
      const float xi = __shfl_sync(~0u, x, first + i * kShare);
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 v = decay_add(exponent(make_float2(di, di), A.pair(j)), h[i].pair(j),
                                   __fmul2_rn(make_float2(xi, xi), B[i].pair(j)));
        h[i].set(j, v);
        sum = __ffma2_rn(C[i].pair(j), v, sum);
      }
      o[i] = sum.x + sum.y;
      if (cache[i]) h[i].template store<kWide>(cache[i], n);
      if (i == mine) live = cache[i] != nullptr;
    }
    reduce_scatter<NB, LS, 1>(o, lane);
    if (!in || sl % kShare != 0) continue;
    float y = fmaf(skip, u, o[0]);
    if (a.gate.p) y *= silu(z);
    a.y.at(0, b)[c] = from_f<T>(live ? y : 0.f);
  }
}

// ---------------------------------------------------------------- gradient
// How the gradient kernel is laid out: blocks of four pairs of warps, as the
// forward kernel's, over tiles of kMark rows from the last to the first.  The
// first warp of a pair recomputes a tile's states from its mark, down the
// rows, and puts each into tensor memory, its own lane's columns -- 16 rows x
// 16 states of fp32 a thread are more than its registers or shared memory hold
// -- then walks the adjoint up.  The second warp turns u, dt, gate, dy into d,
// d u, q for the next tile and the sums o, r, v (in their places) into du,
// ddt, dgate for the one before.  Two blocks fill an SM and its tensor memory.
//
// Measured at 8 x 2048 rows x 4096 channels x 16 states, bf16: 1224 us, of which
// the first warps alone take 1000: three quarters of the 380 instructions a row
// and warp, at 59 % of the issue slots.  FMA pipe alone: 360 us.  States kept every fourth
// row in shared memory and recomputed twice instead of once: 3960 us.
template <int LS_, typename T>
struct GradLay {
  static constexpr int LS = LS_, CH = scan_ch(LS), NP = 4 * LS, E = 4 * CH, CL = 32 / LS;
  static constexpr int kPairs = 4, kBlock = 64 * kPairs;
  static constexpr int WC = CL * CH, DB = kPairs * WC;
  static constexpr int V = LS <= 8 ? 8 : LS == 16 ? 4 : 2;
  static constexpr int COLS = WC / V, RP = 32 / COLS, PASSES = kMark / RP;
  static constexpr int kColumns = kMark * E;  // of tensor memory
  // shared memory, in floats
  static constexpr int kRow = WC + 4;
  static constexpr int kPlane = kMark * kRow;         // d, d u or q of a tile
  static constexpr int kBC = kMark * NP;              // B or C of a tile
  static constexpr int kPairFloats = 2 * (3 * kPlane + 2 * kBC) + 2 * WC;
  static constexpr int kThreadFloats = 2 * E;         // a first warp's thread: mark, sum of dA
  static constexpr int kLaneFloats = 2 * V;           // a second warp's: sums of dskip, dbias
  static constexpr int kLanesAt = 4 + 4 * kBC + kPairs * (kPairFloats + 32 * kThreadFloats);
  static constexpr int kFloats = kLanesAt + kPairs * 32 * kLaneFloats;
};
// Tiles whose shares of dA, dskip and dbias are summed before they join the
// rest: a thread's rows in one fp32 chain would lose a bit every time their
// number grows fourfold (2^17 rows of equal terms: 1.6e-4 off, 1e-5 so).
constexpr int kFlush = 8;
constexpr int grad_channels(int ls) { return 4 * (32 / ls) * scan_ch(ls); }
constexpr int grad_resident(int ls) { return ls <= 8 ? 2 : 1; }

template <int E>
__device__ __forceinline__ void tmem_put(uint32_t at, const float2 (&h)[E / 8][4]) {
  float v[E];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) v[2 * i] = h[i / 4][i % 4].x, v[2 * i + 1] = h[i / 4][i % 4].y;
  if constexpr (E == 16) tmem_st16(at, v);
  else tmem_st8u(at, reinterpret_cast<const uint32_t *>(v));
}
template <int E>
__device__ __forceinline__ void tmem_get(uint32_t at, float2 (&h)[E / 8][4]) {
  float v[E];
  if constexpr (E == 16) tmem_ld16(at, v);
  else tmem_ld8(at, v);
#pragma unroll
  for (int i = 0; i < E / 2; ++i) h[i / 4][i % 4] = make_float2(v[2 * i], v[2 * i + 1]);
}

template <typename T, int LS, bool kPacked, bool kWide>
__global__ void __launch_bounds__(256, grad_resident(LS)) scan_grad_kernel(ScanArgs<T> a) {
  using L = GradLay<LS, T>;
  constexpr int CH = L::CH, PAIRS = CH / 2, V = L::V, E = L::E;
  extern __shared__ __align__(16) float smem[];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, pair = warp % L::kPairs;
  float *sBC = smem + 4;                                       // [2][B, C][row][states]
  float *own = sBC + 4 * L::kBC + pair * L::kPairFloats;
  float *sdxq = own;                                           // [2][d, x, q][row][kRow]
  float *ssum = own + 6 * L::kPlane;                           // [2][row][dB, dC][states]
  float *sbias = ssum + 4 * L::kBC, *sskip = sbias + L::WC;
  const Place<L::DB, T> w(a, a.chunks, 0);
  const int64_t c0 = w.c0 + pair * L::WC;
  const int nc = w.nc - pair * L::WC;
  const int tiles = (w.r1 - w.r0 + kMark - 1) / kMark;
  const int64_t part = w.b * a.chunks + w.k;
  // the i-th tile of the walk up, and its rows
  auto row_of = [&](int i) { return w.r0 + (tiles - 1 - i) * kMark; };
  if (warp == 0) tmem_alloc(smem_u32(smem), L::kColumns);

  if (warp >= L::kPairs) {
    // ---- rows in and out
    const int vr = lane / L::COLS, vc = lane % L::COLS * V, vcount = min(V, nc - vc);
    const int me = threadIdx.x - 32 * L::kPairs;  // of the second warps
    for (int c = lane; c < L::WC; c += 32) {
      sbias[c] = a.dt_bias && c < nc ? a.dt_bias[c0 + c] : 0.f;
      sskip[c] = a.skip && c < nc ? a.skip[c0 + c] : 0.f;
    }
    __syncwarp();
    const float *bias = sbias + vc, *skip = sskip + vc;
    const bool gated = a.gate.p != nullptr;
    float2 dskip[V / 2], dbias[V / 2];
#pragma unroll
    for (int v = 0; v < V / 2; ++v) dskip[v] = dbias[v] = make_float2(0.f, 0.f);
    // their sums over earlier tiles, this lane's alone
    float4 *sums = reinterpret_cast<float4 *>(smem + L::kLanesAt) + pair * 32 * (V / 2) + lane;
#pragma unroll
    for (int v = 0; v < V / 2; ++v) sums[32 * v] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto flush = [&]() {
#pragma unroll
      for (int v = 0; v < V / 2; ++v) {
        const float4 s = sums[32 * v];
        sums[32 * v] = make_float4(s.x + dskip[v].x, s.y + dskip[v].y, s.z + dbias[v].x,
                                   s.w + dbias[v].y);
        dskip[v] = dbias[v] = make_float2(0.f, 0.f);
      }
    };
    struct In {
      Raw<T, V, !kWide> u, dt, z, dy;
    };
    // this lane's first row of the tile that the first warps are at
    const int row = row_of(0) + vr;
    const T *pu = a.u.at(w.b, row) + c0 + vc, *pd = a.dt.at(w.b, row) + c0 + vc,
            *pz = gated ? a.gate.at(w.b, row) + c0 + vc : nullptr,
            *py = a.dy.at(w.b, row) + c0 + vc;
    // pass `pass` of the tile `to` tiles further up
    auto load = [&](In &in, int i, int to, int pass) {
      const int up = to * kMark - pass * L::RP;
      const int r = row_of(i + to) + pass * L::RP + vr;
      const int count = i + to >= 0 && i + to < tiles && r < w.r1 ? vcount : 0;
      in.u.template load<kWide>(pu - (int64_t)up * a.u.row, count);
      in.dt.template load<kWide>(pd - (int64_t)up * a.dt.row, count);
      if (gated) in.z.template load<kWide>(pz - (int64_t)up * a.gate.row, count);
      in.dy.template load<kWide>(py - (int64_t)up * a.dy.row, count);
    };
    auto stage = [&](const In &in, int i, int pass) {
      float *o = sdxq + i % 2 * 3 * L::kPlane + (pass * L::RP + vr) * L::kRow + vc;
#pragma unroll
      for (int v = 0; v < V / 2; ++v) {
        float2 d = __fadd2_rn(in.dt.pair(v), *reinterpret_cast<const float2 *>(bias + 2 * v));
        if (a.softplus) d = softplus2(d);
        float2 q = in.dy.pair(v);
        if (gated) q = __fmul2_rn(q, silu2(in.z.pair(v)));
        *reinterpret_cast<float2 *>(o + 2 * v) = __fmul2_rn(d, make_float2(kLog2e, kLog2e));
        *reinterpret_cast<float2 *>(o + L::kPlane + 2 * v) = __fmul2_rn(d, in.u.pair(v));
        *reinterpret_cast<float2 *>(o + 2 * L::kPlane + 2 * v) = q;
      }
    };
    auto finish = [&](const In &in, int i, int pass) {
      const float *from = sdxq + i % 2 * 3 * L::kPlane + (pass * L::RP + vr) * L::kRow + vc;
      const int r = row_of(i) + pass * L::RP + vr;
      const int count = r < w.r1 ? vcount : 0;
      Raw<T, V, !kWide> du, ddt, dz;
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        const float2 v = *reinterpret_cast<const float2 *>(from + 2 * k);
        const float2 o = *reinterpret_cast<const float2 *>(from + L::kPlane + 2 * k);
        const float2 rr = *reinterpret_cast<const float2 *>(from + 2 * L::kPlane + 2 * k);
        const float2 s2 = *reinterpret_cast<const float2 *>(skip + 2 * k);
        const float2 u = in.u.pair(k), dy = in.dy.pair(k);
        const float2 raw = __fadd2_rn(in.dt.pair(k), *reinterpret_cast<const float2 *>(bias + 2 * k));
        const float2 d = a.softplus ? softplus2(raw) : raw;
        float2 q = dy;
        if (gated) {
          const float2 z = in.z.pair(k);
          const float2 s = make_float2(sigmoid(z.x), sigmoid(z.y));
          const float2 zs = __fmul2_rn(z, s);
          q = __fmul2_rn(dy, zs);
          // (z s)' = s + z s (1 - s)
          const float2 ds = __ffma2_rn(zs, make_float2(1.f - s.x, 1.f - s.y), s);
          dz.set(k, __fmul2_rn(__fmul2_rn(dy, __ffma2_rn(s2, u, o)), ds));
        }
        float2 g = __ffma2_rn(rr, u, v);
        if (a.softplus) g = __fmul2_rn(g, make_float2(sigmoid(raw.x), sigmoid(raw.y)));
        du.set(k, __ffma2_rn(rr, d, __fmul2_rn(s2, q)));
        ddt.set(k, g);
        if (count > 0) {
          dskip[k] = __ffma2_rn(q, u, dskip[k]);
          dbias[k] = __fadd2_rn(dbias[k], g);
        }
      }
      du.template store<kWide>(a.du.at(w.b, r) + c0 + vc, count);
      ddt.template store<kWide>(a.ddt.at(w.b, r) + c0 + vc, count);
      if (gated && a.dgate.p) dz.template store<kWide>(a.dgate.at(w.b, r) + c0 + vc, count);
    };
    auto stage_bc = [&](int i) {
      constexpr int items = kMark * LS;  // quads of B, then of C
      const int row0 = row_of(i);
      for (int item = me; item < 2 * items; item += 32 * L::kPairs) {
        const int which = item / items, t = item % items / LS, n = item % LS * 4;
        const Rows<const T> &src = which ? a.C : a.B;
        const int r = row0 + t;
        const int count = r < w.r1 ? min(4, a.states - n) : 0;
        const T *from = src.at(w.b, r) + (int64_t)w.g * a.states + n;
        Raw<T, 4> q;
        if (a.wide_bc) q.template load<true>(from, count);
        else q.template load<false>(from, count);
        const float2 v0 = q.pair(0), v1 = q.pair(1);
        reinterpret_cast<float4 *>(sBC + i % 2 * 2 * L::kBC)[item] =
            make_float4(v0.x, v0.y, v1.x, v1.y);
      }
    };
    // the block's shares of dB, dC: its four first warps' sums, in order
    // A lane's values keep their column where a row has at most 128 of them.
    constexpr int kCols = 2 * L::NP, kLanes = 32 * L::kPairs;
    const int live = min(L::kPairs, (w.nc + L::WC - 1) / L::WC);
    const int64_t pitch = (int64_t)a.groups * 2 * a.states;
    float *shares = a.bc_parts + (((int64_t)w.cb * a.batches + w.b) * a.rows) * pitch +
                    (int64_t)w.g * 2 * a.states;
    auto share_bc = [&](int i) {
      const int row0 = row_of(i), rows = min(kMark, w.r1 - row0);
      const float *from = sBC + 4 * L::kBC + 6 * L::kPlane + i % 2 * 2 * L::kBC;
      for (int col = me % kCols; col < kCols; col += kLanes) {
        const int n = col % L::NP, which = col / L::NP;
        if (n >= a.states) continue;
        float *to = shares + row0 * pitch + which * a.states + n;
        for (int t = me / kCols; t < rows; t += kCols < kLanes ? kLanes / kCols : 1) {
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < L::kPairs; ++k)
            if (k < live) s += from[k * L::kPairFloats + t * kCols + col];
          to[t * pitch] = s;
        }
      }
    };
    // the passes of an iteration: those of the tile behind, then those of the
    // one ahead, each loaded while the one before is worked on
    In in[2];
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) {
      load(in[0], 0, 0, p);
      stage(in[0], 0, p);
    }
    stage_bc(0);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i <= tiles; ++i) {
      constexpr int jobs = 2 * L::PASSES;
      load(in[0], i, -1, 0);
#pragma unroll
      for (int j = 0; j < jobs; ++j) {
        const int to = j < L::PASSES ? -1 : 1, pass = j % L::PASSES;
        if (j + 1 < jobs) load(in[(j + 1) % 2], i, j + 1 < L::PASSES ? -1 : 1, (j + 1) % L::PASSES);
        if (to < 0 && i > 0) finish(in[j % 2], i - 1, pass);
        if (to > 0 && i + 1 < tiles) stage(in[j % 2], i + 1, pass);
      }
      if (i % kFlush == 0) flush();
      if (i > 0) share_bc(i - 1);
      if (i + 1 < tiles) stage_bc(i + 1);
      pu -= (int64_t)kMark * a.u.row;
      pd -= (int64_t)kMark * a.dt.row;
      if (gated) pz -= (int64_t)kMark * a.gate.row;
      py -= (int64_t)kMark * a.dy.row;
      __syncthreads();
    }
    // a channel's shares lie in the lanes of its column
    flush();
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const float4 sum = sums[32 * k];
      dskip[k] = make_float2(sum.x, sum.y), dbias[k] = make_float2(sum.z, sum.w);
#pragma unroll
      for (int s = L::COLS; s < 32; s *= 2) {
        dskip[k].x += __shfl_xor_sync(~0u, dskip[k].x, s);
        dskip[k].y += __shfl_xor_sync(~0u, dskip[k].y, s);
        dbias[k].x += __shfl_xor_sync(~0u, dbias[k].x, s);
        dbias[k].y += __shfl_xor_sync(~0u, dbias[k].y, s);
      }
      if (vr != 0) continue;
      const int64_t at = part * a.channels + c0 + vc + 2 * k;
      if (2 * k < vcount && a.skip_parts) a.skip_parts[at] = dskip[k].x;
      if (2 * k + 1 < vcount && a.skip_parts) a.skip_parts[at + 1] = dskip[k].y;
      if (2 * k < vcount && a.bias_parts) a.bias_parts[at] = dbias[k].x;
      if (2 * k + 1 < vcount && a.bias_parts) a.bias_parts[at + 1] = dbias[k].y;
    }
    return;
  }

  // ---- states down, adjoint up
  const int sl = lane % LS, n0 = sl * 4, ch0 = lane / LS * CH, count = nc - ch0;
  const int64_t at = c0 + ch0;
  // this thread's 16-byte slots: its mark, then its sum of dA
  float4 *slots = reinterpret_cast<float4 *>(sBC + 4 * L::kBC + L::kPairs * L::kPairFloats) +
                  warp * 32 * (L::kThreadFloats / 4) + lane;
  float4 *asum = slots + 32 * (E / 4);
  float2 A[PAIRS][4], e[PAIRS][4], dA[PAIRS][4];
  load_states(A, a, a.A + at * a.states, n0, count);
  const float *below = nullptr;
  if (w.r1 < a.rows) below = a.carry + (part * a.channels + at) * a.states;
  else if (!kPacked && a.dlast) below = a.dlast + (w.b * a.channels + at) * a.states;
  load_states(e, a, below, n0, count);
#pragma unroll
  for (int p = 0; p < PAIRS; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) dA[p][i] = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < E / 4; ++j) asum[32 * j] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto flush = [&]() {
#pragma unroll
    for (int p = 0; p < PAIRS; ++p)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        float4 *s = asum + 32 * (p * 2 + i / 2);
        const float4 v = *s;
        *s = make_float4(v.x + dA[p][i].x, v.y + dA[p][i].y, v.z + dA[p][i + 1].x,
                         v.w + dA[p][i + 1].y);
        dA[p][i] = dA[p][i + 1] = make_float2(0.f, 0.f);
      }
  };
  const int64_t marks = (a.rows + kMark - 1) / kMark;
  auto mark_of = [&](int i) {
    return a.marks + ((w.b * marks + (uint32_t)row_of(i) / kMark) * a.channels + at) * a.states;
  };
  // the mark of the i-th tile on its way, one 16-byte copy a channel
  auto fetch_mark = [&](int i) {
    if (!a.wide_states) return;
    if (i < tiles && n0 < a.states) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (c < count)
          copy_async(reinterpret_cast<uint32_t *>(slots + 32 * c),
                     mark_of(i) + (int64_t)c * a.states + n0, 16);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) slots[32 * c] = make_float4(0.f, 0.f, 0.f, 0.f);
  fetch_mark(0);
  __syncthreads();
  const uint32_t column = *reinterpret_cast<volatile uint32_t *>(smem) + ((uint32_t)warp << 21);
#pragma unroll 1
  for (int i = 0; i <= tiles; ++i) {
    if (i == tiles) {
      __syncthreads();
      break;
    }
    const int row0 = row_of(i);
    const int rows = min(kMark, w.r1 - row0);
    const uint32_t opens = kPacked ? opens_mask(a, row0, lane) : 0;
    const uint32_t closes = kPacked ? closes_mask(a, row0, lane) : 0;
    float *sd = sdxq + i % 2 * 3 * L::kPlane, *sx = sd + L::kPlane, *sq = sx + L::kPlane;
    const float4 *sB = reinterpret_cast<const float4 *>(sBC + i % 2 * 2 * L::kBC) + sl,
                 *sC = sB + kMark * LS;
    float *sum = ssum + i % 2 * 2 * L::kBC;
    float2 h[PAIRS][4];
    if (a.wide_states) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        const float4 v0 = slots[32 * 2 * p], v1 = slots[32 * (2 * p + 1)];
        h[p][0] = make_float2(v0.x, v1.x), h[p][1] = make_float2(v0.y, v1.y);
        h[p][2] = make_float2(v0.z, v1.z), h[p][3] = make_float2(v0.w, v1.w);
      }
    } else {
      load_states(h, a, mark_of(i), n0, count);
    }
    auto load2 = [&](float2 (&v)[PAIRS], const float *from, int t) {
      if constexpr (CH == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(from + t * L::kRow + ch0);
        v[0] = make_float2(q.x, q.y), v[PAIRS - 1] = make_float2(q.z, q.w);
      } else {
        v[0] = *reinterpret_cast<const float2 *>(from + t * L::kRow + ch0);
      }
    };
    auto open_state = [&](float2 (&to)[PAIRS][4], int t) {
      const int s = a.row_seq[row0 + t];
      load_states(to, a, a.state && s >= 0 ? a.state + (s * a.channels + at) * a.states : nullptr,
                  n0, count);
    };
    // down the rows: column block t holds the state that enters row t
#pragma unroll 8
    for (int t = 0; t < rows; ++t) {
      tmem_put<E>(column + t * E, h);
      if (kPacked && (opens >> t & 1)) open_state(h, t);
      float2 d[PAIRS], x[PAIRS];
      load2(d, sd, t);
      load2(x, sx, t);
      const float4 B4 = sB[t * LS];
      const float B[4] = {B4.x, B4.y, B4.z, B4.w};
#pragma unroll
      for (int p = 0; p < PAIRS; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 z = exponent(d[p], A[p][j]);
          h[p][j] = decay_add(z, h[p][j], __fmul2_rn(x[p], make_float2(B[j], B[j])));
        }
    }
    tmem_wait_st();
    fetch_mark(i + 1);
    // up the rows: h the state after row t, before the one that enters it
    auto up = [&](int t, const float2 (&h)[PAIRS][4], float2 (&before)[PAIRS][4]) {
      tmem_get<E>(column + t * E, before);
      if (kPacked && (closes >> t & 1)) {
        const int s = a.row_seq[row0 + t];
        load_states(e, a, a.dlast && s >= 0 ? a.dlast + (s * a.channels + at) * a.states : nullptr,
                    n0, count);
      }
      const bool opening = kPacked && (opens >> t & 1);
      float2 d[PAIRS], x[PAIRS], q[PAIRS];
      load2(d, sd, t);
      load2(x, sx, t);
      load2(q, sq, t);
      const float4 B4 = sB[t * LS], C4 = sC[t * LS];
      const float B[4] = {B4.x, B4.y, B4.z, B4.w}, C[4] = {C4.x, C4.y, C4.z, C4.w};
      float bc[8], o[CH], r[CH], v[CH];
      float2 bb[4], cc[4];
      if (kPacked && opening) open_state(before, t);  // the state the sequence starts from
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        float2 oo, rr, vv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 Bj = make_float2(B[j], B[j]), Cj = make_float2(C[j], C[j]);
          const float2 z = exponent(d[p], A[p][j]);
          const float2 ee = __ffma2_rn(Cj, q[p], e[p][j]);
          bb[j] = p == 0 ? __fmul2_rn(x[p], ee) : __ffma2_rn(x[p], ee, bb[j]);
          cc[j] = p == 0 ? __fmul2_rn(q[p], h[p][j]) : __ffma2_rn(q[p], h[p][j], cc[j]);
          rr = j == 0 ? __fmul2_rn(ee, Bj) : __ffma2_rn(ee, Bj, rr);
          oo = j == 0 ? __fmul2_rn(h[p][j], Cj) : __ffma2_rn(h[p][j], Cj, oo);
          e[p][j] = decay(z, ee);
          const float2 g = __fmul2_rn(e[p][j], before[p][j]);
          vv = j == 0 ? __fmul2_rn(g, A[p][j]) : __ffma2_rn(g, A[p][j], vv);
          dA[p][j] = __ffma2_rn(g, d[p], dA[p][j]);
        }
        o[2 * p] = oo.x, o[2 * p + 1] = oo.y;
        r[2 * p] = rr.x, r[2 * p + 1] = rr.y;
        v[2 * p] = vv.x, v[2 * p + 1] = vv.y;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) bc[j] = bb[j].x + bb[j].y, bc[4 + j] = cc[j].x + cc[j].y;
      if (kPacked && opening) tmem_get<E>(column + t * E, before);  // the last one's end again
      if (kPacked && opening && a.dstate && a.row_seq[row0 + t] >= 0)
        store_states(e, a, a.dstate + ((int64_t)a.row_seq[row0 + t] * a.channels + at) * a.states,
                     n0, count);
      reduce_scatter<CH, LS, 1>(o, lane);
      reduce_scatter<CH, LS, 1>(r, lane);
      reduce_scatter<CH, LS, 1>(v, lane);
      reduce_scatter<8, L::CL, LS>(bc, lane);
      __syncwarp();  // the row's d, x, q have been read by all
      if (owner_of<CH, LS>(sl)) {
        constexpr int held = CH > LS ? CH / LS : 1;
        const int to = t * L::kRow + ch0 + first_of<CH, LS>(sl);
#pragma unroll
        for (int k = 0; k < held; ++k) sd[to + k] = v[k], sx[to + k] = o[k], sq[to + k] = r[k];
      }
      if (owner_of<8, L::CL>(lane / LS)) {
        constexpr int held = 8 > L::CL ? 8 / L::CL : 1;
        const int f = first_of<8, L::CL>(lane / LS);
#pragma unroll
        for (int k = 0; k < held; ++k)
          sum[(t * 2 + (f + k) / 4) * L::NP + n0 + (f + k) % 4] = bc[k];
      }
    };
    float2 other[PAIRS][4];
    int t = rows - 1;
#pragma unroll 1
    for (; t > 0; t -= 2) {
      up(t, h, other);
      up(t - 1, other, h);
    }
    if (t == 0) up(0, h, other);
    if (i % kFlush == kFlush - 1) flush();
    __syncthreads();
  }
  flush();
#pragma unroll
  for (int p = 0; p < PAIRS; ++p)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float4 v = asum[32 * (p * 2 + i / 2)];
      // the rows' d came times log2 e
      dA[p][i] = make_float2(v.x * kLn2, v.y * kLn2);
      dA[p][i + 1] = make_float2(v.z * kLn2, v.w * kLn2);
    }
  store_states(dA, a, a.A_parts + (part * a.channels + at) * a.states, n0, count);
  if (!kPacked && a.dstate && w.k == 0)
    store_states(e, a, a.dstate + (w.b * a.channels + at) * a.states, n0, count);
  asm volatile("bar.sync 1, %0;" ::"r"(32 * L::kPairs) : "memory");  // the first warps
  if (warp == 0) tmem_dealloc(*reinterpret_cast<volatile uint32_t *>(smem), L::kColumns);
}

// dB and dC from the channel blocks' shares, in order: a block takes as many
// rows as fit its threads, blockIdx.y the batch entries.  A block's share is an
// fp32 value for each state of dB and of dC, written and read once, for the 128
// channels that it covers up to 16 states, 64, 32 and 16 up to 32, 64 and 128: 8
// bytes times states / channels for each row and channel, 1 at 16 states and 64
// at 128, where they are most of the gradient's traffic.
constexpr int kSumThreads = 256;  // at least the values of a row and group: 2 * 128
template <typename T>
__global__ void __launch_bounds__(kSumThreads) sum_bc_kernel(ScanArgs<T> a) {
  const int per = 2 * a.states, down = threadIdx.x / per, at = threadIdx.x - down * per;
  const int each = kSumThreads / per;  // rows and groups a block takes
  const int which = at >= a.states, n = at - which * a.states;
  const int64_t item = (int64_t)blockIdx.x * each + down;
  if (down >= each || item >= (int64_t)a.rows * a.groups) return;
  const int t = (int)((uint64_t)item / (unsigned)a.groups), g = (int)(item - (int64_t)t * a.groups);
  const int64_t entry = (int64_t)a.rows * a.groups * per;
  for (int64_t b = blockIdx.y; b < a.batches; b += gridDim.y) {
    const float *from = a.bc_parts + b * entry + item * per + at;
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < a.group_blocks; ++k) s += from[k * a.batches * entry];
    const Rows<T> &out = which ? a.dC : a.dB;
    out.at(b, t)[(int64_t)g * a.states + n] = from_f<T>(s);
  }
}

// ------------------------------------------------------------- host side
enum ScanCall { kScan, kScanGrad, kScanStep };

inline int lanes_of(int64_t states) {
  int ls = 2;
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
