// gated_scan.cu -- the gated linear recurrence, its gradient and its
// single-token form (include/tcu_seq.h).
//
// Per sequence and channel, s(v) = 1 / (1 + exp(-v)):
//     L_t = -rate s(forget_t),   a_t = exp(L_t),   m_t = sqrt(1 - a_t^2)
//     h_t = a_t h_{t-1} + m_t s(admit_t) x_t,      y_t = h_t
//     e_t = dy_t + a_{t+1} e_{t+1}  (the gradient of h_t; dlast enters at the end)
//     dx_t = e_t m_t s(admit_t),   dadmit_t = dx_t x_t (1 - s(admit_t))
//     dL_t = a_t e_t h_{t-1} - (a_t^2 / m_t) e_t s(admit_t) x_t
//     dforget_t = dL_t L_t (1 - s(forget_t)),   drate = sum_t dL_t L_t / rate
//     dstate = a_1 e_1
// Some thirty operations for each value and four rows of memory (seven in the
// gradient): HBM bounds it if rows are read once and enough of them are on
// their way, so the recurrence is cut along time.  A thread owns two channels
// of a run of 8 rows (forward: of two); 8 warps below each other make a tile,
// whose rows come through rings in shared memory, a tile or two ahead.  The
// rows of a run compose to one map h -> A h + H, maps of warps through shared
// memory, maps of blocks through a cluster of up to 16 that send them to each
// other, and then the rows, still in registers, are walked once more from the
// state that enters.  From run to run decays near one are held as a - 1.  What composes with what is fixed by the sizes: the same
// call gives the same bits.  The gradient walks the tiles from the end, forward
// within a run from the state that the forward pass kept of it, and back.
//
// Measured, bf16: forward 8 x 2048 x 4096 (537 MB) 119 us, 4.5 TB/s, gradient
// (933 MB) 228 us, 4.1 TB/s; forward 65536 x 1536 (805 MB) 259 us, 3.1 TB/s.
// Copying runs at 6.8 TB/s.  58 % of the issue slots are in use at two blocks an
// SM: latency of the exchange and of short chains is what is left.  With decays
// rounded from run to run the same took 114, 222 and 238 us.
#include <cooperative_groups.h>

#include <algorithm>

#include "seq_common.cuh"
#include "tcgen05.cuh"

namespace tcu {
namespace seq {

__global__ void row_sequence_kernel(int32_t *row_seq, const int32_t *offsets, int count,
                                    int rows);

namespace {

namespace cg = cooperative_groups;

constexpr int kRun = TCU_SEQ_GATED_MARK;  // rows of a thread
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kTile = kRun * kWarps;  // rows of a block at a time, in the gradient
// Forward a thread takes two runs below each other: a tile's exchange costs as
// much as 64 rows' arithmetic.  The gradient's registers hold one.
constexpr int kRuns = 2, kMine = kRuns * kRun, kLongTile = kRuns * kTile;
constexpr int kStrip = 64;  // channels of a block
constexpr int kMostCluster = 16;

template <typename T>
struct GatedArgs {
  Rows<const T> x, forget, admit, dy;
  Rows<T> y, dx, dforget, dadmit;
  const float *rate, *state, *dlast;
  float *last, *dstate, *marks, *parts;
  const int32_t *offsets, *row_seq, *slots;
  int64_t channels, num_slots;
  int rows, sequences, batches, runs;
};

__device__ __forceinline__ float2 splat(float v) { return make_float2(v, v); }
// For each value: v where h is finite, else w.
__device__ __forceinline__ float2 if_finite(float2 h, float2 v, float2 w) {
  return make_float2(fabsf(h.x) < INFINITY ? v.x : w.x, fabsf(h.y) < INFINITY ? v.y : w.y);
}
// Whether a value of the warp's is not finite.
__device__ __forceinline__ bool any_odd(float2 v) {
  return __any_sync(~0u, !(fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY));
}

// a = exp(L), a - 1 and m = sqrt(1 - a^2) for L <= 0.  1 - a^2 loses what a lacks in
// its last place where a is near one, so a - 1 is a Taylor sum of degree 6 for L >
// -kNear (the next term is 5e-8 of it); kAllNear: there is no other L.
//
// So does a state lose, at every row, where a gate hardly changes: an a within
// 1e-5 of one, rounded to fp32, is off by 3e-3 of 1 - a, and the state remembers 1
// / (1 - a) rows.  Within a run a is used as it is rounded (16 rows: 5e-7 of the
// state); from run to run, and where a state is handed out or taken, a - 1 is.
constexpr float kNear = 0.25f;
struct Decay {
  float2 a, less, m;
};
__device__ __forceinline__ float rsqrt_fast(float v) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v));
  return y;
}
template <bool kAllNear>
__device__ __forceinline__ Decay decay2(float2 L) {
  float2 p = __ffma2_rn(L, splat(1.f / 720), splat(1.f / 120));
  p = __ffma2_rn(p, L, splat(1.f / 24));
  p = __ffma2_rn(p, L, splat(1.f / 6));
  p = __ffma2_rn(p, L, splat(0.5f));
  p = __ffma2_rn(p, L, splat(1.f));
  p = __fmul2_rn(p, L);
  Decay d;
  d.a = __fadd2_rn(p, splat(1.f));
  if constexpr (!kAllNear) {
    const float2 z = __fmul2_rn(L, splat(kLog2e));
    const float2 e = make_float2(exp2_fast(z.x), exp2_fast(z.y)), q = __fadd2_rn(e, splat(-1.f));
    if (!(L.x > -kNear)) p.x = q.x, d.a.x = e.x;
    if (!(L.y > -kNear)) p.y = q.y, d.a.y = e.y;
  }
  d.less = p;
  // 1 - a^2, kept off zero, where its root's reciprocal is none
  float2 r = __fmul2_rn(p, __ffma2_rn(p, splat(-1.f), splat(-2.f)));
  r = make_float2(fmaxf(r.x, 1e-37f), fmaxf(r.y, 1e-37f));
  d.m = __fmul2_rn(r, make_float2(rsqrt_fast(r.x), rsqrt_fast(r.y)));
  return d;
}
// A decay in one word: a - 1, below zero, where it is near one, else itself.  In runs in which a sequence opens or closes, and on the way between
// blocks.
__device__ __forceinline__ float held(float a, float less) {
  return a > 0.5f ? fminf(less, -1e-37f) : a;
}
__device__ __forceinline__ float2 held(const Decay &d) {
  return make_float2(held(d.a.x, d.less.x), held(d.a.y, d.less.y));
}
__device__ __forceinline__ float near_one(float v) {  // one or zero
  return v < 0.f ? 1.f : 0.f;
}
__device__ __forceinline__ float2 near_one(float2 v) { return make_float2(near_one(v.x), near_one(v.y)); }
__device__ __forceinline__ float2 decay_of(float2 v) { return __fadd2_rn(near_one(v), v); }
// a h + v, which carries an infinite h on only where kOdd
template <bool kOdd>
__device__ __forceinline__ float2 decayed(float2 a, float2 h, float2 v) {
  const float2 w = __ffma2_rn(near_one(a), h, __ffma2_rn(a, h, v));
  return kOdd ? if_finite(h, w, __ffma2_rn(decay_of(a), h, v)) : w;
}

// h -> (A + rest) h + H of two channels, rest what A lacks in its last place where
// it is near one.  kCut in the place of A: a sequence opens on the way, and h goes
// no further, not even one that is not finite.  (A product of decays that has
// become zero is no cut: it is the same sequence.)
struct alignas(16) Map {
  float2 A, H;
};
constexpr float kCut = -1.f;
template <bool kPacked>
__device__ __forceinline__ float2 unless_cut(const Map &m, float2 v) {
  if constexpr (!kPacked) return v;
  return make_float2(m.A.x == kCut ? m.H.x : v.x, m.A.y == kCut ? m.H.y : v.y);
}
template <bool kPacked, bool kOdd>
__device__ __forceinline__ float2 apply(const Map &m, float2 rest, float2 h) {
  float2 v = __ffma2_rn(m.A, h, __ffma2_rn(rest, h, m.H));
  if constexpr (kOdd) v = if_finite(h, v, __ffma2_rn(m.A, h, m.H));
  return unless_cut<kPacked>(m, v);
}
// Rows and maps that follow on each other: the product of decays (kAllNear: one
// and `less`) and that less one.
template <bool kAllNear>
struct Path {
  float2 A, less, H;
  bool cut;  // in both channels
  __device__ __forceinline__ Path() : A(splat(1.f)), less(splat(0.f)), H(splat(0.f)), cut(false) {}
  __device__ __forceinline__ void decay(const Decay &d) {
    if constexpr (!kAllNear) A = __fmul2_rn(A, d.a);
    less = __fadd2_rn(less, __ffma2_rn(less, d.less, d.less));
  }
  // (H is the caller's)
  __device__ __forceinline__ void decay(const Map &m, float2 rest) {
    const float2 p = __fadd2_rn(__fadd2_rn(m.A, splat(-1.f)), rest);
    A = __fmul2_rn(A, m.A);
    less = __fadd2_rn(less, __ffma2_rn(less, p, p));
    cut = cut || m.A.x == kCut;
  }
  template <bool kPacked>
  __device__ __forceinline__ Map map(float2 &rest) const {
    const float2 near = __fadd2_rn(less, splat(1.f));
    rest = __fadd2_rn(less, __ffma2_rn(near, splat(-1.f), splat(1.f)));
    Map m{near, H};
    if constexpr (!kAllNear) {
      if (!(A.x > 0.5f)) m.A.x = A.x, rest.x = 0.f;
      if (!(A.y > 0.5f)) m.A.y = A.y, rest.y = 0.f;
    }
    if (kPacked && cut) m.A = splat(kCut);
    return m;
  }
  // the same with A in one word
  template <bool kPacked>
  __device__ __forceinline__ Map message() const {
    return {kPacked && cut ? splat(kCut) : make_float2(held(A.x, less.x), held(A.y, less.y)), H};
  }
};

// Where sequences open and close in the 8 rows from r0 (bit i: row r0 + i),
// which rows lie in one, and the sequence of row r0 + lane.
struct Marks8 {
  uint32_t open, close, inside;
  int seq;
};
template <bool kPacked, typename T>
__device__ __forceinline__ Marks8 sequences_of(const GatedArgs<T> &a, int b, int r0, int lane) {
  Marks8 m;
  if constexpr (kPacked) {
    const int t = r0 - 1 + lane;  // r0 < rows <= 2^31 - 4097
    const int v = lane < kRun + 2 && t >= 0 && t < a.rows ? a.row_seq[t] : -2;
    m.seq = __shfl_down_sync(~0u, v, 1);
    const int next = __shfl_down_sync(~0u, v, 2);
    const bool in = lane < kRun && m.seq >= 0;
    m.open = __ballot_sync(~0u, in && m.seq != v);
    m.close = __ballot_sync(~0u, in && m.seq != next);
    m.inside = __ballot_sync(~0u, in);
  } else {
    m.open = r0 == 0 ? 1u : 0u;
    m.close = a.rows - 1 - r0 < kRun ? 1u << (a.rows - 1 - r0) : 0u;
    m.inside = a.rows - r0 < kRun ? (1u << (a.rows - r0)) - 1u : (1u << kRun) - 1u;
    m.seq = b;
  }
  return m;
}

// Two values of a per-sequence array at channel c (count of them exist).
template <bool kWide>
__device__ __forceinline__ float2 pair_at(const float *p, int64_t at, int count) {
  if constexpr (kWide)
    return count > 0 ? *reinterpret_cast<const float2 *>(p + at) : make_float2(0.f, 0.f);
  return make_float2(count > 0 ? p[at] : 0.f, count > 1 ? p[at + 1] : 0.f);
}
template <bool kWide>
__device__ __forceinline__ void put_pair(float *p, int64_t at, int count, float2 v) {
  if constexpr (kWide) {
    if (count > 0) *reinterpret_cast<float2 *>(p + at) = v;
    return;
  }
  if (count > 0) p[at] = v.x;
  if (count > 1) p[at + 1] = v.y;
}

// Gives a warp the value that enters its rows: the maps of the warps before it
// (kBack: behind it) are applied to what enters the block's.  In a block of its
// own that is what left the tile before, as its maps give it and not the walk
// over its rows, put down by the warp that comes last (`leaves`: ahead of the
// first tile); in a cluster what left the cluster's rows before, `carry`, through
// the maps of the blocks before it.  Blocks send their maps to each other as
// stores that the receiver's mbarrier counts; two sets of maps are enough, since
// a block sends the next but one only when all have sent the next, and so have
// read the last.
struct Joint {
  Map warps[2][kWarps][32];
  float2 rests[2][kWarps][32];
  Map blocks[2][kMostCluster][32];  // A in one word: what counts is how many words are sent
  float2 carry[2][32];
  uint64_t arrived[2];
};
__device__ __forceinline__ void send_map(uint32_t to, const Map &m, uint32_t mbar) {
  asm volatile(
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, "
      "[%5];" ::"r"(to),
      "f"(m.A.x), "f"(m.A.y), "f"(m.H.x), "f"(m.H.y), "r"(mbar)
      : "memory");
}
__device__ __forceinline__ void expect_maps(Joint &s, int turn, int size) {
  mbar_expect_tx(smem_u32(&s.arrived[turn]), size * 32 * (uint32_t)sizeof(Map));
}
__device__ __forceinline__ void start_joint(Joint &s, int size) {
  if (size == 1) return;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&s.arrived[0]), 1);
    mbar_init(smem_u32(&s.arrived[1]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    expect_maps(s, 0, size);
    expect_maps(s, 1, size);
  }
  cg::this_cluster().sync();
}
// h through the maps of the warps before (behind) this one.
template <bool kBack, bool kPacked, bool kOdd>
__device__ __forceinline__ float2 through_warps(const Joint &s, int turn, float2 h, int warp, int lane) {
  constexpr int first = kBack ? kWarps - 1 : 0, by = kBack ? -1 : 1;
#pragma unroll 2
  for (int w = first; w != warp; w += by)
    h = apply<kPacked, kOdd>(s.warps[turn][w][lane], s.rests[turn][w][lane], h);
  return h;
}
// carry through the maps of all blocks; what enters this one.
template <bool kBack, bool kPacked, bool kOdd>
__device__ __forceinline__ float2 through_blocks(const Joint &s, int turn, float2 &carry, int lane,
                                                 int rank, int size) {
  float2 enters = carry;
  for (int i = 0; i < size; ++i) {
    const int r = kBack ? size - 1 - i : i;
    if (r == rank) enters = carry;
    const Map m = s.blocks[turn][r][lane];
    carry = unless_cut<kPacked>(m, decayed<kOdd>(m.A, carry, m.H));
  }
  return enters;
}
template <bool kPacked>
__device__ __forceinline__ float2 apply_any(const Map &m, float2 rest, float2 h) {
  const float2 v = apply<kPacked, false>(m, rest, h);
  return any_odd(v) ? apply<kPacked, true>(m, rest, h) : v;
}
template <bool kBack, bool kPacked, bool kAllNear>
__device__ __forceinline__ float2 join(Joint &s, int turn, const Path<kAllNear> &own, float2 &carry,
                                       int warp, int lane, int rank, int size, int &phase) {
  float2 rest;
  const Map mine = own.template map<kPacked>(rest);
  s.warps[turn][warp][lane] = mine;
  s.rests[turn][warp][lane] = rest;
  __syncthreads();
  constexpr int first = kBack ? kWarps - 1 : 0, by = kBack ? -1 : 1;
  const bool last = warp == kWarps - 1 - first;
  if (size == 1) {
    const float2 from = s.carry[turn][lane];
    float2 enters = through_warps<kBack, kPacked, false>(s, turn, from, warp, lane);
    if (any_odd(enters)) enters = through_warps<kBack, kPacked, true>(s, turn, from, warp, lane);
    if (last) s.carry[turn ^ 1][lane] = apply_any<kPacked>(mine, rest, enters);
    return enters;
  }
  if (last) {
    Path<false> path;
#pragma unroll 2
    for (int w = first; w != warp; w += by) {
      path.decay(s.warps[turn][w][lane], s.rests[turn][w][lane]);
      path.H = apply<kPacked, false>(s.warps[turn][w][lane], s.rests[turn][w][lane], path.H);
    }
    path.decay(mine, rest);
    path.H = apply<kPacked, false>(mine, rest, path.H);
    if (any_odd(path.H))
      path.H = apply<kPacked, true>(
          mine, rest, through_warps<kBack, kPacked, true>(s, turn, splat(0.f), warp, lane));
    const Map all = path.template message<kPacked>();
    const uint32_t to = smem_u32(&s.blocks[turn][rank][lane]), mbar = smem_u32(&s.arrived[turn]);
    for (int r = 0; r < size; ++r) send_map(mapa_shared(to, r), all, mapa_shared(mbar, r));
  }
  // phase: -1 once a wait has run out, for the whole warp, and what follows is no
  // number
  if (phase >= 0 && !__all_sync(~0u, mbar_wait_cluster_bounded(smem_u32(&s.arrived[turn]), phase >> 1 & 1)))
    phase = -1;
  if (phase < 0) return splat(__int_as_float(0x7fffffff));
  ++phase;
  if (threadIdx.x == 0) expect_maps(s, turn, size);
  const float2 from = carry;
  float2 enters = through_blocks<kBack, kPacked, false>(s, turn, carry, lane, rank, size);
  enters = through_warps<kBack, kPacked, false>(s, turn, enters, warp, lane);
  if (any_odd(__ffma2_rn(carry, splat(0.f), enters))) {
    carry = from;
    enters = through_blocks<kBack, kPacked, true>(s, turn, carry, lane, rank, size);
    enters = through_warps<kBack, kPacked, true>(s, turn, enters, warp, lane);
  }
  return enters;
}
template <bool kBack>
__device__ __forceinline__ void leaves(Joint &s, int turn, float2 h, int warp, int lane, int size) {
  if (size == 1 && warp == (kBack ? 0 : kWarps - 1)) s.carry[turn][lane] = h;
}

// An empty sequence ends in the state it starts from.
template <bool kWide, typename T>
__device__ __forceinline__ void empty_sequences(const GatedArgs<T> &a, float *to, const float *from,
                                                int64_t c, int count, int first, int step) {
  for (int64_t s = first; s < a.sequences; s += step)
    if (a.offsets[s] >= a.offsets[s + 1])
      put_pair<kWide>(to, s * a.channels + c, count,
                      from ? pair_at<kWide>(from, s * a.channels + c, count) : splat(0.f));
}

// ------------------------------------------------------------ rows on the way
// A warp's ring of kStages tiles of 8 rows x 64 channels of kTensors row
// tensors, filled by copies that nothing waits for until their rows are due:
// 16 bytes at a time where rows are aligned so (kWide), 4 for other 32-bit
// rows; 16-bit rows at odd places go through registers.
template <typename T, int kTensors, int kStages>
struct alignas(16) Ring {
  T v[kStages][kTensors][kRun][kStrip];
};
// Zeros for channels behind the last, which no copy brings: numbers, so that
// what is not finite is looked for in all of a warp's values.
template <typename R>
__device__ __forceinline__ void clear_ring(R &ring, int64_t c0, int64_t channels, int lane) {
  if (c0 + kStrip <= channels) return;
  uint4 *at = reinterpret_cast<uint4 *>(&ring);
  for (int i = lane; i < (int)(sizeof(R) / 16); i += 32) at[i] = make_uint4(0, 0, 0, 0);
  __syncwarp();
}
template <int kBytes>
__device__ __forceinline__ void copy_async(void *dst, const void *src, bool has) {
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(has ? 16 : 0)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(src), "r"(has ? 4 : 0)
                 : "memory");
}
// Where a lane's part of a run of rows is, n <= 8 of them (the others become
// zeros), the first a row `pitch` values long apart.
template <typename T, bool kWide>
struct Source {
  static constexpr int kPer = 16 / sizeof(T), kChunks = kStrip / kPer;
  const T *p;
  int64_t pitch;
  __device__ __forceinline__ void init(const Rows<const T> &from, int64_t b, int r0, int64_t c0,
                                       int lane) {
    pitch = from.row;
    p = from.p + b * from.batch + c0 + (kWide ? lane % kChunks * kPer : lane) +
        ((int64_t)r0 + (kWide ? lane / kChunks : 0)) * pitch;
  }
  __device__ __forceinline__ void copy(T (*to)[kStrip], int n, int64_t c0, int64_t channels,
                                       int lane) const {
    if constexpr (kWide) {
      constexpr int each = 32 / kChunks;
      const int r = lane / kChunks, c = lane % kChunks * kPer;
      const bool in = c0 + c < channels;
      const T *q = p;
#pragma unroll
      for (int i = 0; i < kRun / each; ++i, q += each * pitch)
        if (in) copy_async<16>(&to[r + i * each][c], r + i * each < n ? q : p, r + i * each < n);
    } else if constexpr (sizeof(T) == 4) {
      const T *q = p;
#pragma unroll
      for (int r = 0; r < kRun; ++r, q += pitch)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (c0 + lane + 32 * k < channels)
            copy_async<4>(&to[r][lane + 32 * k], r < n ? q + 32 * k : p, r < n);
    } else {
      T v[kRun][2];
      const T *q = p;
#pragma unroll
      for (int r = 0; r < kRun; ++r, q += pitch)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          v[r][k] = r < n && c0 + lane + 32 * k < channels ? q[32 * k] : from_f<T>(0.f);
#pragma unroll
      for (int r = 0; r < kRun; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k) to[r][lane + 32 * k] = v[r][k];
    }
  }
};
__device__ __forceinline__ void copies_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
  __syncwarp();
}
template <typename T>
__device__ __forceinline__ float2 pair_of(const T (*rows)[kStrip], int i, int lane) {
  uint32_t w[Pair<T>::kWords];
  const Vec<uint32_t, Pair<T>::kWords> v =
      *reinterpret_cast<const Vec<uint32_t, Pair<T>::kWords> *>(&rows[i][2 * lane]);
#pragma unroll
  for (int k = 0; k < Pair<T>::kWords; ++k) w[k] = v.v[k];
  return Pair<T>::get(w);
}
template <typename T, bool kWide>
__device__ __forceinline__ void put_row(T *to, float2 v, int count) {
  Raw<T, 2> out;
  out.set(0, v);
  out.template store<kWide>(to, count);
}

// Blocks an SM, and stages: what its shared memory holds, and the registers.
template <typename T>
struct Sizes {
  static constexpr int kStages = sizeof(T) == 2 ? 3 : 1, kGradStages = sizeof(T) == 2 ? 2 : 1;
  static constexpr int kBlocks = 2, kGradBlocks = 2;
};

template <typename T>
struct GatedShared {
  Joint joint;
  Ring<T, 3, Sizes<T>::kStages> ring[kWarps];
};
template <typename T>
struct GradShared {
  Joint joint;
  float2 sums[kWarps][32];
  Ring<T, 4, Sizes<T>::kGradStages> ring[kWarps];
};

template <typename T, bool kPacked, bool kWide, bool kAllNear>
__device__ __forceinline__ void gated_rows(const GatedArgs<T> &a, GatedShared<T> &s, int size,
                                           float2 rate) {
  constexpr int kStages = Sizes<T>::kStages;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int rank = (int)(blockIdx.x % size);
  const int64_t c0 = (int64_t)(blockIdx.x / size) * kStrip, c = c0 + 2 * lane;
  const int count = (int)max((int64_t)0, min((int64_t)2, a.channels - c));
  const float2 minus = make_float2(-rate.x, -rate.y);
  const int step = size * kLongTile;
  auto &ring = s.ring[warp];
  clear_ring(ring, c0, a.channels, lane);
  int turn = 0, phase = 0;
  for (int b = blockIdx.y; b < a.batches; b += gridDim.y) {
    const int start = rank * kLongTile + warp * kMine;  // this warp's rows, a step apart
    float2 carry = splat(0.f);
    if (!kPacked && a.state) carry = pair_at<kWide>(a.state, (int64_t)b * a.channels + c, count);
    leaves<false>(s.joint, turn, carry, warp, lane, size);
    Source<T, kWide> from[3];
    from[0].init(a.forget, b, start, c0, lane);
    from[1].init(a.admit, b, start, c0, lane);
    from[2].init(a.x, b, start, c0, lane);
    T *y = a.y.at(b, 0) + c + (int64_t)start * a.y.row;
    float *mark = a.marks + ((int64_t)b * a.runs + start / kRun) * a.channels + c;
    int ahead = start, sub = 0;  // row that is asked for next, which of a tile's runs
    const auto ask = [&](int stage) {
      const int n = min(kRun, a.rows - ahead);
      if (n > 0) {
#pragma unroll
        for (int k = 0; k < 3; ++k) from[k].copy(ring.v[stage][k], n, c0, a.channels, lane);
      }
      const int hop = sub == kRuns - 1 ? step - kMine + kRun : kRun;
      sub = sub == kRuns - 1 ? 0 : sub + 1;
#pragma unroll
      for (int k = 0; k < 3; ++k) from[k].p += hop * from[k].pitch;
      ahead = a.rows - ahead > hop ? ahead + hop : a.rows;  // the sum may pass 2^31
      copies_commit();
    };
    __syncwarp();
    for (int i = 0; i < kStages; ++i) ask(i);
    int stage = 0;
    for (int t0 = 0; t0 < a.rows; t0 += step) {
      const int r0 = t0 + start;
      float2 keep[kRuns][kRun], add[kRuns][kRun];
      Marks8 seqs[kRuns] = {};
      bool plain[kRuns];
      Path<kAllNear> run;
      const auto opens = [&](int u, int i) {  // what enters the sequence that opens in a row
        const int64_t q = __shfl_sync(~0u, seqs[u].seq, i);
        return a.state ? pair_at<kWide>(a.state, q * a.channels + c, count) : splat(0.f);
      };
#pragma unroll
      for (int u = 0; u < kRuns; ++u) {
        if (r0 + u * kRun < a.rows) seqs[u] = sequences_of<kPacked>(a, b, r0 + u * kRun, lane);
        // a run of whole rows in which no sequence opens (dense: a row 0 takes
        // the carry) or closes goes without a look at each row
        plain[u] = seqs[u].inside == (1u << kRun) - 1 && seqs[u].close == 0 &&
                   (!kPacked || seqs[u].open == 0);
        run.cut = run.cut || (kPacked && seqs[u].open);
        copies_wait<kStages - 1>();
        const auto gates = [&](int u, int i) {
          const float2 f = pair_of(ring.v[stage][0], i, lane), g = pair_of(ring.v[stage][1], i, lane),
                       x = pair_of(ring.v[stage][2], i, lane);
          const Decay d = decay2<kAllNear>(__fmul2_rn(sigmoid2(f), minus));
          add[u][i] = __fmul2_rn(__fmul2_rn(d.m, sigmoid2(g)), x);
          return d;
        };
        if (plain[u]) {
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            const Decay d = gates(u, i);
            keep[u][i] = d.a;
            run.decay(d);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            const Decay d = gates(u, i);
            keep[u][i] = held(d);
            if (seqs[u].inside >> i & 1) run.decay(d);
          }
        }
        __syncwarp();
        ask(stage);
        stage = stage == kStages - 1 ? 0 : stage + 1;
        if (plain[u]) {
#pragma unroll
          for (int i = 0; i < kRun; ++i) run.H = __ffma2_rn(run.H, keep[u][i], add[u][i]);
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i) {
            if (kPacked && (seqs[u].open >> i & 1)) run.H = opens(u, i);
            if (seqs[u].inside >> i & 1) run.H = decayed<true>(keep[u][i], run.H, add[u][i]);
          }
        }
      }
      float2 h = join<false, kPacked>(s.joint, turn, run, carry, warp, lane, rank, size, phase);
      turn ^= 1;
      T *to = y;
#pragma unroll
      for (int u = 0; u < kRuns; ++u) {
        if (r0 + u * kRun >= a.rows) break;
        if (a.marks) put_pair<kWide>(mark + u * a.channels, 0, count, h);
        if (plain[u]) {
#pragma unroll
          for (int i = 0; i < kRun; ++i, to += a.y.row) {
            h = __ffma2_rn(h, keep[u][i], add[u][i]);
            put_row<T, kWide>(to, h, count);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kRun; ++i, to += a.y.row) {
            if (kPacked && (seqs[u].open >> i & 1)) h = opens(u, i);
            if (!(seqs[u].inside >> i & 1)) continue;
            h = decayed<true>(keep[u][i], h, add[u][i]);
            put_row<T, kWide>(to, h, count);
            if (seqs[u].close >> i & 1) {
              const int64_t q = __shfl_sync(~0u, seqs[u].seq, i);
              if (a.last) put_pair<kWide>(a.last, q * a.channels + c, count, h);
            }
          }
        }
      }
      y += step * (int64_t)a.y.row;
      mark += (int64_t)(step / kRun) * a.channels;
    }
    copies_wait<0>();
  }
  if (kPacked && a.last && blockIdx.y == 0)
    empty_sequences<kWide>(a, a.last, a.state, c, count, rank * kWarps + warp, size * kWarps);
  if (size > 1) cg::this_cluster().sync();  // no block leaves while others send to it
}

// The rate of each of the lane's channels, and whether no decay of the warp's
// is far from one.
template <bool kWide, typename T>
__device__ __forceinline__ float2 rates(const GatedArgs<T> &a, int size, bool &near) {
  const int64_t c = (int64_t)(blockIdx.x / size) * kStrip + 2 * (threadIdx.x % 32);
  const float2 r = pair_at<kWide>(a.rate, c, (int)max((int64_t)0, min((int64_t)2, a.channels - c)));
  near = __syncthreads_and(r.x < kNear && r.y < kNear);
  return r;
}

template <typename T, bool kPacked, bool kWide>
__global__ void __launch_bounds__(kThreads, Sizes<T>::kBlocks)
    gated_kernel(const GatedArgs<T> a, int size) {
  extern __shared__ __align__(16) uint8_t raw[];
  GatedShared<T> &s = *reinterpret_cast<GatedShared<T> *>(raw);
  start_joint(s.joint, size);
  bool near;
  const float2 rate = rates<kWide>(a, size, near);
  if (near) gated_rows<T, kPacked, kWide, true>(a, s, size, rate);
  else gated_rows<T, kPacked, kWide, false>(a, s, size, rate);
}

template <typename T, bool kPacked, bool kWide, bool kAllNear>
__device__ __forceinline__ void grad_rows(const GatedArgs<T> &a, GradShared<T> &s, int size,
                                          float2 rate) {
  constexpr int kStages = Sizes<T>::kGradStages;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int rank = (int)(blockIdx.x % size);
  const int64_t c0 = (int64_t)(blockIdx.x / size) * kStrip, c = c0 + 2 * lane;
  const int count = (int)max((int64_t)0, min((int64_t)2, a.channels - c));
  const float2 minus = make_float2(-rate.x, -rate.y);
  const int step = size * kTile;
  auto &ring = s.ring[warp];
  clear_ring(ring, c0, a.channels, lane);
  float2 drate = splat(0.f);
  int turn = 0, phase = 0;
  const int end = (a.rows - 1) / step * step;  // the last tile
  for (int b = blockIdx.y; b < a.batches; b += gridDim.y) {
    const int start = end + rank * kTile + warp * kRun;
    float2 carry = splat(0.f);  // a_{t+1} e_{t+1} of the row below
    if (!kPacked && a.dlast) carry = pair_at<kWide>(a.dlast, (int64_t)b * a.channels + c, count);
    leaves<true>(s.joint, turn, carry, warp, lane, size);
    Source<T, kWide> from[4];
    from[0].init(a.forget, b, start, c0, lane);
    from[1].init(a.admit, b, start, c0, lane);
    from[2].init(a.x, b, start, c0, lane);
    from[3].init(a.dy, b, start, c0, lane);
    // outputs: at the run's last row, walked upwards
    T *to[3];
    const Rows<T> *outs[3] = {&a.dx, &a.dadmit, &a.dforget};
#pragma unroll
    for (int k = 0; k < 3; ++k)
      to[k] = outs[k]->at(b, 0) + c + ((int64_t)start + kRun - 1) * outs[k]->row;
    const float *mark = a.marks + ((int64_t)b * a.runs + start / kRun) * a.channels + c;
    int ahead = start;
    const auto ask = [&](int stage) {
      const int n = min(kRun, a.rows - ahead);
      if (n > 0 && ahead >= 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) from[k].copy(ring.v[stage][k], n, c0, a.channels, lane);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) from[k].p -= step * from[k].pitch;
      ahead -= step;
      copies_commit();
    };
    __syncwarp();
    for (int i = 0; i < kStages; ++i) ask(i);
    int stage = 0;
    for (int t0 = end; t0 >= 0; t0 -= step) {
      const int r0 = t0 + rank * kTile + warp * kRun, n = min(kRun, a.rows - r0);
      Marks8 seqs{};
      float2 h = splat(0.f);
      if (n > 0) {
        seqs = sequences_of<kPacked>(a, b, r0, lane);
        h = pair_at<kWide>(mark, 0, count);
      }
      copies_wait<kStages - 1>();
      const bool plain = seqs.inside == (1u << kRun) - 1 && seqs.close == 0 && seqs.open == 0;
      const auto &rows = ring.v[stage];
      // forward: decays and the state before each row
      float2 keep[kRun], root[kRun], before[kRun];
      Path<kAllNear> run;
      run.cut = kPacked && (seqs.open | seqs.close);
      const auto gates = [&](int i) {
        const Decay d = decay2<kAllNear>(__fmul2_rn(sigmoid2(pair_of(rows[0], i, lane)), minus));
        root[i] = d.m;
        before[i] = h;
        h = __ffma2_rn(h, d.a, __fmul2_rn(__fmul2_rn(d.m, sigmoid2(pair_of(rows[1], i, lane))),
                                          pair_of(rows[2], i, lane)));
        return d;
      };
      if (plain) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          const Decay d = gates(i);
          keep[i] = d.a;
          run.decay(d);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          if (kPacked && (seqs.open >> i & 1)) {
            const int64_t q = __shfl_sync(~0u, seqs.seq, i);
            h = a.state ? pair_at<kWide>(a.state, q * a.channels + c, count) : splat(0.f);
          }
          const Decay d = gates(i);
          keep[i] = held(d);
          if (seqs.inside >> i & 1) run.decay(d);
        }
      }
      const auto closes = [&](int i) {  // what enters the sequence that ends in a row
        const int64_t q = __shfl_sync(~0u, seqs.seq, i);
        return a.dlast ? pair_at<kWide>(a.dlast, q * a.channels + c, count) : splat(0.f);
      };
      if (plain) {
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i)
          run.H = __fmul2_rn(__fadd2_rn(run.H, pair_of(rows[3], i, lane)), keep[i]);
      } else {
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i) {
          if (kPacked && (seqs.close >> i & 1)) run.H = closes(i);
          if (!(seqs.inside >> i & 1)) continue;
          run.H = decayed<true>(keep[i], __fadd2_rn(run.H, pair_of(rows[3], i, lane)), splat(0.f));
          if (kPacked && (seqs.open >> i & 1)) run.H = splat(0.f);
        }
      }
      float2 e = join<true, kPacked>(s.joint, turn, run, carry, warp, lane, rank, size, phase);
      turn ^= 1;
      float2 share = splat(0.f);
      // the gradients of row i, of decay k, from that of its state, e
      const auto row = [&](int i, float2 k, T *dx, T *dg, T *df) {
        e = __fadd2_rn(e, pair_of(rows[3], i, lane));
        const float2 open = sigmoid2(pair_of(rows[0], i, lane)), way = sigmoid2(pair_of(rows[1], i, lane)),
                     x = pair_of(rows[2], i, lane);
        const float2 L = __fmul2_rn(open, minus), ew = __fmul2_rn(e, way);
        const float2 gx = __fmul2_rn(ew, root[i]);
        put_row<T, kWide>(dx, gx, count);
        const float2 gxx = __fmul2_rn(gx, x);
        put_row<T, kWide>(dg, __ffma2_rn(gxx, __fmul2_rn(way, splat(-1.f)), gxx), count);
        // dL L, with L / m, which goes to zero with L as -sqrt(-L / 2)
        const float2 lm = __fmul2_rn(L, make_float2(rcp_fast(root[i].x), rcp_fast(root[i].y)));
        const float2 one = __fmul2_rn(__fmul2_rn(e, before[i]), L);
        const float2 two = __fmul2_rn(__fmul2_rn(__fmul2_rn(ew, x), k), lm);
        const float2 dL = __fmul2_rn(k, __ffma2_rn(two, splat(-1.f), one));
        share = __fadd2_rn(share, dL);
        put_row<T, kWide>(df, __ffma2_rn(dL, __fmul2_rn(open, splat(-1.f)), dL), count);
      };
      T *dx = to[0], *dg = to[1], *df = to[2];
      if (plain) {
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i, dx -= a.dx.row, dg -= a.dadmit.row, df -= a.dforget.row) {
          row(i, keep[i], dx, dg, df);
          e = __fmul2_rn(e, keep[i]);  // the row above's
        }
      } else {
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i, dx -= a.dx.row, dg -= a.dadmit.row, df -= a.dforget.row) {
          if (i >= n) continue;
          if (kPacked && !(seqs.inside >> i & 1)) {  // rows of no sequence
            put_row<T, kWide>(dx, splat(0.f), count);
            put_row<T, kWide>(dg, splat(0.f), count);
            put_row<T, kWide>(df, splat(0.f), count);
            continue;
          }
          if (kPacked && (seqs.close >> i & 1)) e = closes(i);
          row(i, decay_of(keep[i]), dx, dg, df);
          e = decayed<true>(keep[i], e, splat(0.f));
          if ((seqs.open >> i & 1) && a.dstate) {
            const int64_t q = __shfl_sync(~0u, seqs.seq, i);
            put_pair<kWide>(a.dstate, q * a.channels + c, count, e);
          }
        }
      }
      drate = __fadd2_rn(drate, share);
      __syncwarp();
      ask(stage);
      stage = stage == kStages - 1 ? 0 : stage + 1;
#pragma unroll
      for (int k = 0; k < 3; ++k) to[k] -= step * (int64_t)outs[k]->row;
      mark -= (int64_t)(step / kRun) * a.channels;
    }
    copies_wait<0>();
  }
  if (kPacked && a.dstate && blockIdx.y == 0)
    empty_sequences<kWide>(a, a.dstate, a.dlast, c, count, rank * kWarps + warp, size * kWarps);
  s.sums[warp][lane] = drate;
  __syncthreads();
  if (warp == 0) {
    float2 sum = splat(0.f);
    for (int w = 0; w < kWarps; ++w) sum = __fadd2_rn(sum, s.sums[w][lane]);
    // of L = -rate s(forget): d rate = dL L / rate
    sum = make_float2(sum.x / rate.x, sum.y / rate.y);
    put_pair<kWide>(a.parts, ((int64_t)blockIdx.y * size + rank) * a.channels + c, count, sum);
  }
  if (size > 1) cg::this_cluster().sync();
}

template <typename T, bool kPacked, bool kWide>
__global__ void __launch_bounds__(kThreads, Sizes<T>::kGradBlocks)
    gated_grad_kernel(const GatedArgs<T> a, int size) {
  extern __shared__ __align__(16) uint8_t raw[];
  GradShared<T> &s = *reinterpret_cast<GradShared<T> *>(raw);
  start_joint(s.joint, size);
  bool near;
  const float2 rate = rates<kWide>(a, size, near);
  if (near) grad_rows<T, kPacked, kWide, true>(a, s, size, rate);
  else grad_rows<T, kPacked, kWide, false>(a, s, size, rate);
}

// One thread for two channels of an entry.
template <typename T, bool kWide>
__global__ void __launch_bounds__(128) gated_step_kernel(const GatedArgs<T> a) {
  const int64_t c = 2 * ((int64_t)blockIdx.x * blockDim.x + threadIdx.x);
  const int count = (int)max((int64_t)0, min((int64_t)2, a.channels - c));
  if (count == 0) return;
  const float2 rate = pair_at<kWide>(a.rate, c, count);
  for (int64_t b = blockIdx.y; b < a.sequences; b += gridDim.y) {
    const int64_t slot = a.slots ? a.slots[b] : b;
    Raw<T, 2> x, f, g, y;
    f.template load<kWide>(a.forget.p + b * a.forget.batch + c, count);
    g.template load<kWide>(a.admit.p + b * a.admit.batch + c, count);
    x.template load<kWide>(a.x.p + b * a.x.batch + c, count);
    const bool found = slot >= 0 && slot < a.num_slots;
    float2 h = splat(0.f);
    if (found) {
      const Decay d = decay2<false>(__fmul2_rn(sigmoid2(f.pair(0)), make_float2(-rate.x, -rate.y)));
      const int64_t at = slot * a.channels + c;
      const float2 add = __fmul2_rn(__fmul2_rn(d.m, sigmoid2(g.pair(0))), x.pair(0));
      h = decayed<true>(held(d), pair_at<kWide>(a.last, at, count), add);
      put_pair<kWide>(a.last, at, count, h);
    }
    y.set(0, h);
    y.template store<kWide>(a.y.p + b * a.y.batch + c, count);
  }
}

// ------------------------------------------------------------- host side
struct GatedPlan {
  int64_t batches, strips, size, entries;  // blocks of a cluster, along the batch
  int64_t row_seq, parts;                  // workspace, in words
};

GatedPlan plan_of(const tcu_gated_scan_args &a, bool grad) {
  GatedPlan p{};
  p.batches = a.offsets ? 1 : a.sequences;
  p.strips = (a.channels + kStrip - 1) / kStrip;
  p.entries = std::min<int64_t>(p.batches, 65535);
  // Blocks of a cluster share a strip's rows, where strips are fewer than the
  // card's places, two an SM: the largest size at which all clusters run at
  // once.  Large clusters find fewer places, since each lies within one part of
  // the card.  65536 x 1536, 24 strips, forward: 371, 302, 261, 320, 306 us in
  // clusters of 4, 8, 9, 12, 16; 4121 x 1031 f32, packed, 17 strips: 70, 53, 48,
  // 42, 60; 8192 x 4096, 64 strips: 78, 87 us in clusters of 4, 8; 8 x 2048 x 4096,
  // 512 strips: 124 us whole, 134 in clusters of 2 (launch included).
  const int64_t tile = grad ? kTile : kLongTile, tiles = (a.rows + tile - 1) / tile;
  const int64_t strips = p.strips * p.entries, sms = num_sms();
  p.size = 1;
  for (const int size : {16, 12, 9, 8, 6, 4, 3, 2})
    if (size <= tiles && strips * size <= (size > 4 ? sms * 29 / 20 : sms * 9 / 5)) {
      p.size = size;
      break;
    }
  p.row_seq = a.offsets ? (a.rows + 3) / 4 * 4 : 0;
  p.parts = grad ? p.entries * p.size * a.channels : 0;
  return p;
}

template <typename T>
GatedArgs<T> args_of(const tcu_gated_scan_args &s, const GatedPlan &p, bool step) {
  GatedArgs<T> a{};
  a.x = rows_of<const T>(s.x);
  a.forget = rows_of<const T>(s.forget);
  a.admit = rows_of<const T>(s.admit);
  a.y = rows_of<T>(s.y);
  a.dy = rows_of<const T>(s.dy);
  a.dx = rows_of<T>(s.dx);
  a.dforget = rows_of<T>(s.dforget);
  a.dadmit = rows_of<T>(s.dadmit);
  a.rate = s.rate;
  a.state = s.state;
  a.dlast = s.dlast;
  a.last = s.last;
  a.dstate = s.dstate;
  a.marks = s.marks;
  a.offsets = s.offsets;
  a.slots = s.slots;
  a.channels = s.channels;
  a.num_slots = s.num_slots;
  a.rows = (int)s.rows;
  a.sequences = s.sequences;
  a.batches = (int)p.batches;
  a.runs = (int)((s.rows + kRun - 1) / kRun);
  if (!step) {
    int32_t *w = static_cast<int32_t *>(s.workspace);
    a.row_seq = s.offsets ? w : nullptr;
    a.parts = reinterpret_cast<float *>(w + p.row_seq);
  }
  return a;
}

enum Call { kPrompt, kGrad, kStep };

template <typename K, typename T>
int start(K kernel, int bytes, const GatedPlan &p, const GatedArgs<T> &a, cudaStream_t st) {
  if (p.strips * p.size > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.strips * p.size), (unsigned)p.entries);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.size > 1 ? 1 : 0;
  cudaError_t e = cudaFuncSetAttribute((const void *)kernel,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && p.size > 8)
    e = cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, a, (int)p.size);
  if (e == cudaSuccess) return launched();
  cudaGetLastError();
  return TCU_DFT_ERR_CUDA;
}

template <typename T, bool kPacked, bool kWide>
int run_rows(Call call, const GatedPlan &p, const GatedArgs<T> &a, cudaStream_t st) {
  return call == kGrad
             ? start(gated_grad_kernel<T, kPacked, kWide>, (int)sizeof(GradShared<T>), p, a, st)
             : start(gated_kernel<T, kPacked, kWide>, (int)sizeof(GatedShared<T>), p, a, st);
}

template <typename T>
int run(Call call, const tcu_gated_scan_args &s, cudaStream_t st) {
  const GatedPlan p = plan_of(s, call == kGrad);
  GatedArgs<T> a = args_of<T>(s, p, call == kStep);
  const int64_t batches = call == kStep ? s.sequences : p.batches;
  // prompts are copied in 16 bytes, tokens read in pairs
  const int word = call == kStep ? 2 * (int)sizeof(T) : 16;
  bool wide = s.channels % (word / (int)sizeof(T)) == 0;
  for (const void *q : {(const void *)s.rate, (const void *)s.state, (const void *)s.dlast,
                        (const void *)s.last, (const void *)s.dstate, (const void *)s.marks,
                        (const void *)a.parts})
    wide = wide && (uintptr_t)q % 8 == 0;
  for (const tcu_seq_rows *r : {&s.x, &s.forget, &s.admit})
    wide = wide && rows_aligned(*r, s.type, batches, s.rows, word);
  if (call != kGrad) wide = wide && rows_aligned(s.y, s.type, batches, s.rows, word);
  else
    for (const tcu_seq_rows *r : {&s.dy, &s.dx, &s.dforget, &s.dadmit})
      wide = wide && rows_aligned(*r, s.type, batches, s.rows, word);
  if (call == kStep) {
    const int64_t blocks = (s.channels + 255) / 256;
    if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)std::min(s.sequences, 65535));
    if (wide) gated_step_kernel<T, true><<<grid, 128, 0, st>>>(a);
    else gated_step_kernel<T, false><<<grid, 128, 0, st>>>(a);
    return launched();
  }
  const bool none = p.batches == 0 || s.rows == 0;
  if (!none) {
    if (s.offsets) {
      row_sequence_kernel<<<(unsigned)((s.rows + 127) / 128), 128, 0, st>>>(
          const_cast<int32_t *>(a.row_seq), s.offsets, s.sequences, (int)s.rows);
      if (const int rc = launched()) return rc;
    }
    const int rc = s.offsets ? wide ? run_rows<T, true, true>(call, p, a, st)
                                    : run_rows<T, true, false>(call, p, a, st)
                   : wide    ? run_rows<T, false, true>(call, p, a, st)
                             : run_rows<T, false, false>(call, p, a, st);
    if (rc) return rc;
  }
  if (call != kGrad) return TCU_DFT_OK;
  const Sum sum = {s.drate, a.parts, s.channels};
  return sum_parts(&sum, 1, none ? 0 : p.entries * p.size, 0, st);
}

int by_type(Call call, const tcu_gated_scan_args &a, void *stream) {
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (a.type) {
    case TCU_SEQ_F32: return run<float>(call, a, st);
    case TCU_SEQ_BF16: return run<bf16>(call, a, st);
    default: return run<f16>(call, a, st);
  }
}

int check_sizes(const tcu_gated_scan_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->channels < 1)
    return TCU_DFT_ERR_INVALID;
  if (a->rows > kMostRows || a->channels > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r :
       {&a->x, &a->forget, &a->admit, &a->y, &a->dy, &a->dx, &a->dforget, &a->dadmit})
    if (!pitch_fits(a->rows, r->row_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  return TCU_DFT_OK;
}

bool inputs_ok(const tcu_gated_scan_args &a) {
  const int sz = type_size(a.type);
  return f32_ok(a.rate) && opt_ok(a.state, 4) && opt_ok(a.last, 4) && opt_ok(a.marks, 4) &&
         opt_ok(a.offsets, 4) && row_ok(a.x, sz) && row_ok(a.forget, sz) && row_ok(a.admit, sz);
}

bool workspace_ok(const tcu_gated_scan_args &a, const GatedPlan &p) {
  const int64_t bytes = 4 * (p.row_seq + p.parts);
  return a.workspace_bytes >= bytes && (bytes == 0 || f32_ok(a.workspace));
}

// Sequences without any row end in the state they start from.
int no_rows(const tcu_gated_scan_args &a, float *to, const float *from, void *stream) {
  if (!to || a.sequences == 0 || a.rows > 0) return TCU_DFT_OK;
  const size_t bytes = (size_t)a.sequences * a.channels * 4;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, st)
                             : cudaMemsetAsync(to, 0, bytes, st);
  if (e == cudaSuccess) return TCU_DFT_OK;
  cudaGetLastError();
  return TCU_DFT_ERR_CUDA;
}

bool any_rows(const tcu_gated_scan_args &a) {
  return a.rows > 0 && a.sequences + (a.offsets != nullptr) > 0;
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_gated_scan_workspace(const tcu_gated_scan_args *a) {
  if (check_sizes(a)) return -1;
  return 4 * plan_of(*a, false).row_seq;
}

extern "C" int64_t tcu_gated_scan_grad_workspace(const tcu_gated_scan_args *a) {
  if (check_sizes(a)) return -1;
  const GatedPlan p = plan_of(*a, true);
  return 4 * (p.row_seq + p.parts);
}

extern "C" int tcu_gated_scan(const tcu_gated_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (any_rows(*a) && (!inputs_ok(*a) || !row_ok(a->y, type_size(a->type)) ||
                       !workspace_ok(*a, plan_of(*a, false))))
    return TCU_DFT_ERR_INVALID;
  if (const int rc = no_rows(*a, a->last, a->state, stream)) return rc;
  return by_type(kPrompt, *a, stream);
}

extern "C" int tcu_gated_scan_grad(const tcu_gated_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  const int sz = type_size(a->type);
  if (!f32_ok(a->drate) || !opt_ok(a->dlast, 4) || !opt_ok(a->dstate, 4)) return TCU_DFT_ERR_INVALID;
  if (any_rows(*a) && (!inputs_ok(*a) || !a->marks || !row_ok(a->dy, sz) || !row_ok(a->dx, sz) ||
                       !row_ok(a->dforget, sz) || !row_ok(a->dadmit, sz) ||
                       !workspace_ok(*a, plan_of(*a, true))))
    return TCU_DFT_ERR_INVALID;
  if (const int rc = no_rows(*a, a->dstate, a->dlast, stream)) return rc;
  return by_type(kGrad, *a, stream);
}

extern "C" int tcu_gated_scan_step(const tcu_gated_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (a->rows != 1 || a->offsets || a->num_slots < 0 ||
      (!a->slots && a->num_slots < a->sequences) || !opt_ok(a->slots, 4))
    return TCU_DFT_ERR_INVALID;
  if (a->sequences == 0) return TCU_DFT_OK;
  const int sz = type_size(a->type);
  if (!inputs_ok(*a) || !row_ok(a->y, sz) || (a->num_slots > 0 && !a->last))
    return TCU_DFT_ERR_INVALID;
  const int64_t entry = a->channels * 4;
  const wide_int cache = (wide_int)a->num_slots * entry;
  for (const tcu_seq_rows *r : {&a->x, &a->forget, &a->admit, &a->y})
    if (over(a->last, cache, r->ptr, a->channels * sz, a->sequences, r->batch_stride * sz))
      return TCU_DFT_ERR_INVALID;
  if (over(a->last, cache, a->rate, entry) ||
      over(a->last, cache, a->slots, (int64_t)a->sequences * 4))
    return TCU_DFT_ERR_INVALID;
  return by_type(kStep, *a, stream);
}
