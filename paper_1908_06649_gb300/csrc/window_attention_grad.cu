// window_attention_grad.cu -- the gradient of window attention
// (include/tcu_attn.h).
//
// With the scores s_ij = scale q_i.k_j and weights p_ij = exp(s_ij - lse_i):
//     delta_i = dy_i.y_i,      dp_ij = dy_i.v_j,      ds_ij = p_ij (dp_ij - delta_i)
//     dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,   dv_j = sum_i p_ij dy_i
// over the visible pairs and, for dk and dv, the query heads of a key head.
//
// Two kernels form p and ds anew, one a block of 128 queries at a time for dq,
// one a block of 128 keys for dk and dv: seven products where five would do,
// but every sum stays in tensor memory, in a fixed order, and nothing is added
// up in memory.  What a thread owns is half of a row of the accumulator's 128;
// p and ds go back to tensor memory in the rows' type, over the scores that the
// thread has read, and the tiles of keys (queries) are read along their rows by
// the second products.  A warp each issues products, copies, and looks over
// tiles that not all rows see.
//
// Products bound it, 10 dim flops a visible pair and head (14 as done here).
// Measured, bf16, 4 x 2048 rows, 16 heads (4 of keys) x 128, window 1024 (1.3e11
// flops): dq 120 us, dk and dv 153 us, delta 16 us, joining 8 us: 0.44 PFLOP/s
// of what is asked for, 0.61 of what is done.  Tiles of 64 rows read the other
// operand anew from shared memory for each product (55 to 60 cycles where 32
// would do), and tensor memory holds no larger ones beside the sums.  At 640
// threads dkv_kernel has 96 registers, and spills 100 to 140 bytes of them.
#include <algorithm>

#include "attn_common.cuh"

namespace tcu {
namespace seq {
namespace {

constexpr int kRows = 128;  // of the block
constexpr int kStep = 64;   // of a tile that it walks over
constexpr int kSoft = 256;  // threads that form weights: two for each row

// fp16 holds 2^-14 to 2^16 with all its bits, less than weights of long rows and
// gradients of different sizes span.  So its p goes to dv's product times 2^12
// (and may be 16, where an lse of some millions is rounded), and ds times a power
// of two of its own for each row of an accumulator, which brings the row's largest
// term near 2^6: in dq a row's, from the terms seen so far, with the sums brought
// to a new one where a term passes 2^14; in dk a key's, from the largest term of
// its column, which dq_kernel leaves.  What one row or key brings says nothing of
// another's.  (bf16 has fp32's range.)  It costs dq_kernel a barrier, a maximum and
// 31 exchanges between lanes a tile: 16 heads (4) x 128, 4 x 4096 rows, window 300,
// gradient 416 us, in bf16 375.
template <typename T>
constexpr bool kNarrow = __is_same(T, f16);
constexpr int kWeightUp = 12, kTermUp = 6, kTermRoom = 8;
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// The power for terms whose largest has the biased exponent e, at least kLeast.
constexpr int kLeast = 32;
__device__ __forceinline__ float lift_of(int e) { return power_of_two(kTermUp + 127 - e); }
// dq and dk form ds with deltas that differ by the rounding of y, and so not
// from terms of the same size where ds is next to nothing: a term's size has
// this part of p sum_c |dy_c y_c| added.
constexpr float kSlack = 1.f / 512;

// ------------------------------------------------------------------- delta
// delta = dy.y of each row and head, 16 lanes a head; for fp16 the sum of the
// products' sizes too, and zeros for the largest terms of keys.
template <typename T>
__global__ void __launch_bounds__(256) delta_kernel(const Rows<const T> y, const Rows<const T> dy,
                                                    float *delta, const AttendArgs a, int64_t total,
                                                    int64_t keys) {
  const int64_t step = (int64_t)gridDim.x * 16;
  const int lane = threadIdx.x % 16;
  for (int64_t pair = (int64_t)blockIdx.x * 16 + threadIdx.x / 32 * 2; pair < total; pair += step) {
    const int64_t id = pair + threadIdx.x / 16 % 2;
    float sum = 0.f, size = 0.f;
    if (id < total && lane * 8 < a.dim) {
      const int64_t row = id / a.heads, b = row / a.rows, t = row - b * a.rows;
      const int64_t at = (id - row * a.heads) * a.dim + lane * 8;
      const Vec<T, 8> u = *reinterpret_cast<const Vec<T, 8> *>(y.at(b, (int)t) + at);
      const Vec<T, 8> v = *reinterpret_cast<const Vec<T, 8> *>(dy.at(b, (int)t) + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(to_f(u.v[i]), to_f(v.v[i]), sum);
        if constexpr (kNarrow<T>) size = fmaf(fabsf(to_f(u.v[i])), fabsf(to_f(v.v[i])), size);
      }
    }
#pragma unroll
    for (int m = 1; m < 16; m *= 2) {
      sum += __shfl_xor_sync(~0u, sum, m);
      if constexpr (kNarrow<T>) size += __shfl_xor_sync(~0u, size, m);
    }
    if (lane == 0 && id < total) {
      delta[id] = sum;
      if constexpr (kNarrow<T>) {
        a.sizes[id] = size;
        if (id < keys) a.peaks[id] = 0;
      }
    }
  }
}

// The largest of 32 values, none below zero, of each of 32 columns, over the
// warp's rows (a lane has one row): lane j leaves column j's, its upper 16
// bits, in *to.  Halves of the columns change places five times.
__device__ __forceinline__ void column_peaks(const float *m, int lane, uint32_t *to) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    w[i] = __byte_perm(__float_as_uint(m[2 * i]), __float_as_uint(m[2 * i + 1]), 0x7632);
#pragma unroll
  for (int n = 8; n >= 1; n /= 2) {
    const bool upper = lane & 2 * n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const uint32_t keep = upper ? w[i + n] : w[i], send = upper ? w[i] : w[i + n];
      w[i] = __vmaxu2(keep, __shfl_xor_sync(~0u, send, 2 * n));
    }
  }
  w[0] = __vmaxu2(w[0], __shfl_xor_sync(~0u, w[0], 1));
  const uint32_t own = lane & 1 ? w[0] & 0xffff0000u : w[0] << 16;
  if (own) atomicMax(to + lane, own);  // of all rows: the order of a maximum has no say
}

// ---------------------------------------------------------------------- dq
struct QueryMaps {
  CUtensorMap q, dy, k, v;  // k and v in boxes of kStep rows
};

template <int DP>
struct QueryShared {
  uint8_t q[kTileBytes<DP, kRows>], dy[kTileBytes<DP, kRows>];
  uint8_t k[2][kTileBytes<DP, kStep>], v[kTileBytes<DP, kStep>];
  uint64_t full_k[2], full_v, scores, weights, done[2];
  union {
    float sums[kRows];
    uint8_t tops[2][2][kRows];  // exponents of largest terms: [turn][half]
  };
  uint32_t tmem;
  int low, high, sink_at, sink_end, failed;
};

constexpr int kTwice = 4;

// Two blocks share an SM, which holds 228 KB, 1 KB beside each block's own.
static_assert(2 * (sizeof(QueryShared<128>) + 1024) <= 228 * 1024, "two blocks an SM");

template <typename T, int DP>
__global__ void __launch_bounds__(kSoft + 64, 2)
    dq_kernel(const __grid_constant__ QueryMaps maps, const AttendArgs a, const Rows<T> dq,
              float *exact) {
  extern __shared__ __align__(1024) uint8_t raw[];
  QueryShared<DP> &s = *reinterpret_cast<QueryShared<DP> *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t id = blockIdx.x;
  const int tile = (int)(id % a.q_tiles);
  const int head = (int)(id / a.q_tiles % a.heads), batch = (int)(id / a.q_tiles / a.heads);
  const int kv = head / (a.heads / a.kv_heads);
  const uint32_t full_k = smem_u32(s.full_k), full_v = smem_u32(&s.full_v),
                 scores = smem_u32(&s.scores), weights = smem_u32(&s.weights),
                 done = smem_u32(s.done);
  if (threadIdx.x == 0) {
    mbar_init(done + 8, 1);
    mbar_init(full_k, 1);
    mbar_init(full_k + 8, 1);
    mbar_init(full_v, 1);
    mbar_init(scores, 1);
    mbar_init(weights, kSoft + 32);
    mbar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.low = INT32_MAX;
    s.high = 0;
    s.sink_end = 0;
    s.failed = 0;
  }
  if (warp == kSoft / 32) tmem_alloc(smem_u32(&s.tmem), 256);
  Seen seen{-1, INT32_MAX, 0, 0};
  const int own = threadIdx.x % kRows;
  if (threadIdx.x < kSoft) seen = seen_by(a, (int64_t)tile * kRows + own);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  if (threadIdx.x < kSoft) {
    const int low = __reduce_min_sync(~0u, seen.lo);
    const int high = __reduce_max_sync(~0u, seen.i >= 0 ? seen.lo : 0);
    if (lane == 0) {
      atomicMin(&s.low, low);
      atomicMax(&s.high, high);
    }
  }
  __syncthreads();
  const int first = s.low / kStep;
  if (threadIdx.x < kSoft && seen.s0 < seen.s1 && seen.s0 < (int64_t)first * kStep) {
    atomicMax(&s.sink_end, min(seen.s1, first * kStep));
    s.sink_at = seen.s0 / kStep;
  }
  __syncthreads();
  const uint32_t tmem = s.tmem, tS = tmem, tP = tmem + kStep, tQ = tmem + 2 * kStep;
  const bool any = s.low != INT32_MAX;
  const int sink_tiles = s.sink_end > 0 ? (s.sink_end - 1) / kStep - s.sink_at + 1 : 0;
  const int sink_first = sink_tiles ? s.sink_at : 0;
  const int last = (int)min((int64_t)tile * 2 + 1, (a.rows - 1) / kStep);
  const int tiles = any ? sink_tiles + last - first + 1 : 0;
  const auto key_row = [&](int t) {
    return (t < sink_tiles ? sink_first + t : first + t - sink_tiles) * kStep;
  };
  // delta from the rounded y is off by what it is rounded by, which counts where
  // a row sees few keys and y is as large as they are: few tiles are walked over
  // twice, and delta is the sum of p dp that the first walk finds
  const int before = tiles <= kTwice ? tiles : 0, steps = before + tiles;
  const auto row_at = [&](int t) { return key_row(t < before ? t : t - before); };
  const float c = a.scale * kLog2e;

  // whether not all rows see all keys of a tile
  const auto edge = [&](int j0) { return j0 < s.high || j0 + kStep - 1 > tile * kRows; };
  const uint32_t q = smem_u32(s.q), dy = smem_u32(s.dy), k = smem_u32(s.k), v = smem_u32(s.v);
  constexpr uint32_t bytes = kTileBytes<DP, kStep>;
  if (warp == kSoft / 32 + 1) {  // copies, and a look at keys that not all rows see
    const Filled filled(a);
    bool ok = true;
    int keys = 0, values = 0;  // tiles asked for
    // after the scores: keys in no sequence, and those that are not finite, go
    // (who sees one of the latter has no number for its lse)
    const auto look = [&](int t) {
      if (t >= before && edge(row_at(t))) {
        clean_tile<T, DP, 32>(k + (t & 1) * bytes, lane, row_at(t), filled, nullptr);
        fence_proxy_async_shared();
      }
      mbar_arrive(weights);
    };
    for (int t = 0; t < steps && ok; ++t) {
      const uint32_t stage = t & 1;
      // dq of t - 2 has read its keys, the scores of t - 1 their values
      if (t > 1) ok = warp_waits(done + 8 * stage, ((t - 2) >> 1) & 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(full_k + 8 * stage, bytes + (t == 0 ? 2 * kTileBytes<DP, kRows> : 0));
        if (t == 0) {
          load_tile<DP, kRows>(q, &maps.q, head, tile * kRows, batch, full_k);
          load_tile<DP, kRows>(dy, &maps.dy, head, tile * kRows, batch, full_k);
        }
        load_tile<DP, kStep>(k + stage * bytes, &maps.k, kv, row_at(t), batch, full_k + 8 * stage);
      }
      __syncwarp();
      keys = t + 1;
      if (t > 0) ok = warp_waits(scores, (t - 1) & 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(full_v, bytes);
        load_tile<DP, kStep>(v, &maps.v, kv, row_at(t), batch, full_v);
      }
      __syncwarp();
      values = t + 1;
      if (t > 0) look(t - 1);
    }
    if (steps > 0 && ok) {
      ok = warp_waits(scores, (steps - 1) & 1);
      look(steps - 1);
    }
    if (!ok) {  // copies in flight end before the block does
      s.failed = 1;
      if (values > 0) warp_waits(full_v, (values - 1) & 1);
      for (int i = 1; i <= 2; ++i)
        if (keys >= i) warp_waits(full_k + 8 * ((keys - i) & 1), ((keys - i) >> 1) & 1);
    }
  } else if (warp == kSoft / 32) {  // products
    bool ok = true;
    for (int t = 0; t < steps; ++t) {
      const uint32_t ph = t & 1, stage = t & 1;
      ok = warp_waits(full_k + 8 * stage, (t >> 1) & 1) && warp_waits(full_v, ph);
      // scores take the place of what the last product has read
      if (t > 0) ok = ok && warp_waits(done + 8 * (stage ^ 1), ((t - 1) >> 1) & 1);
      if (!ok) break;
      fence_after_sync();
      if (elect_one()) {
        product_rows<T, DP, kStep>(tS, q, k + stage * bytes);
        product_rows<T, DP, kStep>(tP, dy, v);
        mma_commit(scores);
      }
      __syncwarp();
      ok = warp_waits(weights, ph);
      if (!ok) break;
      fence_after_sync();
      if (elect_one()) {
        if (t >= before) product_values<T, DP, kStep>(tQ, tS, k + stage * bytes, t > before);
        mma_commit(done + 8 * stage);
      }
      __syncwarp();
    }
    if (!ok) s.failed = 1;
  } else {
    const int half = threadIdx.x / kRows;  // of the row: 32 keys, and half of its dq
    const uint32_t mine = (uint32_t)((warp % 4) * 32) << 16;
    const int64_t at = ((int64_t)batch * a.rows + max(0, seen.i)) * a.heads + head;
    float lse = 0.f, delta = 0.f, slack = 0.f;
    if (seen.i >= 0) {
      lse = a.lse[at] * kLog2e;
      delta = a.delta[at];
      if constexpr (kNarrow<T>) slack = a.sizes[at] * kSlack;
    }
    int top = kLeast;  // exponent that the row's terms are brought near 2^kTermUp from
    float lift = 1.f;
    float2 total = splat(0.f);
    bool ok = true;
    for (int t = 0; t < steps; ++t) {
      const uint32_t ph = t & 1;
      const int j0 = row_at(t);
      // a warp whose wait ran out goes on without waiting: others share its barriers
      ok = ok && warp_waits(scores, ph);
      fence_after_sync();
      const int j1 = j0 + 32 * half;
      float v[64];
      uint32_t w[16];
      tmem_ld32x2(tS + mine + 32 * half, tP + mine + 32 * half, v);
      const float2 by = splat(c), minus = splat(-lse), less = splat(-delta);
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        const float2 z = __ffma2_rn(make_float2(v[j], v[j + 1]), by, minus);
        const float2 d = __fadd2_rn(make_float2(v[32 + j], v[33 + j]), less);
        const float2 p = make_float2(exp2_fast(z.x), exp2_fast(z.y)), x = __fmul2_rn(p, d);
        v[j] = x.x;
        v[j + 1] = x.y;
        if constexpr (kNarrow<T>) {  // the terms' sizes
          const float2 m = __fmul2_rn(p, __fadd2_rn(make_float2(fabsf(d.x), fabsf(d.y)), splat(slack)));
          v[32 + j] = m.x;
          v[33 + j] = m.y;
        }
      }
      if (!__all_sync(~0u, seen.whole(j1, j1 + 32))) {
        const uint32_t bits = seen.bits(j1);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          v[j] = bits >> j & 1 ? v[j] : 0.f;
          if constexpr (kNarrow<T>) v[32 + j] = bits >> j & 1 ? v[32 + j] : 0.f;
        }
      }
      if constexpr (kNarrow<T>) {
        if (t >= before) {
          column_peaks(v + 32, lane, a.peaks + ((int64_t)batch * a.kv_heads + kv) * a.rows + j1);
          float most = v[32];
#pragma unroll
          for (int j = 1; j < 32; ++j) most = fmaxf(most, v[32 + j]);
          int e = __float_as_int(most) >> 23;
          s.tops[t & 1][half][own] = (uint8_t)e;
          asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
          e = max(e, (int)s.tops[t & 1][half ^ 1][own]);
          const bool rise = t == before || e > top + kTermRoom;
          if (t > before && __any_sync(~0u, rise)) {
            // the product before has ended: the scores were asked for after it
            const float less = rise ? power_of_two(max(top - e, -126)) : 1.f;
#pragma unroll 1
            for (int k = DP / 2 * half; k < DP / 2 * (half + 1); k += 16) {
              float o[16];
              tmem_ld16(tQ + mine + k, o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] *= less;
              tmem_st16(tQ + mine + k, o);
            }
          }
          if (rise) top = max(e, kLeast);
          lift = lift_of(top);
        }
      }
      const float2 up = splat(lift);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        float2 x = make_float2(v[2 * j], v[2 * j + 1]);
        total = __fadd2_rn(total, x);
        if constexpr (kNarrow<T>) x = __fmul2_rn(x, up);
        w[j] = pack2<T>(x.x, x.y);
      }
      if (t >= before) tmem_st16u(tS + mine + 32 * half, w);
      if (t == before - 1) {  // both halves take their joint sum
        if (half == 1) s.sums[own] = total.x + total.y;
        asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
        if (half == 0) s.sums[own] += total.x + total.y;
        asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
        delta += s.sums[own];
        total = splat(0.f);
        if constexpr (kNarrow<T>) asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
      }
      tmem_wait_st();
      fence_before_sync();
      mbar_arrive(weights);
    }
    if (steps > 0) ok = ok && warp_waits(done + 8 * ((steps - 1) & 1), ((steps - 1) >> 1) & 1);
    if (!ok) s.failed = 1;
    fence_after_sync();
    // a row's ds add up to nothing: what they do add up to is what delta, from
    // the rounded y, is off by, and dk takes it without
    if constexpr (kNarrow<T>) asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
    if (half == 1) s.sums[own] = total.x + total.y;
    asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
    const float bad = s.failed ? __int_as_float(0x7fffffff) : 1.f;  // no number
    if (half == 0 && seen.i >= 0) exact[at] = bad * (delta + s.sums[own] + total.x + total.y);
    const int64_t i = (int64_t)tile * kRows + own;
    const bool row = i < a.rows;
    const float by = bad * a.scale / lift;
    T *to = dq.at(batch, row ? (int)i : 0) + (int64_t)head * a.dim;
#pragma unroll 1
    for (int k = DP / 2 * half; k < DP / 2 * (half + 1); k += 32) {
      float o[32];
      if (tiles > 0) tmem_ld32(tQ + mine + k, o);
      if (tiles == 0 || seen.i < 0) {  // rows of no sequence
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = 0.f;
      }
      if (row) store_values(to, k, a.dim, o, by);
    }
    fence_before_sync();
  }
  __syncthreads();
  if (warp == kSoft / 32) tmem_dealloc(tmem, 256);
}

// --------------------------------------------------------------- dk and dv
struct KeyMaps {
  CUtensorMap k, v, q, dy;  // q and dy in boxes of kStep rows
};

constexpr int kStages = 4;

template <int DP>
struct KeyShared {
  uint8_t k[kTileBytes<DP, kRows>], v[kTileBytes<DP, kRows>];
  uint8_t q[kStages][kTileBytes<DP, kStep>], dy[kStages][kTileBytes<DP, kStep>];
  float4 lse[2][2][kStep / 4], delta[2][2][kStep / 4];  // of a tile's query rows: [side][turn]
  uint64_t full_kv, full[kStages], read[kStages], scores[2], weights[2], done[2];
  uint32_t tmem;
  int last, begin, least, failed;
};

// A tile of queries of one head among those that a block walks over.
struct QueryTile {
  int head, at;
  __device__ __forceinline__ void forward(int by, int first, int end) {
    at += by;
    while (at >= end) at -= end - first, ++head;
  }
};

// The first chunk that a tile's first tokens leave to far blocks, and where
// sums of a chunk and the nth tile of a sequence's first tokens lie.
__device__ __forceinline__ int far_from(const AttendArgs &a, int tile) {
  return (tile * (kRows / kStep) + 2 * a.chunk - 1) / a.chunk;
}
__device__ __forceinline__ int64_t slot_of(const AttendArgs &a, int batch, int x, int nth, int kv) {
  return (((int64_t)batch * a.chunks + x) * a.sink_tiles + nth) * a.kv_heads + kv;
}

// Two sides of 256 threads take the tiles of queries in turn: while one forms
// weights, the tensor cores work on the other's tile.  Of a side's threads two
// share a key, 32 queries each.
//
// Most keys are seen from a window's rows, first tokens from all rows of
// their sequence.  So that no block walks over more tiles than twice another,
// those beyond the first multiple of `chunk` that is `chunk` tiles or more
// behind the key tile go, `chunk` at a time, to blocks of their own, the first
// `far_blocks` of the launch.  A chunk has far first tokens of one sequence at
// most, that of its first row.  Such sums, and the key tile's own, go to
// memory in fp32, [chunk][tile of first tokens], a key tile's own behind all far
// ones, at its first far chunk; join_kernel adds them in order.
template <typename T, int DP>
__global__ void __launch_bounds__(2 * kSoft + 128, 1)
    dkv_kernel(const __grid_constant__ KeyMaps maps, const AttendArgs a, const Rows<T> dk,
               const Rows<T> dv, float *sums, int far_blocks) {
  extern __shared__ __align__(1024) uint8_t raw[];
  KeyShared<DP> &s = *reinterpret_cast<KeyShared<DP> *>(raw);
  const int warp = threadIdx.x / 32;
  const bool is_far = blockIdx.x < far_blocks;
  int64_t id = is_far ? blockIdx.x : blockIdx.x - far_blocks;
  const int kv = (int)(id % a.kv_heads);
  id /= a.kv_heads;
  const int group = a.heads / a.kv_heads;
  int tile, batch, first, end = 0;  // tiles of queries: [first, end)
  int64_t slot = -1;                // of fp32 sums
  if (is_far) {
    const int nth = (int)(id % a.sink_tiles);
    id /= a.sink_tiles;
    const int x = (int)(id % a.chunks);
    batch = (int)(id / a.chunks);
    slot = blockIdx.x;
    int b, e;
    if (!sequence_at(a, (int64_t)x * a.chunk * kStep, b, e)) return;
    tile = b / kRows + nth;
    if ((int64_t)tile * kRows >= (int64_t)b + a.sinks || x < far_from(a, tile)) return;
    first = x * a.chunk;
    end = (int)min((int64_t)first + a.chunk, ((int64_t)e + kStep - 1) / kStep);
  } else {  // early tiles, which are seen from most rows, before late ones
    const int64_t batches = (gridDim.x - far_blocks) / a.kv_heads / a.k_tiles;
    batch = (int)(id % batches);
    tile = (int)(id / batches);
    first = tile * (kRows / kStep);
  }
  const uint32_t full_kv = smem_u32(&s.full_kv), full = smem_u32(s.full),
                 scores = smem_u32(s.scores), weights = smem_u32(s.weights), done = smem_u32(s.done),
                 read = smem_u32(s.read);
  if (threadIdx.x == 0) {
    mbar_init(full_kv, 1);
    for (int i = 0; i < kStages; ++i) mbar_init(full + 8 * i, 1), mbar_init(read + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(scores + 8 * i, 1);
      mbar_init(weights + 8 * i, kSoft + 64);
      mbar_init(done + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.last = 0;
    s.least = INT32_MAX;
    s.failed = 0;
  }
  if (warp == 2 * kSoft / 32) tmem_alloc(smem_u32(&s.tmem), 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  // this thread's key is seen from rows [j, past)
  const int64_t j64 = (int64_t)tile * kRows + threadIdx.x % kRows;
  const int j = (int)min(j64, (int64_t)INT32_MAX);
  int begin = 0, past = 0;
  {
    int e;
    if (sequence_at(a, j64, begin, e))
      past = j - begin < a.sinks || e - j <= a.window ? e : j + a.window;
  }
  const int least = __reduce_min_sync(~0u, past > 0 ? past : INT32_MAX);
  if (threadIdx.x % 32 == 0) atomicMin(&s.least, least);
  if (is_far) {
    __syncthreads();
  } else {
    const int top = __reduce_max_sync(~0u, past);
    if (threadIdx.x % 32 == 0) atomicMax(&s.last, top);
    __syncthreads();
    if (past > 0 && past == s.last) s.begin = begin;
    end = max(first, (s.last + kStep - 1) / kStep);
    __syncthreads();
    if (a.chunk > 0 && end > far_from(a, tile) * a.chunk) {
      const int x = far_from(a, tile);
      end = x * a.chunk;
      slot = far_blocks + slot_of(a, batch, x, tile - s.begin / kRows, kv);
    }
  }
  const uint32_t tmem = s.tmem, tV = tmem + 256, tK = tV + DP;
  const int64_t n = (int64_t)max(0, end - first) * group;
  const float c = a.scale * kLog2e;

  const uint32_t k = smem_u32(s.k), v = smem_u32(s.v), q = smem_u32(s.q), dy = smem_u32(s.dy);
  constexpr uint32_t bytes = kTileBytes<DP, kStep>;
  // whether not all keys of the block are seen from all rows of a tile
  const auto edge = [&](int i0) { return i0 < (tile + 1) * kRows - 1 || i0 + kStep > s.least; };
  if (warp >= 2 * kSoft / 32 + 2) {
    // a look at queries (one warp) and dy (another), after the scores: rows in no
    // sequence, and those that are not finite, go; a key that one of the latter
    // sees has no number for its gradients, dk through p or dp, dv through dp
    const Filled filled(a);
    const uint32_t from = warp == 2 * kSoft / 32 + 2 ? q : dy;
    QueryTile next{kv * group, first};
    for (int64_t t = 0; t < n; ++t, next.forward(1, first, end)) {
      if (!warp_waits(scores + 8 * (t & 1), (uint32_t)(t >> 1) & 1)) {
        s.failed = 1;
        break;
      }
      if (edge(next.at * kStep)) {
        clean_tile<T, DP, 32>(from + (uint32_t)t % kStages * bytes, threadIdx.x % 32, next.at * kStep,
                              filled, nullptr);
        fence_proxy_async_shared();
      }
      mbar_arrive(weights + 8 * (t & 1));
    }
  } else if (warp == 2 * kSoft / 32 + 1) {  // copies
    bool ok = true;
    int64_t asked = 0;
    QueryTile next{kv * group, first};
    if (n > 0) {
      if (elect_one()) {
        mbar_expect_tx(full_kv, 2 * kTileBytes<DP, kRows>);
        load_tile<DP, kRows>(k, &maps.k, kv, tile * kRows, batch, full_kv);
        load_tile<DP, kRows>(v, &maps.v, kv, tile * kRows, batch, full_kv);
      }
      __syncwarp();
    }
    for (; asked < n; ++asked, next.forward(1, first, end)) {
      const uint32_t stage = (uint32_t)asked % kStages;
      // the products of the tile before in this place have read it
      if (asked >= kStages)
        ok = warp_waits(read + 8 * stage, (uint32_t)(asked / kStages - 1) & 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(full + 8 * stage, 2 * bytes);
        load_tile<DP, kStep>(q + stage * bytes, &maps.q, next.head, next.at * kStep, batch,
                             full + 8 * stage);
        load_tile<DP, kStep>(dy + stage * bytes, &maps.dy, next.head, next.at * kStep, batch,
                             full + 8 * stage);
      }
      __syncwarp();
    }
    if (!ok) {  // copies in flight end before the block does
      s.failed = 1;
      warp_waits(full_kv, 0);
      for (int64_t u = max((int64_t)0, asked - kStages); u < asked; ++u)
        warp_waits(full + 8 * ((uint32_t)u % kStages), (uint32_t)(u / kStages) & 1);
    }
  } else if (warp == 2 * kSoft / 32) {  // products
    bool ok = n == 0 || warp_waits(full_kv, 0);
    for (int64_t t = 0; n > 0 && t <= n && ok; ++t) {
      if (t < n) {
        const uint32_t side = t & 1, stage = (uint32_t)t % kStages;
        ok = warp_waits(full + 8 * stage, (uint32_t)(t / kStages) & 1);
        // the side's tensor memory has been read
        if (t >= 2) ok = ok && warp_waits(done + 8 * side, ((t - 2) >> 1) & 1);
        if (!ok) break;
        fence_after_sync();
        if (elect_one()) {
          product_rows<T, DP, kStep>(tmem + 128 * side, k, q + stage * bytes);
          product_rows<T, DP, kStep>(tmem + 128 * side + kStep, v, dy + stage * bytes);
          mma_commit(scores + 8 * side);
        }
        __syncwarp();
      }
      if (t > 0) {
        const int64_t u = t - 1;
        const uint32_t side = u & 1, stage = (uint32_t)u % kStages;
        ok = warp_waits(weights + 8 * side, (uint32_t)(u >> 1) & 1);
        if (!ok) break;
        fence_after_sync();
        if (elect_one()) {
          product_values<T, DP, kStep>(tV, tmem + 128 * side, dy + stage * bytes, u > 0);
          product_values<T, DP, kStep>(tK, tmem + 128 * side + kStep, q + stage * bytes, u > 0);
          mma_commit(done + 8 * side);
          mma_commit(read + 8 * stage);
        }
        __syncwarp();
      }
    }
    if (!ok) s.failed = 1;
  } else {
    const int side = threadIdx.x / kSoft, own = threadIdx.x % kSoft;
    const int half = own / kRows;  // of the tile's queries
    const uint32_t mine = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t tS = tmem + 128 * side + 32 * half + mine, tP = tS + kStep;
    float lift = 1.f;  // of the thread's key
    if constexpr (kNarrow<T>)
      if (past > 0) {
        const uint32_t most = a.peaks[((int64_t)batch * a.kv_heads + kv) * a.rows + j];
        lift = lift_of(max((int)(most >> 23), kLeast));
      }
    // what the next tile's query rows bring, a row a thread: asked for a tile
    // ahead, and not touched before it is needed
    float lse = 0.f, delta = 0.f;
    QueryTile next{kv * group, first};
    const auto fetch = [&](int64_t t) {
      const int64_t i = (int64_t)next.at * kStep + own;
      if (own < kStep && t < n && i < a.rows) {
        const int64_t at = ((int64_t)batch * a.rows + i) * a.heads + next.head;
        lse = a.lse[at];
        delta = a.delta[at];
      }
    };
    if (n > 0 && side) next.forward(1, first, end);
    fetch(side);
    bool ok = true;
    for (int64_t t = side; t < n; t += 2) {
      const int turn = (t >> 1) & 1;
      if (own < kStep) {
        reinterpret_cast<float *>(s.lse[side][turn])[own] =
            fmaf(-lse, kLog2e, kNarrow<T> ? (float)kWeightUp : 0.f);
        reinterpret_cast<float *>(s.delta[side][turn])[own] = -delta;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + side), "n"(kSoft) : "memory");
      const int i0 = next.at * kStep, i1 = i0 + 32 * half;
      next.forward(2, first, end);
      fetch(t + 2);
      // a warp whose wait ran out goes on without waiting: others share its barriers
      ok = ok && warp_waits(scores + 8 * side, (uint32_t)(t >> 1) & 1);
      fence_after_sync();
      float v[64];
      tmem_ld32x2(tS, tP, v);
      const float2 by = splat(c), up = splat(lift * power_of_two(-kWeightUp));
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const float4 l = s.lse[side][turn][8 * half + i / 4], d = s.delta[side][turn][8 * half + i / 4];
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const float2 z = __ffma2_rn(make_float2(v[i + k], v[i + k + 1]), by,
                                      k ? make_float2(l.z, l.w) : make_float2(l.x, l.y));
          float2 x = __fadd2_rn(make_float2(v[32 + i + k], v[33 + i + k]),
                                k ? make_float2(d.z, d.w) : make_float2(d.x, d.y));
          if constexpr (kNarrow<T>) x = __fmul2_rn(x, up);
          const float2 p = make_float2(exp2_fast(z.x), exp2_fast(z.y)), ds = __fmul2_rn(p, x);
          v[i + k] = p.x;
          v[i + k + 1] = p.y;
          v[32 + i + k] = ds.x;
          v[33 + i + k] = ds.y;
        }
      }
      if (edge(i0)) {
        const uint32_t bits = bits_between(j - i1, past - i1);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          v[i] = bits >> i & 1 ? fmaf(v[32 + i], 0.f, v[i]) : 0.f;
          v[32 + i] = bits >> i & 1 ? v[32 + i] : 0.f;
        }
      }
      uint32_t w[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) w[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
      tmem_st16u(tS, w);
      tmem_st16u(tP, w + 16);
      tmem_wait_st();
      fence_before_sync();
      mbar_arrive(weights + 8 * side);
    }
    // all products: the last tile's after the one's before, as a barrier may be
    // waited for only one phase ahead
    if (n > 1) ok = ok && warp_waits(done + 8 * (n & 1), (uint32_t)((n - 2) >> 1) & 1);
    if (n > 0) ok = ok && warp_waits(done + 8 * ((n - 1) & 1), (uint32_t)((n - 1) >> 1) & 1);
    if (!ok) s.failed = 1;
    asm volatile("bar.sync 3, %0;" ::"n"(2 * kSoft) : "memory");
    fence_after_sync();
    // side 0 stores dv, side 1 dk, each thread half of a row
    const int r = own % kRows;
    const float bad = s.failed ? __int_as_float(0x7fffffff) : 1.f;
    const float by = bad * (side ? a.scale / lift : kNarrow<T> ? power_of_two(-kWeightUp) : 1.f);
    const bool in = past > 0;
    T *to = (side ? dk : dv).at(batch, j64 < a.rows ? j : 0) + (int64_t)kv * a.dim;
#pragma unroll 1
    for (int k = DP / 2 * half; k < DP / 2 * (half + 1); k += 32) {
      float o[32];
      if (n > 0) tmem_ld32((side ? tK : tV) + mine + k, o);
      if (n == 0 || !in) {  // rows of no sequence
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = 0.f;
      }
      if (slot >= 0) {
        float *row = sums + ((slot * 2 + side) * kRows + r) * DP + k;
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          *reinterpret_cast<float4 *>(row + i) =
              make_float4(o[i] * by, o[i + 1] * by, o[i + 2] * by, o[i + 3] * by);
      } else if (j64 < a.rows) {
        store_values(to, k, a.dim, o, by);
      }
    }
    fence_before_sync();
  }
  __syncthreads();
  if (warp == 2 * kSoft / 32) tmem_dealloc(tmem, 512);
}

// The sums of key tiles that far blocks share, eight blocks a tile, head and
// entry: few tiles have any, and one block each took 45 us.
constexpr int kJoin = 8;
template <typename T, int DP>
__global__ void __launch_bounds__(kRows) join_kernel(const AttendArgs a, const Rows<T> dk,
                                                     const Rows<T> dv, const float *sums,
                                                     int far_blocks) {
  __shared__ int last, first;
  int64_t id = blockIdx.x;
  const int kv = (int)(id % a.kv_heads);
  id /= a.kv_heads;
  const int64_t batches = gridDim.x / a.kv_heads / a.k_tiles;
  const int batch = (int)(id % batches), tile = (int)(id / batches);
  const int64_t j = (int64_t)tile * kRows + threadIdx.x;
  int begin = 0, e = 0, past = 0;
  if (threadIdx.x == 0) last = 0;
  __syncthreads();
  if (sequence_at(a, j, begin, e))
    past = j - begin < a.sinks || e - j <= a.window ? e : (int)j + a.window;
  const int top = __reduce_max_sync(~0u, past);
  if (threadIdx.x % 32 == 0) atomicMax(&last, top);
  __syncthreads();
  if (past > 0 && past == last) first = begin;
  __syncthreads();
  const int from = far_from(a, tile), end = (last + kStep - 1) / kStep;
  if (end <= from * a.chunk) return;
  const int to = (end + a.chunk - 1) / a.chunk, nth = tile - first / kRows;
  // eight adjacent values of a row a thread at a time
  for (int i = blockIdx.y * kRows + threadIdx.x; i < 2 * kRows * (DP / 8); i += kJoin * kRows) {
    const int c = i % (DP / 8) * 8, r = i / (DP / 8) % kRows, side = i / (DP / 8) / kRows;
    if (c >= a.dim || (int64_t)tile * kRows + r >= a.rows) continue;
    float v[8] = {};
    for (int x = from - 1; x < to; ++x) {
      const int64_t slot = x < from ? far_blocks + slot_of(a, batch, from, nth, kv)
                                    : slot_of(a, batch, x, nth, kv);
      const float4 *p =
          reinterpret_cast<const float4 *>(sums + ((slot * 2 + side) * kRows + r) * DP + c);
      const float4 f = p[0], g = p[1];
      v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
      v[4] += g.x, v[5] += g.y, v[6] += g.z, v[7] += g.w;
    }
    uint4 w;
    w.x = pack2<T>(v[0], v[1]), w.y = pack2<T>(v[2], v[3]);
    w.z = pack2<T>(v[4], v[5]), w.w = pack2<T>(v[6], v[7]);
    T *row = (side ? dk : dv).at(batch, tile * kRows + r) + (int64_t)kv * a.dim;
    *reinterpret_cast<uint4 *>(row + c) = w;
  }
}

// Tiles of queries to a chunk: what a key outside the first tokens is seen
// from, 16 at least; 0 where nothing is split.  Past 256 first tokens most
// blocks walk over a whole sequence, and need not be made alike.
void split_rows(const tcu_window_attention_args &s, AttendArgs &a) {
  const int64_t tiles = (s.rows + kStep - 1) / kStep;
  const int64_t chunk = std::max<int64_t>(16, ((int64_t)a.window + kRows + kStep - 1) / kStep + 1);
  a.chunk = a.chunks = a.sink_tiles = 0;
  if (a.sinks == 0 || a.sinks > 256 || tiles <= chunk) return;
  a.chunk = (int)chunk;
  a.chunks = (int)((tiles + chunk - 1) / chunk);
  a.sink_tiles = (a.sinks + kRows - 1) / kRows + (s.offsets ? 1 : 0);
}
int padded_dim(int dim) { return dim <= 64 ? 64 : 128; }
// Floats of workspace: delta, for fp16 the sums of sizes and the largest terms of
// keys, then the far sums, 16-byte aligned.
int64_t far_offset(const tcu_window_attention_args &s) {
  const int64_t rows = attn_batches(s) * s.rows;
  const int64_t n = rows * s.heads + (s.type == TCU_SEQ_F16 ? rows * ((int64_t)s.heads + s.kv_heads) : 0);
  return (n + 3) / 4 * 4;
}
int64_t far_blocks(const tcu_window_attention_args &s, const AttendArgs &a) {
  return attn_batches(s) * a.chunks * a.sink_tiles * s.kv_heads;
}

template <typename K>
bool shared_bytes(K kernel, int bytes) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) ==
      cudaSuccess)
    return true;
  cudaGetLastError();
  return false;
}

template <typename T, int DP>
int gradient(const tcu_window_attention_args &s, cudaStream_t st) {
  AttendArgs a = attend_args(s);
  const int64_t batches = attn_batches(s);
  a.q_tiles = a.k_tiles = (s.rows + kRows - 1) / kRows;
  float *delta = static_cast<float *>(s.workspace);
  const int64_t total = batches * s.rows * s.heads;
  a.delta = delta;
  a.sizes = delta + total;
  a.peaks = reinterpret_cast<uint32_t *>(a.sizes + total);
  const int64_t q_blocks = a.q_tiles * s.heads * batches, k_blocks = a.k_tiles * s.kv_heads * batches;
  if (q_blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  QueryMaps qm;
  KeyMaps km;
  const auto map = [&](CUtensorMap *m, const tcu_seq_rows &r, int heads, int box) {
    return attn_map(m, r, s.type, batches, s.rows, heads, s.dim, box);
  };
  if (!map(&qm.q, s.q, s.heads, kRows) || !map(&qm.dy, s.dy, s.heads, kRows) ||
      !map(&qm.k, s.k, s.kv_heads, kStep) || !map(&qm.v, s.v, s.kv_heads, kStep) ||
      !map(&km.q, s.q, s.heads, kStep) || !map(&km.dy, s.dy, s.heads, kStep) ||
      !map(&km.k, s.k, s.kv_heads, kRows) || !map(&km.v, s.v, s.kv_heads, kRows))
    return TCU_DFT_ERR_CUDA;
  split_rows(s, a);
  const int64_t far = far_blocks(s, a);
  if (far + k_blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  float *sums = delta + far_offset(s);
  constexpr int q_bytes = sizeof(QueryShared<DP>), k_bytes = sizeof(KeyShared<DP>);
  if (!shared_bytes(dq_kernel<T, DP>, q_bytes) || !shared_bytes(dkv_kernel<T, DP>, k_bytes))
    return TCU_DFT_ERR_CUDA;
  const unsigned blocks = (unsigned)std::min<int64_t>((total + 15) / 16, 16 * (int64_t)num_sms());
  delta_kernel<T><<<blocks, 256, 0, st>>>(rows_of<const T>(s.y), rows_of<const T>(s.dy), delta, a,
                                          total, batches * s.rows * s.kv_heads);
  if (const int rc = launched()) return rc;
  const Rows<T> dk = rows_of<T>(s.dk), dv = rows_of<T>(s.dv);
  dq_kernel<T, DP><<<(unsigned)q_blocks, kSoft + 64, q_bytes, st>>>(qm, a, rows_of<T>(s.dq), delta);
  if (const int rc = launched()) return rc;
  dkv_kernel<T, DP><<<(unsigned)(far + k_blocks), 2 * kSoft + 128, k_bytes, st>>>(km, a, dk, dv, sums,
                                                                             (int)far);
  if (const int rc = launched()) return rc;
  if (far == 0) return TCU_DFT_OK;
  join_kernel<T, DP><<<dim3((unsigned)k_blocks, kJoin), kRows, 0, st>>>(a, dk, dv, sums, (int)far);
  return launched();
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_window_attention_grad_workspace(const tcu_window_attention_args *a) {
  if (check_attention(a)) return -1;
  AttendArgs g = attend_args(*a);
  split_rows(*a, g);
  return 4 * (far_offset(*a) + far_blocks(*a, g) * 4 * kRows * padded_dim(a->dim));
}

extern "C" int tcu_window_attention_grad(const tcu_window_attention_args *a, void *stream) {
  if (const int rc = check_attention(a)) return rc;
  const int64_t batches = attn_batches(*a);
  if (a->rows == 0 || batches == 0) return TCU_DFT_OK;
  const int64_t qs = (int64_t)a->heads * a->dim, ks = (int64_t)a->kv_heads * a->dim;
  for (const tcu_seq_rows *r : {&a->q, &a->y, &a->dy, &a->dq})
    if (!attn_rows_ok(*r, batches, a->rows, qs)) return TCU_DFT_ERR_INVALID;
  for (const tcu_seq_rows *r : {&a->k, &a->v, &a->dk, &a->dv})
    if (!attn_rows_ok(*r, batches, a->rows, ks)) return TCU_DFT_ERR_INVALID;
  if (!a->lse || a->workspace_bytes < tcu_window_attention_grad_workspace(a) || !f32_ok(a->workspace) ||
      (uintptr_t)a->workspace % 16)
    return TCU_DFT_ERR_INVALID;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->type == TCU_SEQ_BF16)
    return a->dim <= 64 ? gradient<bf16, 64>(*a, st) : gradient<bf16, 128>(*a, st);
  return a->dim <= 64 ? gradient<f16, 64>(*a, st) : gradient<f16, 128>(*a, st);
}
