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
// up in memory.  Both hold the transposed role of the pass before: what a
// thread owns is a row of the accumulator's 128, p and ds go back to tensor
// memory in the rows' type, and the tiles of keys (queries) are read along
// their rows by the second products.
#include <algorithm>

#include "attn_common.cuh"

namespace tcu {
namespace seq {
namespace {

constexpr int kRows = 128;  // of the block
constexpr int kStep = 64;   // of a tile that it walks over
constexpr int kSoft = 128;

// ------------------------------------------------------------------- delta
// delta = dy.y of each row and head, 16 lanes a head; for fp16 the largest
// |dy| of rows in a sequence too (atomics: the order of a maximum has no say).
template <typename T>
__global__ void __launch_bounds__(256) delta_kernel(const Rows<const T> y, const Rows<const T> dy,
                                                    float *delta, int *most, const AttendArgs a,
                                                    int64_t total) {
  constexpr bool kMost = __is_same(T, f16);
  const int64_t step = (int64_t)gridDim.x * 16;
  const int lane = threadIdx.x % 16;
  float top = 0.f;
  for (int64_t pair = (int64_t)blockIdx.x * 16 + threadIdx.x / 32 * 2; pair < total; pair += step) {
    const int64_t id = pair + threadIdx.x / 16 % 2;
    float sum = 0.f;
    if (id < total && lane * 8 < a.dim) {
      const int64_t row = id / a.heads, b = row / a.rows, t = row - b * a.rows;
      const int64_t at = (id - row * a.heads) * a.dim + lane * 8;
      const Vec<T, 8> u = *reinterpret_cast<const Vec<T, 8> *>(y.at(b, (int)t) + at);
      const Vec<T, 8> v = *reinterpret_cast<const Vec<T, 8> *>(dy.at(b, (int)t) + at);
      int begin, end;
      const bool in = kMost && sequence_at(a, t, begin, end);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(to_f(u.v[i]), to_f(v.v[i]), sum);
        const float size = fabsf(to_f(v.v[i]));
        if (in && size < INFINITY) top = fmaxf(top, size);
      }
    }
#pragma unroll
    for (int m = 1; m < 16; m *= 2) sum += __shfl_xor_sync(~0u, sum, m);
    if (lane == 0 && id < total) delta[id] = sum;
  }
  if constexpr (kMost) {
    __shared__ int block;
    if (threadIdx.x == 0) block = 0;
    __syncthreads();
    const int bits = __reduce_max_sync(~0u, __float_as_int(top));
    if (threadIdx.x % 32 == 0) atomicMax(&block, bits);
    __syncthreads();
    if (threadIdx.x == 0 && block > 0) atomicMax(most, block);
  }
}

// A power of two that brings the largest |dy| to [1/2, 1): ds, rounded to fp16,
// then loses nothing to its range at the small gradients of long rows (bf16
// has fp32's range).
__device__ __forceinline__ float lift_of(const int *most) {
  const int e = most ? *most >> 23 : 0;
  return e > 0 ? __int_as_float((253 - e) << 23) : 1.f;
}

// ---------------------------------------------------------------------- dq
struct QueryMaps {
  CUtensorMap q, dy, k, v;  // k and v in boxes of kStep rows
};

template <int DP>
struct QueryShared {
  uint8_t q[kTileBytes<DP, kRows>], dy[kTileBytes<DP, kRows>];
  uint8_t k[2][kTileBytes<DP, kStep>], v[kTileBytes<DP, kStep>];
  uint64_t full_k[2], full_v, scores, weights, done;
  uint32_t tmem;
  int low, sink_at, sink_end, failed;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kSoft + 32, 2)
    dq_kernel(const __grid_constant__ QueryMaps maps, const AttendArgs a, const Rows<T> dq,
              const int *most) {
  extern __shared__ __align__(1024) uint8_t raw[];
  QueryShared<DP> &s = *reinterpret_cast<QueryShared<DP> *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t id = blockIdx.x;
  const int tile = (int)(id % a.q_tiles);
  const int head = (int)(id / a.q_tiles % a.heads), batch = (int)(id / a.q_tiles / a.heads);
  const int kv = head / (a.heads / a.kv_heads);
  const uint32_t full_k = smem_u32(s.full_k), full_v = smem_u32(&s.full_v),
                 scores = smem_u32(&s.scores), weights = smem_u32(&s.weights),
                 done = smem_u32(&s.done);
  if (threadIdx.x == 0) {
    mbar_init(full_k, 1);
    mbar_init(full_k + 8, 1);
    mbar_init(full_v, 1);
    mbar_init(scores, 1);
    mbar_init(weights, kSoft);
    mbar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.low = INT32_MAX;
    s.sink_end = 0;
    s.failed = 0;
  }
  if (warp == kSoft / 32) tmem_alloc(smem_u32(&s.tmem), 256);
  Seen seen{-1, INT32_MAX, 0, 0};
  if (threadIdx.x < kSoft) seen = seen_by(a, (int64_t)tile * kRows + threadIdx.x);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  if (threadIdx.x < kSoft) {
    const int low = __reduce_min_sync(~0u, seen.lo);
    if (lane == 0) atomicMin(&s.low, low);
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
  const float c = a.scale * kLog2e;

  if (warp == kSoft / 32) {
    const uint32_t q = smem_u32(s.q), dy = smem_u32(s.dy), k = smem_u32(s.k), v = smem_u32(s.v);
    constexpr uint32_t bytes = kTileBytes<DP, kStep>;
    bool ok = true;
    int keys = min(2, tiles), values = 1;  // tiles asked for
    if (tiles > 0 && elect_one()) {
      mbar_expect_tx(full_k, 2 * kTileBytes<DP, kRows> + bytes);
      load_tile<DP, kRows>(q, &maps.q, head, tile * kRows, batch, full_k);
      load_tile<DP, kStep>(k, &maps.k, kv, key_row(0), batch, full_k);
      load_tile<DP, kRows>(dy, &maps.dy, head, tile * kRows, batch, full_k);
      mbar_expect_tx(full_v, bytes);
      load_tile<DP, kStep>(v, &maps.v, kv, key_row(0), batch, full_v);
      if (tiles > 1) {
        mbar_expect_tx(full_k + 8, bytes);
        load_tile<DP, kStep>(k + bytes, &maps.k, kv, key_row(1), batch, full_k + 8);
      }
    }
    __syncwarp();
    for (int t = 0; t < tiles; ++t) {
      const uint32_t ph = t & 1, stage = t & 1, other = stage ^ 1;
      ok = mbar_wait_bounded(full_k + 8 * stage, (t >> 1) & 1) && mbar_wait_bounded(full_v, ph);
      // scores take the place of what the last product has read
      if (t > 0) ok = ok && mbar_wait_bounded(done, ph ^ 1);
      if (!ok) break;
      fence_after_sync();
      if (elect_one()) {
        if (t > 0 && t + 1 < tiles) {
          mbar_expect_tx(full_k + 8 * other, bytes);
          load_tile<DP, kStep>(k + other * bytes, &maps.k, kv, key_row(t + 1), batch,
                               full_k + 8 * other);
        }
        product_rows<T, DP, kStep>(tS, q, k + stage * bytes);
        product_rows<T, DP, kStep>(tP, dy, v);
        mma_commit(scores);
      }
      __syncwarp();
      if (t > 0 && t + 1 < tiles) keys = t + 2;
      ok = mbar_wait_bounded(scores, ph);
      if (ok && t + 1 < tiles) {
        if (elect_one()) {
          mbar_expect_tx(full_v, bytes);
          load_tile<DP, kStep>(v, &maps.v, kv, key_row(t + 1), batch, full_v);
        }
        __syncwarp();
        values = t + 2;
      }
      ok = ok && mbar_wait_bounded(weights, ph);
      if (!ok) break;
      fence_after_sync();
      if (elect_one()) {
        product_values<T, DP, kStep>(tQ, tS, k + stage * bytes, t > 0);
        mma_commit(done);
      }
      __syncwarp();
    }
    if (!ok) {  // copies in flight end before the block does
      s.failed = 1;
      mbar_wait_bounded(full_v, (values - 1) & 1);
      mbar_wait_bounded(full_k + 8 * ((keys - 1) & 1), ((keys - 1) >> 1) & 1);
      if (keys > 1) mbar_wait_bounded(full_k + 8 * (keys & 1), ((keys - 2) >> 1) & 1);
    }
  } else {
    const uint32_t mine = (uint32_t)(warp * 32) << 16;
    const int begin = a.offsets ? a.offsets[0] : 0;
    const int end = a.offsets ? a.offsets[a.sequences] : INT32_MAX;
    const float lift = lift_of(most);
    float lse = 0.f, delta = 0.f;
    if (seen.i >= 0) {
      const int64_t at = ((int64_t)batch * a.rows + seen.i) * a.heads + head;
      lse = a.lse[at] * kLog2e;
      delta = a.delta[at] * lift;
    }
    bool ok = true;
    for (int t = 0; t < tiles; ++t) {
      const uint32_t ph = t & 1;
      const int j0 = key_row(t);
      ok = mbar_wait_bounded(scores, ph);
      if (!ok) break;
      fence_after_sync();
      const bool whole = __all_sync(~0u, seen.whole(j0, j0 + kStep));
#pragma unroll
      for (int k = 0; k < kStep; k += 32) {
        float v[64];
        uint32_t w[16];
        tmem_ld32x2(tS + mine + k, tP + mine + k, v);
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          float x = exp2_fast(fmaf(v[j], c, -lse)) * fmaf(v[32 + j], lift, -delta);
          float y = exp2_fast(fmaf(v[j + 1], c, -lse)) * fmaf(v[33 + j], lift, -delta);
          if (!whole) {
            x = seen.at(j0 + k + j) ? x : 0.f;
            y = seen.at(j0 + k + j + 1) ? y : 0.f;
          }
          w[j / 2] = pack2<T>(x, y);
        }
        tmem_st16u(tS + mine + k / 2, w);
      }
      if (j0 + kStep > end || j0 < begin) {
        int b, e;
        if (threadIdx.x < kStep && !sequence_at(a, (int64_t)j0 + threadIdx.x, b, e))
          clear_row<DP, kStep>(smem_u32(s.k[t & 1]), threadIdx.x);
        fence_proxy_async_shared();
      }
      tmem_wait_st();
      fence_before_sync();
      mbar_arrive(weights);
    }
    if (tiles > 0) ok = ok && mbar_wait_bounded(done, (tiles - 1) & 1);
    fence_after_sync();
    const int64_t i = (int64_t)tile * kRows + threadIdx.x;
    const bool row = i < a.rows;
    const float by = !ok || s.failed ? __int_as_float(0x7fffffff) : a.scale / lift;
    T *to = dq.at(batch, row ? (int)i : 0) + (int64_t)head * a.dim;
#pragma unroll 1
    for (int k = 0; k < DP; k += 32) {
      float o[32];
      if (tiles > 0) {
        tmem_ld32(tQ + mine + k, o);
      }
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
  // of the query rows of a tile: [half][turn]
  float lse[2][2][kStep], delta[2][2][kStep];
  int low[2][2][kStep], begin[2][2][kStep], sink_end[2][2][kStep];
  uint64_t full_kv, full[kStages], scores[2], weights[2], done[2];
  uint32_t tmem;
  int last, failed;
};

// Two halves of 128 threads take the tiles of queries in turn: while one half
// forms weights, the tensor cores work on the other's tile.
template <typename T, int DP>
__global__ void __launch_bounds__(2 * kSoft + 32, 1)
    dkv_kernel(const __grid_constant__ KeyMaps maps, const AttendArgs a, const Rows<T> dk,
               const Rows<T> dv, const int *most) {
  extern __shared__ __align__(1024) uint8_t raw[];
  KeyShared<DP> &s = *reinterpret_cast<KeyShared<DP> *>(raw);
  const int warp = threadIdx.x / 32;
  const int64_t id = blockIdx.x;
  const int tile = (int)(id % a.k_tiles);
  const int kv = (int)(id / a.k_tiles % a.kv_heads), batch = (int)(id / a.k_tiles / a.kv_heads);
  const int group = a.heads / a.kv_heads;
  const uint32_t full_kv = smem_u32(&s.full_kv), full = smem_u32(s.full),
                 scores = smem_u32(s.scores), weights = smem_u32(s.weights), done = smem_u32(s.done);
  if (threadIdx.x == 0) {
    mbar_init(full_kv, 1);
    for (int i = 0; i < kStages; ++i) mbar_init(full + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(scores + 8 * i, 1);
      mbar_init(weights + 8 * i, kSoft);
      mbar_init(done + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.last = 0;
    s.failed = 0;
  }
  if (warp == 2 * kSoft / 32) tmem_alloc(smem_u32(&s.tmem), 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const int64_t j64 = (int64_t)tile * kRows + threadIdx.x % kSoft;
  if (threadIdx.x < kSoft) {  // the end of the rows that see this key
    int begin, end, past = 0;
    if (sequence_at(a, j64, begin, end)) {
      const int j = (int)j64;
      past = j - begin < a.sinks || end - j <= a.window ? end : j + a.window;
    }
    past = __reduce_max_sync(~0u, past);
    if (threadIdx.x % 32 == 0) atomicMax(&s.last, past);
  }
  __syncthreads();
  const uint32_t tmem = s.tmem, tV = tmem + 256, tK = tV + DP;
  const int first = tile * (kRows / kStep);
  const int q_tiles = max(0, (s.last + kStep - 1) / kStep - first);
  const int64_t n = (int64_t)q_tiles * group;
  const float c = a.scale * kLog2e;
  const auto head_of = [&](int64_t t) { return kv * group + (int)(t / q_tiles); };
  const auto row_of = [&](int64_t t) { return (first + (int)(t % q_tiles)) * kStep; };

  if (warp == 2 * kSoft / 32) {
    const uint32_t k = smem_u32(s.k), v = smem_u32(s.v), q = smem_u32(s.q), dy = smem_u32(s.dy);
    constexpr uint32_t bytes = kTileBytes<DP, kStep>;
    bool ok = true;
    int64_t asked = 0;
    const auto ask = [&](int64_t t) {
      const uint32_t stage = (uint32_t)t % kStages;
      if (elect_one()) {
        mbar_expect_tx(full + 8 * stage, 2 * bytes);
        load_tile<DP, kStep>(q + stage * bytes, &maps.q, head_of(t), row_of(t), batch,
                             full + 8 * stage);
        load_tile<DP, kStep>(dy + stage * bytes, &maps.dy, head_of(t), row_of(t), batch,
                             full + 8 * stage);
      }
      __syncwarp();
      asked = t + 1;
    };
    if (n > 0) {
      if (elect_one()) {
        mbar_expect_tx(full_kv, 2 * kTileBytes<DP, kRows>);
        load_tile<DP, kRows>(k, &maps.k, kv, tile * kRows, batch, full_kv);
        load_tile<DP, kRows>(v, &maps.v, kv, tile * kRows, batch, full_kv);
      }
      __syncwarp();
      ask(0);
      if (n > 1) ask(1);
      ok = mbar_wait_bounded(full_kv, 0);
    }
    for (int64_t t = 0; n > 0 && t <= n && ok; ++t) {
      if (t < n) {
        const uint32_t half = t & 1, stage = (uint32_t)t % kStages;
        // the half's tensor memory and the tiles of t - 2 have been read
        if (t >= 2) ok = mbar_wait_bounded(done + 8 * half, ((t - 2) >> 1) & 1);
        if (ok && t + 2 < n) ask(t + 2);
        ok = ok && mbar_wait_bounded(full + 8 * stage, (uint32_t)(t / kStages) & 1);
        if (!ok) break;
        fence_after_sync();
        if (elect_one()) {
          product_rows<T, DP, kStep>(tmem + 128 * half, k, q + stage * bytes);
          product_rows<T, DP, kStep>(tmem + 128 * half + kStep, v, dy + stage * bytes);
          mma_commit(scores + 8 * half);
        }
        __syncwarp();
      }
      if (t > 0) {
        const int64_t u = t - 1;
        const uint32_t half = u & 1, stage = (uint32_t)u % kStages;
        ok = mbar_wait_bounded(weights + 8 * half, (uint32_t)(u >> 1) & 1);
        if (!ok) break;
        fence_after_sync();
        if (elect_one()) {
          product_values<T, DP, kStep>(tV, tmem + 128 * half, dy + stage * bytes, u > 0);
          product_values<T, DP, kStep>(tK, tmem + 128 * half + kStep, q + stage * bytes, u > 0);
          mma_commit(done + 8 * half);
        }
        __syncwarp();
      }
    }
    if (!ok) {  // copies in flight end before the block does
      s.failed = 1;
      mbar_wait_bounded(full_kv, 0);
      for (int64_t u = max((int64_t)0, asked - kStages); u < asked; ++u)
        mbar_wait_bounded(full + 8 * ((uint32_t)u % kStages), (uint32_t)(u / kStages) & 1);
    }
  } else {
    const int half = threadIdx.x / kSoft, own = threadIdx.x % kSoft;
    const uint32_t mine = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t tS = tmem + 128 * half + mine, tP = tS + kStep;
    const int begin = a.offsets ? a.offsets[0] : 0;
    const int end = a.offsets ? a.offsets[a.sequences] : INT32_MAX;
    const int j = (int)min(j64, (int64_t)INT32_MAX);
    const float lift = lift_of(most);
    // what the next tile's query rows bring, a row a thread
    float lse = 0.f, delta = 0.f;
    Seen seen{-1, INT32_MAX, 0, 0};
    const auto fetch = [&](int64_t t) {
      if (own >= kStep || t >= n) return;
      seen = seen_by(a, (int64_t)row_of(t) + own);
      lse = delta = 0.f;
      if (seen.i >= 0) {
        const int64_t at = ((int64_t)batch * a.rows + seen.i) * a.heads + head_of(t);
        lse = a.lse[at] * kLog2e;
        delta = a.delta[at] * lift;
      }
    };
    fetch(half);
    bool ok = true;
    for (int64_t t = half; t < n; t += 2) {
      const int turn = (t >> 1) & 1;
      if (own < kStep) {
        s.lse[half][turn][own] = lse;
        s.delta[half][turn][own] = delta;
        s.low[half][turn][own] = seen.lo;
        s.begin[half][turn][own] = seen.s0;
        s.sink_end[half][turn][own] = seen.s1;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + half), "n"(kSoft) : "memory");
      fetch(t + 2);
      const int i0 = row_of(t);
      ok = mbar_wait_bounded(scores + 8 * half, (uint32_t)(t >> 1) & 1);
      if (!ok) break;
      fence_after_sync();
      // rows see more from below as they come: the last one's bound is the highest
      const bool whole = __all_sync(~0u, j <= i0 && j >= s.low[half][turn][kStep - 1]);
#pragma unroll
      for (int k = 0; k < kStep; k += 32) {
        float v[64];
        uint32_t w[16], d[16];
        tmem_ld32x2(tS + k, tP + k, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const int r = k + i;
          float p = exp2_fast(fmaf(v[i], c, -s.lse[half][turn][r]));
          float x = p * fmaf(v[32 + i], lift, -s.delta[half][turn][r]);
          if (!whole) {
            const bool at = (j >= s.low[half][turn][r] && j <= i0 + r) ||
                            (j >= s.begin[half][turn][r] && j < s.sink_end[half][turn][r]);
            p = at ? p : 0.f;
            x = at ? x : 0.f;
          }
          v[i] = p;
          v[32 + i] = x;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          w[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
          d[i] = pack2<T>(v[32 + 2 * i], v[33 + 2 * i]);
        }
        tmem_st16u(tS + k / 2, w);
        tmem_st16u(tP + k / 2, d);
      }
      if (i0 + kStep > end || i0 < begin) {
        int b, e;
        if (own < kStep && !sequence_at(a, (int64_t)i0 + own, b, e)) {
          clear_row<DP, kStep>(smem_u32(s.q[t % kStages]), own);
          clear_row<DP, kStep>(smem_u32(s.dy[t % kStages]), own);
        }
        fence_proxy_async_shared();
      }
      tmem_wait_st();
      fence_before_sync();
      mbar_arrive(weights + 8 * half);
    }
    // all products: the last tile's after the one's before, as a barrier may be
    // waited for only one phase ahead
    if (n > 1) ok = ok && mbar_wait_bounded(done + 8 * (n & 1), (uint32_t)((n - 2) >> 1) & 1);
    if (n > 0) ok = ok && mbar_wait_bounded(done + 8 * ((n - 1) & 1), (uint32_t)((n - 1) >> 1) & 1);
    fence_after_sync();
    const bool row = j64 < a.rows;
    const float by = !ok || s.failed ? __int_as_float(0x7fffffff) : half ? a.scale / lift : 1.f;
    T *to = (half ? dk : dv).at(batch, row ? j : 0) + (int64_t)kv * a.dim;
    int b, e;
    const bool in = sequence_at(a, j64, b, e);
#pragma unroll 1
    for (int k = 0; k < DP; k += 32) {
      float o[32];
      if (n > 0) tmem_ld32((half ? tK : tV) + mine + k, o);
      if (n == 0 || !in) {  // rows of no sequence
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = 0.f;
      }
      if (row) store_values(to, k, a.dim, o, by);
    }
    fence_before_sync();
  }
  __syncthreads();
  if (warp == 2 * kSoft / 32) tmem_dealloc(tmem, 512);
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
  a.delta = delta;
  int *most = __is_same(T, f16) ? reinterpret_cast<int *>(delta + batches * s.rows * s.heads) : nullptr;
  const int64_t total = batches * s.rows * s.heads;
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
  if (!shared_bytes(dq_kernel<T, DP>, sizeof(QueryShared<DP>)) ||
      !shared_bytes(dkv_kernel<T, DP>, sizeof(KeyShared<DP>)))
    return TCU_DFT_ERR_CUDA;
  const unsigned blocks = (unsigned)std::min<int64_t>((total + 15) / 16, 16 * (int64_t)num_sms());
  if (most && cudaMemsetAsync(most, 0, sizeof(int), st) != cudaSuccess) {
    cudaGetLastError();
    return TCU_DFT_ERR_CUDA;
  }
  delta_kernel<T><<<blocks, 256, 0, st>>>(rows_of<const T>(s.y), rows_of<const T>(s.dy), delta, most,
                                          a, total);
  if (const int rc = launched()) return rc;
  dkv_kernel<T, DP><<<(unsigned)k_blocks, 2 * kSoft + 32, sizeof(KeyShared<DP>), st>>>(
      km, a, rows_of<T>(s.dk), rows_of<T>(s.dv), most);
  if (const int rc = launched()) return rc;
  dq_kernel<T, DP><<<(unsigned)q_blocks, kSoft + 32, sizeof(QueryShared<DP>), st>>>(
      qm, a, rows_of<T>(s.dq), most);
  return launched();
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_window_attention_grad_workspace(const tcu_window_attention_args *a) {
  if (check_attention(a)) return -1;
  return (attn_batches(*a) * a->rows * a->heads + 1) * 4;
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
  if (!a->lse || a->workspace_bytes < tcu_window_attention_grad_workspace(a) || !f32_ok(a->workspace))
    return TCU_DFT_ERR_INVALID;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->type == TCU_SEQ_BF16)
    return a->dim <= 64 ? gradient<bf16, 64>(*a, st) : gradient<bf16, 128>(*a, st);
  return a->dim <= 64 ? gradient<f16, 64>(*a, st) : gradient<f16, 128>(*a, st);
}
