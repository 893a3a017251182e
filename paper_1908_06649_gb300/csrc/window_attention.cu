// window_attention.cu -- attention over a sliding window and a sequence's first
// tokens, for prompts (include/tcu_attn.h); entry points and the filling of
// caches.
//
// A block owns 128 query rows of one head and walks over the tiles of 64 keys
// that any of them sees, first tokens' tiles first, with one pass over the
// data: S = Q K^T and O += P V on the tensor cores (tcgen05, accumulators in
// tensor memory), P = exp2(c S - m) between them, a row a thread, m a running
// maximum.  O is brought to a new maximum only where that rose by more than 8
// (P stays below 2^8, sums below 2^39: fp32 holds them); P goes back to tensor
// memory over S, in the rows' type.
//
// Products bound it: 4 dim flops a visible pair and head.  Weights wait for
// scores and products for weights, so scores run a tile ahead, in two places,
// and two blocks share an SM (256 columns of tensor memory, 96 KB of tiles
// each).  A warp each issues products, copies, and looks over values that not
// all rows see.
//
// Measured, bf16: 32768 rows, 32 heads (8 of keys) x 128, window 2048, 4 first
// tokens (1.07e12 flops): 886 us, 1.21 PFLOP/s, 64 % of cuBLAS's burst rate.  Before
// values were looked over it was 808, with copies issued between the products 904,
// with 128 keys a tile, one place for scores and two threads a row 1,007.
#include <algorithm>

#include "attn_common.cuh"

namespace tcu {
namespace seq {
namespace {

constexpr int kRows = 128;  // of a tile of queries
constexpr int kStep = 64;   // of a tile of keys
constexpr int kSoft = 128;  // threads that form weights: a row each
constexpr int kThreads = kSoft + 96;  // and a warp each for products, copies, a look at values

struct PromptMaps {
  CUtensorMap q, k, v;  // k and v in boxes of kStep rows
};

template <int DP>
struct PromptShared {
  uint8_t q[kTileBytes<DP, kRows>];
  uint8_t k[2][kTileBytes<DP, kStep>], v[2][kTileBytes<DP, kStep>];
  uint64_t full_k[2], landed[2], full_v[2], scores[2], weights[2], done[2];
  unsigned long long bad[2];  // rows of values that are not finite, of a tile
  uint32_t tmem;
  int low, high, sink_at, sink_end, failed;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 2)
    attend_kernel(const __grid_constant__ PromptMaps maps, const AttendArgs a, const Rows<T> y) {
  extern __shared__ __align__(1024) uint8_t raw[];
  PromptShared<DP> &s = *reinterpret_cast<PromptShared<DP> *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t id = blockIdx.x;
  const int tile = (int)(id % a.q_tiles);
  const int head = (int)(id / a.q_tiles % a.heads), batch = (int)(id / a.q_tiles / a.heads);
  const int kv = head / (a.heads / a.kv_heads);
  const uint32_t full_k = smem_u32(s.full_k), full_v = smem_u32(s.full_v),
                 scores = smem_u32(s.scores), weights = smem_u32(s.weights),
                 done = smem_u32(s.done), landed = smem_u32(s.landed);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(done + 8 * i, 1);
      mbar_init(full_k + 8 * i, 1);
      mbar_init(landed + 8 * i, 1);
      mbar_init(full_v + 8 * i, 32);
      mbar_init(scores + 8 * i, 1);
      mbar_init(weights + 8 * i, kSoft);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.low = INT32_MAX;
    s.high = 0;
    s.sink_end = 0;
    s.failed = 0;
  }
  if (warp == kSoft / 32) tmem_alloc(smem_u32(&s.tmem), 256);
  Seen seen{-1, INT32_MAX, 0, 0};
  if (threadIdx.x < kSoft) seen = seen_by(a, (int64_t)tile * kRows + threadIdx.x);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  // the key tiles: those of the window, and before them those of first tokens
  if (threadIdx.x < kSoft) {
    const int low = __reduce_min_sync(~0u, seen.lo);
    const int high = __reduce_max_sync(~0u, seen.i >= 0 ? seen.lo : 0);
    if (lane == 0) {
      atomicMin(&s.low, low);
      atomicMax(&s.high, high);
    }
  }
  __syncthreads();
  const int first = s.low / kStep;  // s.low == INT32_MAX: no row is in a sequence
  // only the sequence that the tile's first row continues begins before them
  if (threadIdx.x < kSoft && seen.s0 < seen.s1 && seen.s0 < (int64_t)first * kStep) {
    atomicMax(&s.sink_end, min(seen.s1, first * kStep));
    s.sink_at = seen.s0 / kStep;
  }
  __syncthreads();
  const uint32_t tmem = s.tmem, tO = tmem + 2 * kStep;
  const bool any = s.low != INT32_MAX;
  const int sink_tiles = s.sink_end > 0 ? (s.sink_end - 1) / kStep - s.sink_at + 1 : 0;
  const int sink_first = sink_tiles ? s.sink_at : 0;
  const int last = (int)min((int64_t)tile * 2 + 1, (a.rows - 1) / kStep);
  const int tiles = any ? sink_tiles + last - first + 1 : 0;
  const auto key_row = [&](int t) {
    return (t < sink_tiles ? sink_first + t : first + t - sink_tiles) * kStep;
  };
  // whether not all rows see all keys of a tile
  const auto edge = [&](int j0) { return j0 < s.high || j0 + kStep - 1 > tile * kRows; };
  const float c = a.scale * kLog2e;

  const uint32_t q = smem_u32(s.q), k = smem_u32(s.k), v = smem_u32(s.v);
  constexpr uint32_t bytes = kTileBytes<DP, kStep>;
  if (warp == kSoft / 32 + 1) {  // copies: two tiles ahead
    bool ok = true;
    int keys = 0, values = 0;  // tiles asked for
    for (int t = 0; t < tiles && ok; ++t) {
      const uint32_t stage = t & 1;
      // the scores of t - 2 have read its keys, the product of t - 2 its values
      if (t > 1) ok = warp_waits(scores + 8 * stage, ((t - 2) >> 1) & 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(full_k + 8 * stage, bytes + (t == 0 ? kTileBytes<DP, kRows> : 0));
        if (t == 0) load_tile<DP, kRows>(q, &maps.q, head, tile * kRows, batch, full_k);
        load_tile<DP, kStep>(k + stage * bytes, &maps.k, kv, key_row(t), batch, full_k + 8 * stage);
      }
      __syncwarp();
      keys = t + 1;
      if (t > 1) ok = warp_waits(done + 8 * stage, ((t - 2) >> 1) & 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(landed + 8 * stage, bytes);
        load_tile<DP, kStep>(v + stage * bytes, &maps.v, kv, key_row(t), batch, landed + 8 * stage);
      }
      __syncwarp();
      values = t + 1;
    }
    if (!ok) {  // copies in flight end before the block does
      s.failed = 1;
      for (int i = 1; i <= 2; ++i) {
        if (keys >= i) warp_waits(full_k + 8 * ((keys - i) & 1), ((keys - i) >> 1) & 1);
        if (values >= i) warp_waits(landed + 8 * ((values - i) & 1), ((values - i) >> 1) & 1);
      }
    }
  } else if (warp == kSoft / 32 + 2) {  // a look at values that not all rows see
    const Filled filled(a);
    for (int t = 0; t < tiles; ++t) {
      const uint32_t stage = t & 1;
      if (!warp_waits(landed + 8 * stage, (t >> 1) & 1)) {
        s.failed = 1;
        break;
      }
      if (edge(key_row(t))) {
        // the marks of t - 2 have been read: its values have made room
        if (lane == 0) s.bad[stage] = 0;
        __syncwarp();
        clean_tile<T, DP, 32>(v + stage * bytes, lane, key_row(t), filled, &s.bad[stage]);
        fence_proxy_async_shared();
      }
      mbar_arrive(full_v + 8 * stage);
    }
  } else if (warp == kSoft / 32) {  // products
    bool ok = true;
    // scores run a tile ahead of the weights: while those of one are formed,
    // the next tile's are multiplied
    for (int t = -1; t < tiles && ok; ++t) {
      const uint32_t stage = t & 1, other = stage ^ 1;
      if (t + 1 < tiles) {
        ok = warp_waits(full_k + 8 * other, ((t + 1) >> 1) & 1);
        // they take the place of weights that the product of t - 1 has read
        if (t > 0) ok = ok && warp_waits(done + 8 * other, ((t - 1) >> 1) & 1);
        if (!ok) break;
        fence_after_sync();
        if (elect_one()) {
          product_rows<T, DP, kStep>(tmem + other * kStep, q, k + other * bytes);
          mma_commit(scores + 8 * other);
        }
        __syncwarp();
      }
      if (t < 0) continue;
      ok = warp_waits(full_v + 8 * stage, (t >> 1) & 1) &&
           warp_waits(weights + 8 * stage, (t >> 1) & 1);
      if (!ok) break;
      fence_after_sync();
      if (elect_one()) {
        product_values<T, DP, kStep>(tO, tmem + stage * kStep, v + stage * bytes, t > 0);
        mma_commit(done + 8 * stage);
      }
      __syncwarp();
    }
    if (!ok) s.failed = 1;
  } else {
    const uint32_t mine = (uint32_t)(warp * 32) << 16;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int t = 0; t < tiles && ok; ++t) {
      const int stage = t & 1, ph = (t >> 1) & 1, j0 = key_row(t);
      const uint32_t tS = tmem + mine + kStep * stage;
      ok = warp_waits(scores + 8 * stage, ph);
      fence_after_sync();
      float v[64];
      tmem_ld32x2(tS, tS + 32, v);
      if (edge(j0)) {
        // rows of values in no sequence, and those that are not finite, are gone;
        // who sees one of the latter has no number for its result
        ok = ok && warp_waits(full_v + 8 * stage, ph);
        const unsigned long long bad = s.bad[stage];
        const uint32_t bits0 = seen.bits(j0), bits1 = seen.bits(j0 + 32);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          v[j] = bits0 >> j & 1 ? v[j] : -INFINITY;
          v[32 + j] = bits1 >> j & 1 ? v[32 + j] : -INFINITY;
        }
        if (bad) {
          const uint32_t bad0 = bits0 & (uint32_t)bad, bad1 = bits1 & (uint32_t)(bad >> 32);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            v[j] = bad0 >> j & 1 ? __int_as_float(0x7fffffff) : v[j];
            v[32 + j] = bad1 >> j & 1 ? __int_as_float(0x7fffffff) : v[32 + j];
          }
        }
      }
      float top = v[0], top1 = v[1], top2 = v[2], top3 = v[3];
#pragma unroll
      for (int j = 4; j < 64; j += 4) {
        top = fmaxf(top, v[j]);
        top1 = fmaxf(top1, v[j + 1]);
        top2 = fmaxf(top2, v[j + 2]);
        top3 = fmaxf(top3, v[j + 3]);
      }
      top = fmaxf(fmaxf(top, top1), fmaxf(top2, top3)) * c;
      const bool rise = top > m + 8.f || (m == -INFINITY && top > m);
      if (__any_sync(~0u, rise)) {
        const float now = rise ? top : m;
        const float by = m == -INFINITY ? 0.f : exp2_fast(m - now);
        l *= by;
        if (t > 0) {
          ok = ok && warp_waits(done + 8 * (stage ^ 1), ((t - 1) >> 1) & 1);
          fence_after_sync();
#pragma unroll 1
          for (int k = 0; k < DP; k += 16) {
            float o[16];
            tmem_ld16(tO + mine + k, o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= by;
            tmem_st16(tO + mine + k, o);
          }
        }
        m = now;
      }
      // a row that has seen nothing yet has no maximum
      const float2 off = splat(m == -INFINITY ? 0.f : -m), by = splat(c);
      float2 sum = splat(0.f);
      uint32_t w[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float2 z = __ffma2_rn(make_float2(v[2 * j], v[2 * j + 1]), by, off);
        const float2 p = make_float2(exp2_fast(z.x), exp2_fast(z.y));
        sum = __fadd2_rn(sum, p);
        w[j] = pack2<T>(p.x, p.y);
      }
      tmem_st16u(tS, w);
      tmem_st16u(tS + 32, w + 16);
      l += sum.x + sum.y;
      tmem_wait_st();
      fence_before_sync();
      mbar_arrive(weights + 8 * stage);
    }
    // products end in order
    if (tiles > 0) ok = ok && warp_waits(done + 8 * ((tiles - 1) & 1), ((tiles - 1) >> 1) & 1);
    fence_after_sync();
    const bool row = seen.i >= 0;
    const float by = !ok || s.failed ? __int_as_float(0x7fffffff) : l > 0.f ? 1.f / l : l;
    T *to = y.at(batch, row ? seen.i : 0) + (int64_t)head * a.dim;
    if (tiles > 0) {
#pragma unroll 1
      for (int k = 0; k < DP; k += 32) {
        float o[32];
        tmem_ld32(tO + mine + k, o);
        if (row) store_values(to, k, a.dim, o, by);
      }
    }
    if (row && a.lse)
      a.lse[((int64_t)batch * a.rows + seen.i) * a.heads + head] = (m + log2f(l)) * kLn2;
    fence_before_sync();
  }
  __syncthreads();
  if (warp == kSoft / 32) tmem_dealloc(tmem, 256);
}

template <typename T, int DP>
int prompt(const tcu_window_attention_args &s, cudaStream_t st) {
  AttendArgs a = attend_args(s);
  const int64_t batches = attn_batches(s);
  a.q_tiles = (s.rows + kRows - 1) / kRows;
  const int64_t blocks = a.q_tiles * s.heads * batches;
  if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  PromptMaps maps;
  if (!attn_map(&maps.q, s.q, s.type, batches, s.rows, s.heads, s.dim, kRows) ||
      !attn_map(&maps.k, s.k, s.type, batches, s.rows, s.kv_heads, s.dim, kStep) ||
      !attn_map(&maps.v, s.v, s.type, batches, s.rows, s.kv_heads, s.dim, kStep))
    return TCU_DFT_ERR_CUDA;
  constexpr int bytes = sizeof(PromptShared<DP>);
  if (cudaFuncSetAttribute(attend_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           bytes) != cudaSuccess) {
    cudaGetLastError();
    return TCU_DFT_ERR_CUDA;
  }
  attend_kernel<T, DP><<<(unsigned)blocks, kThreads, bytes, st>>>(maps, a, rows_of<T>(s.y));
  return launched();
}

// ------------------------------------------------------------------- caches
struct FillArgs {
  Rows<const uint4> k, v;  // rows in 16-byte words
  uint4 *cache_k, *cache_v;
  const int32_t *offsets, *slots;
  int64_t rows, num_slots;
  int sequences, words, window, sinks;
};

// A warp for each row of an entry: the last position of the sequence that
// belongs there.
__global__ void __launch_bounds__(128) fill_kernel(const FillArgs a) {
  const int64_t held = (int64_t)a.sinks + a.window;
  const int64_t r = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
  if (r >= held) return;
  for (int64_t s = blockIdx.y; s < a.sequences; s += gridDim.y) {
    int64_t begin = 0, n = a.rows;
    if (a.offsets) {
      begin = max(0, a.offsets[s]);
      n = min(a.rows, (int64_t)a.offsets[s + 1]) - begin;
    }
    const int64_t slot = a.slots ? a.slots[s] : s;
    int64_t p = r;
    if (r >= a.sinks && n > held) p = n - 1 - (n - 1 - r) % a.window;
    if (p >= n || slot < 0 || slot >= a.num_slots) continue;
    const int64_t b = a.offsets ? 0 : s;
    const uint4 *k = a.k.at(b, (int)(begin + p)), *v = a.v.at(b, (int)(begin + p));
    uint4 *to_k = a.cache_k + (slot * held + r) * a.words;
    uint4 *to_v = a.cache_v + (slot * held + r) * a.words;
    for (int i = threadIdx.x % 32; i < a.words; i += 32) to_k[i] = k[i], to_v[i] = v[i];
  }
}

Rows<const uint4> words_of(const tcu_seq_rows &r) {
  return {static_cast<const uint4 *>(r.ptr), r.batch_stride / 8, (int32_t)(r.row_stride / 8)};
}

}  // namespace

int check_attention(const tcu_window_attention_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->dim < 1 || a->window < 1 ||
      a->sinks < 0 || !(a->scale > 0) || a->scale > 1e30f)
    return TCU_DFT_ERR_INVALID;
  if (a->type == TCU_SEQ_F32 || a->dim > TCU_ATTN_MAX_DIM || a->dim % 8 || a->rows > kMostRows ||
      a->heads > (1 << 20))
    return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r : {&a->q, &a->k, &a->v, &a->y, &a->dy, &a->dq, &a->dk, &a->dv})
    if (!pitch_fits(a->rows, r->row_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  return opt_ok(a->offsets, 4) && opt_ok(a->lse, 4) && opt_ok(a->slots, 4) &&
                 opt_ok(a->positions, 4)
             ? TCU_DFT_OK
             : TCU_DFT_ERR_INVALID;
}

}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int tcu_window_attention(const tcu_window_attention_args *a, void *stream) {
  if (const int rc = check_attention(a)) return rc;
  const int64_t batches = attn_batches(*a);
  if (a->rows == 0 || batches == 0) return TCU_DFT_OK;
  const int64_t qs = (int64_t)a->heads * a->dim, ks = (int64_t)a->kv_heads * a->dim;
  if (!attn_rows_ok(a->q, batches, a->rows, qs) || !attn_rows_ok(a->k, batches, a->rows, ks) ||
      !attn_rows_ok(a->v, batches, a->rows, ks) || !attn_rows_ok(a->y, batches, a->rows, qs))
    return TCU_DFT_ERR_INVALID;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->type == TCU_SEQ_BF16)
    return a->dim <= 64 ? prompt<bf16, 64>(*a, st) : prompt<bf16, 128>(*a, st);
  return a->dim <= 64 ? prompt<f16, 64>(*a, st) : prompt<f16, 128>(*a, st);
}

extern "C" int tcu_window_cache(const tcu_window_attention_args *a, void *stream) {
  if (const int rc = check_attention(a)) return rc;
  if (a->num_slots < 0 || (!a->slots && a->num_slots < a->sequences)) return TCU_DFT_ERR_INVALID;
  if (a->rows == 0 || a->sequences == 0 || a->num_slots == 0) return TCU_DFT_OK;
  const int64_t batches = attn_batches(*a), ks = (int64_t)a->kv_heads * a->dim;
  if (!attn_rows_ok(a->k, batches, a->rows, ks) || !attn_rows_ok(a->v, batches, a->rows, ks) ||
      !a->cache_k || !a->cache_v || (uintptr_t)a->cache_k % 16 || (uintptr_t)a->cache_v % 16)
    return TCU_DFT_ERR_INVALID;
  const int64_t held = (int64_t)a->sinks + a->window;
  const wide_int bytes = (wide_int)a->num_slots * held * ks * 2;
  for (const void *c : {a->cache_k, a->cache_v}) {
    for (const tcu_seq_rows *r : {&a->k, &a->v})
      for (int64_t b = 0; b < batches; ++b)
        if (over(c, bytes, static_cast<const char *>(r->ptr) + b * r->batch_stride * 2, ks * 2,
                 a->rows, r->row_stride * 2))
          return TCU_DFT_ERR_INVALID;
    if (over(c, bytes, a->slots, (int64_t)a->sequences * 4) ||
        over(c, bytes, a->offsets, ((int64_t)a->sequences + 1) * 4))
      return TCU_DFT_ERR_INVALID;
  }
  if (over(a->cache_k, bytes, a->cache_v, 1) || over(a->cache_v, bytes, a->cache_k, 1))
    return TCU_DFT_ERR_INVALID;
  FillArgs f{};
  f.k = words_of(a->k);
  f.v = words_of(a->v);
  f.cache_k = static_cast<uint4 *>(a->cache_k);
  f.cache_v = static_cast<uint4 *>(a->cache_v);
  f.offsets = a->offsets;
  f.slots = a->slots;
  f.rows = a->rows;
  f.num_slots = a->num_slots;
  f.sequences = a->sequences;
  f.words = (int)(ks / 8);
  f.window = a->window;
  f.sinks = a->sinks;
  // rows of an entry that no sequence of this length reaches need no block
  const int64_t reach = std::min(held, a->rows);
  const dim3 grid((unsigned)((reach + 3) / 4), (unsigned)std::min(a->sequences, 65535));
  fill_kernel<<<grid, 128, 0, static_cast<cudaStream_t>(stream)>>>(f);
  return launched();
}
