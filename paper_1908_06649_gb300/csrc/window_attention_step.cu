// window_attention_step.cu -- window attention for single tokens from caches
// (include/tcu_attn.h).
//
// A token sees what its entry holds: min(position + 1, sinks + window) rows of
// keys and values, each read once for all query heads that share them, a few
// operations a byte: HBM bounds it, so what counts is that enough rows are on
// their way.  A warp walks over tiles of 16 rows, which it copies into a ring of
// its own in shared memory three tiles ahead, and takes them to a running
// maximum, sum and output (mma.sync, 16 heads by 16 keys: a tile of tcgen05
// would be 128 heads, of which a token has a few for each key head).  Warps of
// a block and blocks of a cluster share an entry's rows, and join their sums
// through shared memory in the order of warps and blocks.
//
// Measured, bf16: 64 tokens, 32 heads (8 of keys) x 128, 2052 rows an entry (538
// MB) 90 us, 6.0 TB/s, 88 % of the copy rate (weights in one part: 88); one token of
// 1028 rows 11 us, five round trips to memory that wait for each other (slot,
// position, q, the new row, which is taken and stored first, the cache) and the
// barriers of a cluster.
#include <cooperative_groups.h>

#include <algorithm>

#include "attn_common.cuh"

namespace tcu {
namespace seq {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 3;
constexpr int kTile = 16;   // rows
constexpr int kHeads = 16;  // of a block
constexpr int kMostCluster = 8;

template <typename T>
struct StepArgs {
  const T *q, *k, *v;
  T *y;
  int64_t q_step, k_step, v_step, y_step;  // between batch entries
  T *cache_k, *cache_v;
  const int32_t *slots, *positions;
  int64_t num_slots;
  int batch, heads, kv_heads, dim, window, sinks, head_groups;
  float c;  // scale log2(e)
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool has) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(has ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
template <bool kTrans>
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t *r) {
  if constexpr (kTrans)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  if constexpr (__is_same(T, f16))
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DP>
struct StepShared {
  // a warp's ring of tiles; after the walk its share of the output, [head][DP]
  uint8_t ring[kWarps][kStages][2][kTile * DP * 2];
  float top[kWarps][kHeads], sum[kWarps][kHeads];  // of a warp
  float block_top[kHeads], block_sum[kHeads];
};

// Chunk c (16 bytes) of row r of a tile: permuted so that eight rows' chunks
// of one column fall on all banks.
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  return (uint32_t)(r * DP * 2 + ((c ^ (r & 7)) << 4));
}

template <typename T, int DP>
struct Walk {
  uint32_t q[DP / 16][4];  // 16 heads x 16 values
  float o[DP / 8][4];
  float m[2], l[2];  // rows lane / 4 and lane / 4 + 8

  // One tile: rows [0, count) of it but `skip`.
  __device__ __forceinline__ void tile(uint32_t k, uint32_t v, int count, int skip, float c,
                                       int lane) {
    float s[2][4] = {};
    const int mat = lane / 8, r = lane % 8;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      uint32_t b[4];
      ldmatrix4<false>(k + chunk_at<DP>((mat >> 1) * 8 + r, 2 * i + (mat & 1)), b);
      mma16<T>(s[0], q[i], b[0], b[1]);
      mma16<T>(s[1], q[i], b[2], b[3]);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = n * 8 + 2 * (lane % 4) + (e & 1);
        s[n][e] = j < count && j != skip ? s[n][e] * c : -INFINITY;
      }
    float now[2], by[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float top = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
      now[h] = fmaxf(m[h], top);
      by[h] = m[h] == -INFINITY ? 0.f : exp2_fast(m[h] - now[h]);
    }
    if (__any_sync(~0u, now[0] != m[0] || now[1] != m[1])) {
#pragma unroll
      for (int i = 0; i < DP / 8; ++i)
        o[i][0] *= by[0], o[i][1] *= by[0], o[i][2] *= by[1], o[i][3] *= by[1];
    }
    // weights in two parts, what the first rounds off in the second: the products
    // they add are hidden behind the rows on their way
    uint32_t p[4], rest[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float off = now[h] == -INFINITY ? 0.f : now[h];
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = exp2_fast(s[i / 2][2 * h + i % 2] - off);
      l[h] = l[h] * (m[h] == now[h] ? 1.f : by[h]) + (e[0] + e[1]) + (e[2] + e[3]);
      m[h] = now[h];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w = pack2<T>(e[2 * i], e[2 * i + 1]);
        const float2 taken = Pair<T>::get(&w);
        p[2 * i + h] = w;
        rest[2 * i + h] = pack2<T>(e[2 * i] - taken.x, e[2 * i + 1] - taken.y);
      }
    }
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      uint32_t b[4];
      ldmatrix4<true>(v + chunk_at<DP>((mat & 1) * 8 + r, 2 * i + (mat >> 1)), b);
      mma16<T>(o[2 * i], p, b[0], b[1]);
      mma16<T>(o[2 * i + 1], p, b[2], b[3]);
      mma16<T>(o[2 * i], rest, b[0], b[1]);
      mma16<T>(o[2 * i + 1], rest, b[2], b[3]);
    }
  }
};

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 2) attend_step_kernel(const StepArgs<T> a, int size) {
  extern __shared__ __align__(16) uint8_t raw[];
  StepShared<DP> &s = *reinterpret_cast<StepShared<DP> *>(raw);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int rank = (int)(blockIdx.x % size);
  int64_t id = blockIdx.x / size;
  const int group = (int)(id % a.head_groups);
  id /= a.head_groups;
  const int kv = (int)(id % a.kv_heads), b = (int)(id / a.kv_heads);
  const int shared_by = a.heads / a.kv_heads;
  const int first = kv * shared_by + group * kHeads;  // head
  const int heads = min(kHeads, shared_by - group * kHeads);
  const int64_t held = (int64_t)a.sinks + a.window;
  const int64_t slot = a.slots ? a.slots[b] : b, position = a.positions[b];
  T *y = a.y + b * a.y_step + (int64_t)first * a.dim;
  if (slot < 0 || slot >= a.num_slots || position < 0) {  // the whole cluster
    if (rank == 0)
      for (int i = threadIdx.x; i < heads * a.dim; i += kThreads) y[i] = from_f<T>(0.f);
    return;
  }
  const int64_t place =
      position < a.sinks ? position : a.sinks + (position - a.sinks) % a.window;
  const int64_t rows = min(position, held);  // of earlier tokens, and `place` among them once full
  const int64_t pitch = (int64_t)a.kv_heads * a.dim;
  T *keys = a.cache_k + (slot * held * a.kv_heads + kv) * a.dim;
  T *values = a.cache_v + (slot * held * a.kv_heads + kv) * a.dim;
  const T *new_k = a.k + b * a.k_step + (int64_t)kv * a.dim;
  const T *new_v = a.v + b * a.v_step + (int64_t)kv * a.dim;

  const int chunks = a.dim / 8;
  uint32_t ring = smem_u32(s.ring[warp]);
  constexpr uint32_t kBytes = kTile * DP * 2;
  if (chunks < DP / 8)  // values from dim on
    for (int i = lane; i < kStages * 2 * kTile * (DP / 8); i += 32) {
      const int c = i % (DP / 8), r = i / (DP / 8);
      if (c >= chunks)
        *reinterpret_cast<uint4 *>(&s.ring[warp][0][0][0] + r / kTile * kBytes +
                                   chunk_at<DP>(r % kTile, c)) = make_uint4(0, 0, 0, 0);
    }

  Walk<T, DP> w;
#pragma unroll
  for (int i = 0; i < DP / 16; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int h = lane / 4 + (e & 1) * 8, at = 16 * i + 2 * (lane % 4) + (e >> 1) * 8;
      w.q[i][e] = h < heads && at < a.dim
                      ? *reinterpret_cast<const uint32_t *>(
                            a.q + b * a.q_step + (int64_t)(first + h) * a.dim + at)
                      : 0u;
    }
#pragma unroll
  for (int i = 0; i < DP / 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) w.o[i][e] = 0.f;
  w.m[0] = w.m[1] = -INFINITY;
  w.l[0] = w.l[1] = 0.f;

  const int64_t tiles = (rows + kTile - 1) / kTile, step = (int64_t)size * kWarps;
  const int64_t from = (int64_t)rank * kWarps + warp;
  auto load = [&](int64_t t, int stage) {
    if (t < tiles) {
#pragma unroll
      for (int i = 0; i < kTile * (DP / 8) / 32; ++i) {
        const int c = lane % (DP / 8), r = lane / (DP / 8) + i * (32 / (DP / 8));
        const int64_t row = t * kTile + r;
        const bool has = row < rows && row != place;  // others read as zeros
        if (c < chunks) {
          const int64_t at = (has ? row : 0) * pitch + c * 8;
          const uint32_t to = ring + stage * 2 * kBytes + chunk_at<DP>(r, c);
          cp_async16(to, keys + at, has);
          cp_async16(to + kBytes, values + at, has);
        }
      }
    }
    cp_commit();
  };
  const bool newest = rank == 0 && warp == 0;  // this warp takes the token's own row
  if (newest) {
    for (int i = lane; i < 2 * kTile * chunks; i += 32) {
      const int c = i % chunks, r = i / chunks;  // rows of keys, then of values
      uint4 word = make_uint4(0, 0, 0, 0);
      if (r % kTile == 0) {
        word = *reinterpret_cast<const uint4 *>((r ? new_v : new_k) + c * 8);
        if (group == 0)
          *reinterpret_cast<uint4 *>((r ? values : keys) + place * pitch + c * 8) = word;
      }
      *reinterpret_cast<uint4 *>(&s.ring[0][0][0][0] + r / kTile * kBytes +
                                 chunk_at<DP>(r % kTile, c)) = word;
    }
    __syncwarp();
    w.tile(ring, ring + kBytes, 1, -1, a.c, lane);
  }
  __syncwarp();
  for (int i = 0; i < kStages - 1; ++i) load(from + i * step, i);
  int stage = 0;
  for (int64_t t = from; t < tiles; t += step) {
    load(t + (kStages - 1) * step, (stage + kStages - 1) % kStages);
    cp_wait<kStages - 1>();
    __syncwarp();
    const int count = (int)min((int64_t)kTile, rows - t * kTile);
    const int64_t skip = place - t * kTile;
    w.tile(ring + stage * 2 * kBytes, ring + stage * 2 * kBytes + kBytes, count,
           skip >= 0 && skip < kTile ? (int)skip : -1, a.c, lane);
    __syncwarp();
    stage = (stage + 1) % kStages;
  }
  cp_wait<0>();
  __syncwarp();

  // join: warps, then blocks
  float *mine = reinterpret_cast<float *>(s.ring[warp]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float l = w.l[h];
    l += __shfl_xor_sync(~0u, l, 1);
    l += __shfl_xor_sync(~0u, l, 2);
    const int row = lane / 4 + 8 * h;
    if (lane % 4 == 0) s.top[warp][row] = w.m[h], s.sum[warp][row] = l;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
      *reinterpret_cast<float2 *>(mine + row * DP + 8 * i + 2 * (lane % 4)) =
          make_float2(w.o[i][2 * h], w.o[i][2 * h + 1]);
  }
  __syncthreads();
  auto part = [&](float top, float of) { return of == -INFINITY ? 0.f : exp2_fast(of - top); };
  float *block = reinterpret_cast<float *>(s.ring[0]);
  for (int e = threadIdx.x; e < kHeads * DP; e += kThreads) {
    const int h = e / DP;
    float top = s.top[0][h], sum = 0.f, o = 0.f;
#pragma unroll
    for (int k = 1; k < kWarps; ++k) top = fmaxf(top, s.top[k][h]);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float by = part(top, s.top[k][h]);
      sum = fmaf(s.sum[k][h], by, sum);
      o = fmaf(reinterpret_cast<const float *>(s.ring[k])[e], by, o);
    }
    block[e] = o;
    if (e % DP == 0) s.block_top[h] = top, s.block_sum[h] = sum;
  }
  if (size == 1) {
    __syncthreads();
    for (int e = threadIdx.x; e < heads * a.dim; e += kThreads) {
      const int h = e / a.dim;
      y[e] = from_f<T>(block[h * DP + e - h * a.dim] / s.block_sum[h]);
    }
    return;
  }
  const cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  for (int e = rank * kThreads + threadIdx.x; e < heads * a.dim; e += size * kThreads) {
    const int h = e / a.dim, at = h * DP + e - h * a.dim;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int r = 0; r < size; ++r) top = fmaxf(top, *cluster.map_shared_rank(&s.block_top[h], r));
    for (int r = 0; r < size; ++r) {
      const float by = part(top, *cluster.map_shared_rank(&s.block_top[h], r));
      sum = fmaf(*cluster.map_shared_rank(&s.block_sum[h], r), by, sum);
      o = fmaf(*cluster.map_shared_rank(block + at, r), by, o);
    }
    y[e] = from_f<T>(o / sum);
  }
  cluster.sync();  // no block leaves while others read from it
}

template <typename T, int DP>
int step(const tcu_window_attention_args &s, cudaStream_t st) {
  StepArgs<T> a{};
  a.q = static_cast<const T *>(s.q.ptr);
  a.k = static_cast<const T *>(s.k.ptr);
  a.v = static_cast<const T *>(s.v.ptr);
  a.y = static_cast<T *>(s.y.ptr);
  a.q_step = s.q.batch_stride;
  a.k_step = s.k.batch_stride;
  a.v_step = s.v.batch_stride;
  a.y_step = s.y.batch_stride;
  a.cache_k = static_cast<T *>(s.cache_k);
  a.cache_v = static_cast<T *>(s.cache_v);
  a.slots = s.slots;
  a.positions = s.positions;
  a.num_slots = s.num_slots;
  a.batch = s.sequences;
  a.heads = s.heads;
  a.kv_heads = s.kv_heads;
  a.dim = s.dim;
  a.window = s.window;
  a.sinks = s.sinks;
  a.head_groups = (s.heads / s.kv_heads + kHeads - 1) / kHeads;
  a.c = s.scale * kLog2e;
  // Blocks of a cluster share an entry's rows, where blocks are fewer than SMs
  // and a warp still has a few tiles: a block costs some 10 us beside its rows (the
  // chain above).  Launch included, 64 entries x 8 key heads x 2052 rows: 109 us
  // whole, 126 in clusters of 2, 138 of 4; 16 x 2 x 4100 rows of 64 values: 37 us
  // whole, 19 in clusters of 8.
  const int64_t blocks = (int64_t)a.head_groups * s.kv_heads * s.sequences;
  const int64_t tiles = ((int64_t)s.window + s.sinks + kTile - 1) / kTile;
  int size = 1;
  while (size < kMostCluster && blocks * size <= num_sms() && tiles >= 4 * size * kWarps) size *= 2;
  if (blocks * size > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  constexpr int bytes = sizeof(StepShared<DP>);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(blocks * size));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = size > 1 ? 1 : 0;
  cudaError_t e = cudaFuncSetAttribute(attend_step_kernel<T, DP>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, attend_step_kernel<T, DP>, a, size);
  if (e == cudaSuccess) return launched();
  cudaGetLastError();
  return TCU_DFT_ERR_CUDA;
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int tcu_window_attention_step(const tcu_window_attention_args *a, void *stream) {
  if (const int rc = check_attention(a)) return rc;
  if (a->rows != 1 || a->offsets || a->num_slots < 0 || (!a->slots && a->num_slots < a->sequences))
    return TCU_DFT_ERR_INVALID;
  if (a->sequences == 0) return TCU_DFT_OK;
  const int64_t qs = (int64_t)a->heads * a->dim, ks = (int64_t)a->kv_heads * a->dim;
  if (!attn_rows_ok(a->q, a->sequences, 1, qs) || !attn_rows_ok(a->k, a->sequences, 1, ks) ||
      !attn_rows_ok(a->v, a->sequences, 1, ks) || !attn_rows_ok(a->y, a->sequences, 1, qs) ||
      !a->positions || (a->num_slots > 0 && (!a->cache_k || !a->cache_v)) ||
      (uintptr_t)a->cache_k % 16 || (uintptr_t)a->cache_v % 16)
    return TCU_DFT_ERR_INVALID;
  const wide_int bytes = (wide_int)a->num_slots * ((int64_t)a->sinks + a->window) * ks * 2;
  for (const void *c : {a->cache_k, a->cache_v}) {
    for (const tcu_seq_rows *r : {&a->q, &a->k, &a->v, &a->y})
      if (over(c, bytes, r->ptr, (r == &a->q || r == &a->y ? qs : ks) * 2, a->sequences,
               r->batch_stride * 2))
        return TCU_DFT_ERR_INVALID;
    if (over(c, bytes, a->slots, (int64_t)a->sequences * 4) ||
        over(c, bytes, a->positions, (int64_t)a->sequences * 4))
      return TCU_DFT_ERR_INVALID;
  }
  if (a->num_slots > 0 &&
      (over(a->cache_k, bytes, a->cache_v, 1) || over(a->cache_v, bytes, a->cache_k, 1)))
    return TCU_DFT_ERR_INVALID;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->type == TCU_SEQ_BF16)
    return a->dim <= 64 ? step<bf16, 64>(*a, st) : step<bf16, 128>(*a, st);
  return a->dim <= 64 ? step<f16, 64>(*a, st) : step<f16, 128>(*a, st);
}
