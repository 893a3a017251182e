// attn_common.cuh -- what the kernels of window attention share: which keys a
// row sees, tiles in shared memory with the 128-byte swizzle and their
// descriptors, products of 16-bit operands, and the tensor maps.
//
// A tile of rows lies in shared memory as one or two blocks of 64 values a
// row, 128 bytes, the 16-byte chunks of row r permuted by r % 8 as TMA's
// 128-byte swizzle leaves them.  The tensor cores read the same tile along
// either axis: as an operand whose inner (summed) axis is the head's values,
// or, with the transposing bit of the instruction descriptor, one whose inner
// axis is the rows.
#pragma once
#include <cuda.h>

#include "../../include/tcu_attn.h"
#include "host_plan.h"
#include "seq_common.cuh"
#include "tcgen05.cuh"

namespace tcu {
namespace seq {

struct AttendArgs {
  const int32_t *offsets;
  float *lse;
  const float *delta;
  float *sizes;     // gradient in fp16: of each row and head, the sum of |dy_c y_c|
  uint32_t *peaks;  // and of each key, the bits of its largest term of ds
  int64_t rows;  // of a batch entry
  int sequences, heads, kv_heads, dim, window, sinks;
  float scale;
  int64_t q_tiles, k_tiles;
  int chunk, chunks, sink_tiles;  // gradient: how the rows that see first tokens are split
};

// ---------------------------------------------------------------- visibility
// The bits of [lo, hi) among 0..31.
__device__ __forceinline__ uint32_t bits_between(int lo, int hi) {
  const auto below = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };
  return below(hi) & ~below(lo);
}

// The keys that row i of a batch entry sees: [lo, i] and [s0, s1), s1 <= lo.
struct Seen {
  int i, lo, s0, s1;
  // which of [j0, j0 + 32), a bit each: a test of a constant bit and a selection
  // for each score, where bounds compared for each take ten times as long
  __device__ __forceinline__ uint32_t bits(int j0) const {
    return bits_between(lo - j0, i + 1 - j0) | bits_between(s0 - j0, s1 - j0);
  }
  // whether all of [j0, j1) is seen
  __device__ __forceinline__ bool whole(int j0, int j1) const { return j0 >= lo && j1 - 1 <= i; }
};

// The sequence [begin, end) of row i; false if it is in none.
__device__ __forceinline__ bool sequence_at(const AttendArgs &a, int64_t i, int &begin, int &end) {
  begin = 0;
  end = (int)a.rows;
  if (i >= a.rows) return false;
  if (a.offsets) {
    const int s = sequence_of(a.offsets, a.sequences, (int)i);
    if (s < 0) return false;
    begin = max(0, a.offsets[s]);
    end = min((int)a.rows, a.offsets[s + 1]);
  }
  return true;
}

// The rows that are in some sequence: [first, last), sequences following on
// each other.
struct Filled {
  int first, last;
  __device__ __forceinline__ explicit Filled(const AttendArgs &a)
      : first(a.offsets ? a.offsets[0] : 0),
        last(a.offsets ? a.offsets[a.sequences] : INT32_MAX) {}
  __device__ __forceinline__ bool holds(int i) const { return i >= first && i < last; }
};

__device__ __forceinline__ Seen seen_by(const AttendArgs &a, int64_t i) {
  Seen v{-1, INT32_MAX, 0, 0};
  int begin, end;
  if (!sequence_at(a, i, begin, end)) return v;
  v.i = (int)i;
  v.lo = max(begin, v.i - (a.window - 1));
  v.s0 = begin;
  v.s1 = a.sinks < v.lo - begin ? begin + a.sinks : v.lo;
  return v;
}

// ------------------------------------------------------------ tensor cores
template <typename T>
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, bool b_rows) {
  const uint32_t type = sizeof(T) == 2 && !__is_same(T, f16) ? 1u : 0u;  // bf16, f16
  return (1u << 4) | (type << 7) | (type << 10) | ((b_rows ? 1u : 0u) << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// A tile with the 128-byte swizzle.  Inner axis along a row's values: groups
// of 8 rows are 1024 bytes apart.  Inner axis along rows: the same step between
// groups of 8 rows, `block` bytes between blocks of 64 values.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr, uint32_t block) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((block >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;  // descriptor version for tcgen05
  d |= (uint64_t)2 << 61;  // 128-byte swizzle
  return d;
}

__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// D[128, ROWS_B] = A B^T over the DP values of a row: tiles of 128 and ROWS_B rows.
template <typename T, int DP, int ROWS_B>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t id = idesc_16<T>(128, ROWS_B, false);
#pragma unroll
  for (int k = 0; k < DP / 16; ++k)
    mma_f16_ss(d, desc_sw128(a + k / 4 * 128 * 128 + k % 4 * 32, 16),
               desc_sw128(b + k / 4 * ROWS_B * 128 + k % 4 * 32, 16), id, k > 0);
}

// D[128, DP] (+)= A B, A of 128 x ROWS_B 16-bit values in tensor memory, two to
// a column, B a tile of ROWS_B rows.  A's halves lie where the 32-bit values
// lay that they were formed from, in the first half of their columns: who
// writes one has read them itself.
template <typename T, int DP, int ROWS_B>
__device__ __forceinline__ void product_values(uint32_t d, uint32_t a, uint32_t b, bool add) {
  constexpr uint32_t id = idesc_16<T>(128, DP, true);
#pragma unroll
  for (int k = 0; k < ROWS_B / 16; ++k)
    mma_f16_ts(d, a + k / (ROWS_B / 32) * (ROWS_B / 2) + k % (ROWS_B / 32) * 8, desc_sw128(b + k * 16 * 128, ROWS_B * 128), id, add || k > 0);
}

__device__ __forceinline__ float2 splat(float v) { return make_float2(v, v); }

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t w;
  Pair<T>::put(&w, make_float2(lo, hi));
  return w;
}

__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t *v) {
  tmem_st16(taddr, reinterpret_cast<const float *>(v));
}

__device__ __forceinline__ void mbar_arrive(uint32_t addr) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory");
}

// A bounded wait of a whole warp, with one verdict for its lanes: a wait that
// runs out for some of them and not for others would part the warp before
// votes, elections and tensor-memory accesses that all lanes take together.
__device__ __forceinline__ bool warp_waits(uint32_t addr, uint32_t parity) {
  return __all_sync(~0u, mbar_wait_bounded(addr, parity));
}

// A box of 64 values x rows of one head: coordinates (value, head, row, batch).
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *map, int c0, int c1, int c2,
                                            int c3, uint32_t mbar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(mbar)
      : "memory");
}
template <int DP, int ROWS>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int head, int row,
                                          int batch, uint32_t mbar) {
#pragma unroll
  for (int c = 0; c < DP / 64; ++c)
    tma_load_4d(dst + c * ROWS * 128, map, c * 64, head, row, batch, mbar);
}
template <int DP, int ROWS>
constexpr uint32_t kTileBytes = DP * ROWS * 2;

// Looks over a tile of 64 rows from row j0 on, THREADS threads together (this
// one is `own`): zeros in the place of 16-byte chunks with values that are not
// finite, whose rows' bits go to `bad` (not null), and of rows in no sequence.
// A weight of zero times such a value is none, and would carry it to rows that
// do not see it.
template <typename T, int DP, int THREADS>
__device__ __forceinline__ void clean_tile(uint32_t tile, int own, int j0, const Filled &filled,
                                           unsigned long long *bad) {
  constexpr uint32_t kExponent = __is_same(T, f16) ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t kOne = __is_same(T, f16) ? 0x04000400u : 0x00800080u;
  constexpr int kChunks = 64 * (DP / 8) / THREADS, kBatch = kChunks < 8 ? kChunks : 8;
  const auto flags = [](const uint4 &w) {  // an exponent of ones carries
    return (((w.x & kExponent) + kOne) | ((w.y & kExponent) + kOne) | ((w.z & kExponent) + kOne) |
            ((w.w & kExponent) + kOne)) & 0x80008000u;
  };
  const auto at = [&](int k) { return tile + (uint32_t)(own + k * THREADS) * 16; };
  const auto load = [&](int k) {
    uint4 w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                 : "r"(at(k)));
    return w;
  };
  // nearly always there is nothing to do: loads by the batch, one test
  uint32_t any = 0;
#pragma unroll 1
  for (int k0 = 0; k0 < kChunks; k0 += kBatch) {
    uint4 w[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) w[k] = load(k0 + k);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) any |= flags(w[k]);
  }
  if (!any && filled.holds(j0) && filled.holds(j0 + 63)) return;
#pragma unroll 1
  for (int k = 0; k < kChunks; ++k) {
    const int r = (own + k * THREADS) / 8 % 64;
    const bool odd = flags(load(k)) != 0;
    if (odd && bad) atomicOr(bad, 1ull << r);
    if (odd || !filled.holds(j0 + r))
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at(k)), "r"(0) : "memory");
  }
}
__device__ __forceinline__ void fence_proxy_async_shared() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Stores 32 fp32 values of a row as 16-bit ones from column c0 on, those
// below dim (a multiple of 8).
template <typename T>
__device__ __forceinline__ void store_values(T *row, int c0, int dim, const float *v, float by) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (c0 + 8 * k >= dim) break;
    uint4 w;
    w.x = pack2<T>(v[8 * k] * by, v[8 * k + 1] * by);
    w.y = pack2<T>(v[8 * k + 2] * by, v[8 * k + 3] * by);
    w.z = pack2<T>(v[8 * k + 4] * by, v[8 * k + 5] * by);
    w.w = pack2<T>(v[8 * k + 6] * by, v[8 * k + 7] * by);
    *reinterpret_cast<uint4 *>(row + c0 + 8 * k) = w;
  }
}

// --------------------------------------------------------------- host side
// The map of a row tensor (batch entries x rows x heads x dim) in boxes of 64
// values x box_rows rows; values from dim on and rows from `rows` on read as
// zeros.
inline bool attn_map(CUtensorMap *m, const tcu_seq_rows &r, int type, int64_t batches,
                     int64_t rows, int heads, int dim, int box_rows) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = host::tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t row = (cuuint64_t)heads * dim * 2;
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)rows,
                              (cuuint64_t)batches};
  // a single row's or entry's pitch is never taken
  const cuuint64_t pitch = rows > 1 ? (cuuint64_t)r.row_stride * 2 : row;
  const cuuint64_t strides[3] = {(cuuint64_t)dim * 2, pitch,
                                 batches > 1 ? (cuuint64_t)r.batch_stride * 2 : pitch};
  const cuuint32_t box[4] = {64, 1, (cuuint32_t)box_rows, 1};
  const cuuint32_t each[4] = {1, 1, 1, 1};
  return enc(m,
             type == TCU_SEQ_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
             4, r.ptr, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows that tensor maps and 16-byte accesses reach: aligned, in rising order,
// apart.
inline bool attn_rows_ok(const tcu_seq_rows &r, int64_t batches, int64_t rows, int64_t values) {
  return r.ptr && rows_aligned(r, TCU_SEQ_BF16, batches, rows, 16) &&
         (rows <= 1 || r.row_stride >= values) &&
         (batches <= 1 || (r.batch_stride >= values && r.batch_stride < (1ll << 38)));
}

int check_attention(const tcu_window_attention_args *a);
inline int64_t attn_batches(const tcu_window_attention_args &a) {
  return a.offsets ? 1 : a.sequences;
}

inline AttendArgs attend_args(const tcu_window_attention_args &s) {
  AttendArgs a{};
  a.offsets = s.offsets;
  a.lse = s.lse;
  a.rows = s.rows;
  a.sequences = s.sequences;
  a.heads = s.heads;
  a.kv_heads = s.kv_heads;
  a.dim = s.dim;
  // beyond every row, and no sum of a row and one of them passes 2^31
  a.window = (int)std::min<int64_t>(s.window, std::max<int64_t>(1, s.rows));
  a.sinks = (int)std::min<int64_t>(s.sinks, s.rows);
  a.scale = s.scale;
  return a;
}

}  // namespace seq
}  // namespace tcu
