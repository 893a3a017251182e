// seq_index.h -- 32-bit row arithmetic of the sequence operators that has to
// hold up to their limits, for the host and the device.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define TCU_SEQ_FN __host__ __device__ __forceinline__
#else
#define TCU_SEQ_FN inline
#endif

namespace tcu {
namespace seq {

// The end of the chunk of `each` rows that starts at row r0 < rows.  r0 + each
// itself may pass 2^31: the last of 304 chunks of 2^31 - 4097 rows would end
// 5633 rows beyond them.
TCU_SEQ_FN int chunk_end(int r0, int each, int rows) {
  return each < rows - r0 ? r0 + each : rows;
}

// The sequence that holds row t of a packed tensor: the last s with
// offsets[s] <= t < offsets[s + 1], -1 if t is in none (values out of order
// still give -1 <= s < count).
TCU_SEQ_FN int sequence_of(const int32_t *offsets, int count, int t) {
  int lo = 0, hi = count;  // offsets[lo] <= t unless lo == 0
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;  // lo + hi may pass 2^31
    if (offsets[mid + 1] <= t) lo = mid + 1; else hi = mid;
  }
  return lo < count && offsets[lo] <= t ? lo : -1;
}

}  // namespace seq
}  // namespace tcu
