// state_scan_f32.cu -- the scan kernels for f32 rows (state_scan.cuh).
#include "state_scan_impl.cuh"

namespace tcu {
namespace seq {
template int run_scan<float>(ScanCall, const tcu_state_scan_args &, cudaStream_t);
}  // namespace seq
}  // namespace tcu
