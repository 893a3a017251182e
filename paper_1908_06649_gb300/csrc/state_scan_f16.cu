// state_scan_f16.cu -- the scan kernels for f16 rows (state_scan.cuh).
#include "state_scan_impl.cuh"

namespace tcu {
namespace seq {
template int run_scan<f16>(ScanCall, const tcu_state_scan_args &, cudaStream_t);
}  // namespace seq
}  // namespace tcu
