// state_scan_bf16.cu -- the scan kernels for bf16 rows (state_scan.cuh).
#include "state_scan_impl.cuh"

namespace tcu {
namespace seq {
template int run_scan<bf16>(ScanCall, const tcu_state_scan_args &, cudaStream_t);
}  // namespace seq
}  // namespace tcu
