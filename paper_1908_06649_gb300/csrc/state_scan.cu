// state_scan.cu -- entry points of the selective state-space scan
// (include/tcu_seq.h): argument checks, the split of rows into chunks and
// the workspace; the kernels are in state_scan.cuh.
#include "state_scan.cuh"

namespace tcu {
namespace seq {

__global__ void row_sequence_kernel(int32_t *row_seq, const int32_t *offsets, int count,
                                    int rows) {
  const int r = (int)(blockIdx.x * blockDim.x + threadIdx.x);
  if (r >= 0 && r < rows) row_seq[r] = sequence_of(offsets, count, r);
}

ScanPlan plan_of(const tcu_state_scan_args &a, bool grad) {
  ScanPlan p{};
  p.batches = a.offsets ? 1 : a.sequences;
  p.ls = lanes_of(a.states);
  p.db = grad ? grad_channels(p.ls) : scan_channels(p.ls);
  p.per_group = (int)(a.channels / a.groups);
  p.group_blocks = (p.per_group + p.db - 1) / p.db;
  const int64_t blocks = p.batches * a.groups * p.group_blocks;
  const int64_t tiles = (a.rows + kTile - 1) / kTile;
  // Where the blocks leave most of the card's slots empty, rows are split so
  // that all blocks run at once.  The forward scan then pays its recurrence
  // almost twice: at 2048 rows x 4096 channels x 16 states, 42 % of the slots,
  // 232 us whole against 276 split; 21 %, 232 against 173.  The gradient pays
  // less for it: 42 %, 852 us against 756.  Two more kernels cost some 130 rows
  // of a block's time (forward; 60, gradient): 37 rows x 768 channels take 11
  // us whole, 22 split (31 and 38), so few rows are left whole.
  const int64_t slots = (grad ? grad_resident(p.ls) : kResident) * (int64_t)num_sms();
  int64_t chunks = blocks == 0 || blocks * (grad ? 2 : 3) > slots ? 1 : slots / blocks;
  chunks = tiles < (grad ? 4 : 6) ? 1 : std::max<int64_t>(1, std::min(chunks, tiles));
  const int64_t chunk_tiles = std::max<int64_t>(1, (tiles + chunks - 1) / chunks);
  p.chunk_rows = chunk_tiles * kTile;
  p.chunks = (int)std::max<int64_t>(1, (a.rows + p.chunk_rows - 1) / p.chunk_rows);
  const int64_t parts = p.batches * p.chunks * a.channels;
  // each a multiple of 16 bytes, so that all are aligned if the workspace is
  auto whole = [](int64_t floats) { return (floats + 3) / 4 * 4; };
  p.carry = p.chunks > 1 ? whole(parts * a.states) : 0;
  p.sum_d = p.chunks > 1 ? whole(parts) : 0;
  p.row_seq = a.offsets ? whole(a.rows) : 0;
  if (grad) {
    p.bc_parts = whole(p.batches * a.rows * a.groups * 2 * a.states * p.group_blocks);
    p.A_parts = whole(parts * a.states);
    p.vec_parts = whole(parts);
  }
  return p;
}

extern template int run_scan<float>(ScanCall, const tcu_state_scan_args &, cudaStream_t);
extern template int run_scan<bf16>(ScanCall, const tcu_state_scan_args &, cudaStream_t);
extern template int run_scan<f16>(ScanCall, const tcu_state_scan_args &, cudaStream_t);

namespace {

int check_sizes(const tcu_state_scan_args *a) {
  if (!a || a->type < TCU_SEQ_F32 || a->type > TCU_SEQ_F16 || a->sequences < 0 || a->rows < 0 ||
      a->channels < 1 || a->states < 1 || a->groups < 1 || a->channels % a->groups)
    return TCU_DFT_ERR_INVALID;
  if (a->states > TCU_SEQ_MAX_STATES || a->rows > kMostRows || a->channels > INT32_MAX)
    return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r : {&a->u, &a->dt, &a->gate, &a->y, &a->B, &a->C, &a->dy, &a->du,
                                &a->ddt, &a->dgate, &a->dB, &a->dC})
    if (!pitch_fits(a->rows, r->row_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  return TCU_DFT_OK;
}

bool inputs_ok(const tcu_state_scan_args &a) {
  const int sz = type_size(a.type);
  return f32_ok(a.A) && opt_ok(a.skip, 4) && opt_ok(a.dt_bias, 4) && opt_ok(a.state, 4) &&
         opt_ok(a.last, 4) && opt_ok(a.marks, 4) && opt_ok(a.offsets, 4) &&
         opt_ok(a.gate.ptr, sz) && row_ok(a.u, sz) && row_ok(a.dt, sz) && row_ok(a.B, sz) &&
         row_ok(a.C, sz);
}

bool workspace_ok(const tcu_state_scan_args &a, int64_t bytes) {
  return a.workspace_bytes >= bytes && (bytes == 0 || f32_ok(a.workspace));
}

// An empty sequence ends in the state it starts from.  The kernels write the
// states of the others.
int empty_states(const tcu_state_scan_args &a, float *to, const float *from, void *stream) {
  if (!to || a.sequences == 0 || (!a.offsets && a.rows > 0)) return TCU_DFT_OK;
  const size_t bytes = (size_t)a.sequences * a.channels * a.states * 4;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, st)
                             : cudaMemsetAsync(to, 0, bytes, st);
  if (e == cudaSuccess) return TCU_DFT_OK;
  cudaGetLastError();
  return TCU_DFT_ERR_CUDA;
}

int by_type(ScanCall call, const tcu_state_scan_args &a, void *stream) {
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (a.type) {
    case TCU_SEQ_F32: return run_scan<float>(call, a, st);
    case TCU_SEQ_BF16: return run_scan<bf16>(call, a, st);
    default: return run_scan<f16>(call, a, st);
  }
}

}  // namespace
}  // namespace seq
}  // namespace tcu

using namespace tcu::seq;

extern "C" int64_t tcu_state_scan_workspace(const tcu_state_scan_args *a) {
  return check_sizes(a) == TCU_DFT_OK ? plan_of(*a, false).total() * 4 : -1;
}

extern "C" int64_t tcu_state_scan_grad_workspace(const tcu_state_scan_args *a) {
  return check_sizes(a) == TCU_DFT_OK ? plan_of(*a, true).total() * 4 : -1;
}

extern "C" int tcu_state_scan(const tcu_state_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (a->rows > 0 && a->sequences + (a->offsets != nullptr) > 0 &&
      (!inputs_ok(*a) || !row_ok(a->y, type_size(a->type)) ||
       !workspace_ok(*a, plan_of(*a, false).total() * 4)))
    return TCU_DFT_ERR_INVALID;
  if (const int rc = empty_states(*a, a->last, a->state, stream)) return rc;
  return by_type(kScan, *a, stream);
}

extern "C" int tcu_state_scan_grad(const tcu_state_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  const int sz = type_size(a->type);
  if (!f32_ok(a->dA) || !opt_ok(a->dskip, 4) || !opt_ok(a->ddt_bias, 4) ||
      !opt_ok(a->dlast, 4) || !opt_ok(a->dstate, 4))
    return TCU_DFT_ERR_INVALID;
  if (a->rows > 0 && a->sequences + (a->offsets != nullptr) > 0 &&
      (!inputs_ok(*a) || !a->marks || !row_ok(a->dy, sz) || !row_ok(a->du, sz) ||
       !row_ok(a->ddt, sz) || !row_ok(a->dB, sz) || !row_ok(a->dC, sz) ||
       !opt_ok(a->dgate.ptr, sz) || !workspace_ok(*a, plan_of(*a, true).total() * 4)))
    return TCU_DFT_ERR_INVALID;
  if (const int rc = empty_states(*a, a->dstate, a->dlast, stream)) return rc;
  return by_type(kScanGrad, *a, stream);
}

extern "C" int tcu_state_scan_step(const tcu_state_scan_args *a, void *stream) {
  if (const int rc = check_sizes(a)) return rc;
  if (a->rows != 1 || a->offsets || a->num_slots < 0 ||
      (!a->slots && a->num_slots < a->sequences) || !opt_ok(a->slots, 4))
    return TCU_DFT_ERR_INVALID;
  if (a->sequences > kMostEntries) return TCU_DFT_ERR_UNSUPPORTED;
  for (const tcu_seq_rows *r : {&a->u, &a->dt, &a->gate, &a->y, &a->B, &a->C})
    if (!pitch_fits(a->sequences, r->batch_stride)) return TCU_DFT_ERR_UNSUPPORTED;
  if (a->sequences == 0) return TCU_DFT_OK;
  if (!inputs_ok(*a) || !row_ok(a->y, type_size(a->type)) || (a->num_slots > 0 && !a->last))
    return TCU_DFT_ERR_INVALID;
  const int64_t entry = a->channels * a->states * 4;
  const wide_int cache = (wide_int)a->num_slots * entry;
  const int64_t row = a->channels * type_size(a->type);
  const int64_t coefficients = a->groups * a->states * type_size(a->type);
  for (const tcu_seq_rows *r : {&a->u, &a->dt, &a->gate, &a->B, &a->C, &a->y})
    if (over(a->last, cache, r->ptr, r == &a->B || r == &a->C ? coefficients : row, a->sequences,
             r->batch_stride * type_size(a->type)))
      return TCU_DFT_ERR_INVALID;
  if (over(a->last, cache, a->A, entry) || over(a->last, cache, a->skip, a->channels * 4) ||
      over(a->last, cache, a->dt_bias, a->channels * 4) ||
      over(a->last, cache, a->slots, (int64_t)a->sequences * 4))
    return TCU_DFT_ERR_INVALID;
  return by_type(kScanStep, *a, stream);
}
