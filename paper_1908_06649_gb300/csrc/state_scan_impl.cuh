// state_scan_impl.cuh -- launches of the scan kernels for one element type.
#pragma once
#include "state_scan.cuh"

namespace tcu {
namespace seq {

template <typename T>
ScanArgs<T> args_of(const tcu_state_scan_args &s, const ScanPlan &p, ScanCall call) {
  const bool grad = call == kScanGrad, step = call == kScanStep;
  ScanArgs<T> a{};
  a.u = rows_of<const T>(s.u);
  a.dt = rows_of<const T>(s.dt);
  a.gate = rows_of<const T>(s.gate);
  a.B = rows_of<const T>(s.B);
  a.C = rows_of<const T>(s.C);
  a.A = s.A;
  a.skip = s.skip;
  a.dt_bias = s.dt_bias;
  a.state = s.state;
  a.last = s.last;
  a.marks = s.marks;
  a.offsets = s.offsets;
  a.slots = s.slots;
  a.rows = (int)s.rows;
  a.channels = s.channels;
  a.num_slots = s.num_slots;
  a.chunk_rows = (int)p.chunk_rows;
  a.states = (int)s.states;
  a.groups = s.groups;
  a.per_group = p.per_group;
  a.group_blocks = p.group_blocks;
  a.sequences = s.sequences;
  a.batches = (int)p.batches;
  a.chunks = p.chunks;
  a.softplus = s.softplus;
  if (!grad) a.y = rows_of<T>(s.y);
  auto whole = [&](const void *q) { return (uintptr_t)q % 16 == 0; };
  a.wide_states = s.states % 4 == 0 && whole(s.A) && whole(s.state) && whole(s.last) &&
                  whole(s.marks) && whole(s.workspace) && whole(s.dlast) && whole(s.dstate);
  const int64_t batches = step ? s.sequences : p.batches, rows = s.rows;
  a.wide_bc = s.states % 4 == 0 && rows_aligned(s.B, s.type, batches, rows, 4 * sizeof(T)) &&
              rows_aligned(s.C, s.type, batches, rows, 4 * sizeof(T));
  constexpr int most = 8;  // values of a word of rows, at most 16 bytes
  const int word = std::min<int>(16, most * sizeof(T));
  a.wide = p.per_group % most == 0;
  for (const tcu_seq_rows *r : {&s.u, &s.dt, &s.gate})
    a.wide = a.wide && rows_aligned(*r, s.type, batches, rows, word);
  if (!grad) a.wide = a.wide && rows_aligned(s.y, s.type, batches, rows, word);
  else
    for (const tcu_seq_rows *r : {&s.dy, &s.du, &s.ddt, &s.dgate})
      a.wide = a.wide && rows_aligned(*r, s.type, batches, rows, word);
  if (step)  // one row an entry: entries step as rows do
    for (Rows<const T> *r : {&a.u, &a.dt, &a.gate, &a.B, &a.C}) r->row = (int32_t)r->batch;
  if (step) a.y.row = (int32_t)(a.y.batch = s.y.batch_stride);
  float *w = static_cast<float *>(s.workspace);
  a.carry = w;
  a.sum_d = a.carry + p.carry;
  a.row_seq = s.offsets ? reinterpret_cast<int32_t *>(a.sum_d + p.sum_d) : nullptr;
  if (grad) {
    a.dy = rows_of<const T>(s.dy);
    a.du = rows_of<T>(s.du);
    a.ddt = rows_of<T>(s.ddt);
    a.dgate = rows_of<T>(s.dgate);
    a.dB = rows_of<T>(s.dB);
    a.dC = rows_of<T>(s.dC);
    a.dlast = s.dlast;
    a.dstate = s.dstate;
    a.bc_parts = a.sum_d + p.sum_d + p.row_seq;
    a.A_parts = a.bc_parts + p.bc_parts;
    a.skip_parts = s.dskip ? a.A_parts + p.A_parts : nullptr;
    a.bias_parts = s.ddt_bias ? a.A_parts + p.A_parts + p.vec_parts : nullptr;
  }
  return a;
}

template <auto *kernel, typename T>
int start(int64_t blocks, int threads, int floats, const ScanArgs<T> &a, cudaStream_t st) {
  if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  const int bytes = floats * 4;
  if (bytes > 48 * 1024 &&
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) !=
          cudaSuccess) {
    cudaGetLastError();
    return TCU_DFT_ERR_CUDA;
  }
  kernel<<<(unsigned)blocks, threads, bytes, st>>>(a);
  return launched();
}

template <typename T, int LS, int NB, bool kWide>
int token_of(const ScanArgs<T> &a, cudaStream_t st) {
  const int64_t blocks = (a.channels * LS + kScanThreads - 1) / kScanThreads;
  if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  const int entries = (a.sequences + NB - 1) / NB;
  const dim3 grid((unsigned)blocks, (unsigned)std::min(entries, 65535));
  scan_step_kernel<T, LS, NB, kWide><<<grid, kScanThreads, 0, st>>>(a);
  return launched();
}

// Four entries a thread (two, where two lanes share a channel) once that
// leaves every SM some 1000 threads.
template <typename T, int LS, bool kWide>
int token(const ScanArgs<T> &a, cudaStream_t st) {
  constexpr int NB = LS < 4 ? 2 : 4;
  const int64_t threads = a.channels * a.sequences * LS;
  return threads >= NB * 1024 * (int64_t)num_sms() ? token_of<T, LS, NB, kWide>(a, st)
                                                   : token_of<T, LS, 1, kWide>(a, st);
}

template <typename T, bool kBack>
int carry(const ScanArgs<T> &a, cudaStream_t st) {
  const int64_t blocks = (a.channels * a.states + 127) / 128;
  if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)std::min(a.batches, 65535));
  carry_kernel<T, kBack><<<grid, 128, 0, st>>>(a);
  return launched();
}

template <typename T, int LS, bool kPacked, bool kWide>
int forward(const ScanPlan &p, const ScanArgs<T> &a, cudaStream_t st) {
  const int64_t blocks = p.batches * a.groups * p.group_blocks;
  constexpr int floats = Lay<LS, T, kWide>::kFloats;
  if (p.chunks > 1) {
    if (const int rc = start<scan_kernel<T, LS, kPacked, kState, kWide>>(blocks * (p.chunks - 1), Lay<LS, T, kWide>::kBlock, floats,
                                                                      a, st))
      return rc;
    if (const int rc = carry<T, false>(a, st)) return rc;
  }
  return start<scan_kernel<T, LS, kPacked, kOutputs, kWide>>(blocks * p.chunks, Lay<LS, T, kWide>::kBlock, floats, a, st);
}

template <typename T, int LS, bool kPacked, bool kWide>
int gradient(const ScanPlan &p, const ScanArgs<T> &a, cudaStream_t st) {
  if (p.chunks > 1) {
    using F = Lay<LS, T, kWide>;
    ScanArgs<T> c = a;
    c.group_blocks = (a.per_group + F::DB - 1) / F::DB;
    const int64_t blocks = p.batches * (p.chunks - 1) * a.groups * c.group_blocks;
    if (const int rc = start<scan_kernel<T, LS, kPacked, kAdjoint, kWide>>(blocks, F::kBlock,
                                                                        F::kFloats, c, st))
      return rc;
    if (const int rc = carry<T, true>(a, st)) return rc;
  }
  using L = GradLay<LS, T>;
  const int64_t blocks = p.batches * p.chunks * a.groups * p.group_blocks;
  return start<scan_grad_kernel<T, LS, kPacked, kWide>>(blocks, L::kBlock, L::kFloats, a, st);
}

template <typename T, int LS>
int by_lanes(ScanCall call, const ScanPlan &p, const ScanArgs<T> &a, cudaStream_t st) {
  if (call == kScanStep)
    return a.wide_states && a.wide_bc ? token<T, LS, true>(a, st) : token<T, LS, false>(a, st);
  if (call == kScan) {
    if (a.row_seq)
      return a.wide ? forward<T, LS, true, true>(p, a, st) : forward<T, LS, true, false>(p, a, st);
    return a.wide ? forward<T, LS, false, true>(p, a, st) : forward<T, LS, false, false>(p, a, st);
  }
  if (a.row_seq)
    return a.wide ? gradient<T, LS, true, true>(p, a, st) : gradient<T, LS, true, false>(p, a, st);
  return a.wide ? gradient<T, LS, false, true>(p, a, st) : gradient<T, LS, false, false>(p, a, st);
}

template <typename T>
int run_scan(ScanCall call, const tcu_state_scan_args &s, cudaStream_t st) {
  const ScanPlan p = plan_of(s, call == kScanGrad);
  const ScanArgs<T> a = args_of<T>(s, p, call);
  if (call != kScanStep && s.offsets && s.rows > 0) {
    row_sequence_kernel<<<(unsigned)((s.rows + 127) / 128), 128, 0, st>>>(
        a.row_seq, s.offsets, s.sequences, (int)s.rows);
    if (const int rc = launched()) return rc;
  }
  int rc = TCU_DFT_ERR_UNSUPPORTED;
  const bool none = call != kScanStep && (p.batches == 0 || s.rows == 0);
  if (none) rc = TCU_DFT_OK;
  else switch (p.ls) {
    case 2: rc = by_lanes<T, 2>(call, p, a, st); break;
    case 4: rc = by_lanes<T, 4>(call, p, a, st); break;
    case 8: rc = by_lanes<T, 8>(call, p, a, st); break;
    case 16: rc = by_lanes<T, 16>(call, p, a, st); break;
    case 32: rc = by_lanes<T, 32>(call, p, a, st); break;
  }
  if (rc != TCU_DFT_OK || call != kScanGrad) return rc;
  if (!none) {
    const int64_t each = kSumThreads / (2 * s.states);
    const int64_t blocks = (s.rows * s.groups + each - 1) / each;
    if (blocks > INT32_MAX) return TCU_DFT_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)std::min<int64_t>(p.batches, 65535));
    sum_bc_kernel<T><<<grid, kSumThreads, 0, st>>>(a);
    if ((rc = launched())) return rc;
  }
  const int64_t parts = none ? 0 : p.batches * p.chunks;
  Sum sums[3] = {{s.dA, a.A_parts, s.channels * s.states}};
  int count = 1;
  if (s.dskip) sums[count++] = {s.dskip, a.skip_parts, s.channels};
  if (s.ddt_bias) sums[count++] = {s.ddt_bias, a.bias_parts, s.channels};
  return sum_parts(sums, count, parts, 0, st);
}

}  // namespace seq
}  // namespace tcu
