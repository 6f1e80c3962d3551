// The kernels for 4-bit microscaled matrices (mx_kernel.hpp) and the host functions that launch them.
#include "mx_kernel.hpp"

namespace dmm {
namespace {

using Mx256 = NtShape<true, 256>;
using Mx128 = NtShape<true, 128>;            // two workgroups on a CU
using Mx128Deep = NtShape<true, 128, 4>;     // one, which then has three steps on their way
static_assert(kMxShape[MX_256].tm == Mx256::TM && kMxShape[MX_256].tn == Mx256::TN && kMxShape[MX_128].tm == Mx128::TM &&
                  kMxShape[MX_128].tn == Mx128::TN && kMxShape[MX_SKINNY_16].tn == 16 && kMxShape[MX_SKINNY_32].tn == 32 &&
                  kMxShape[MX_SKINNY_64].tn == 32,
              "the host cuts tiles as the kernels expect them");

template <class SH>
bool launch(hipEvent_t behind, const MxItem *items, int n, const NtSeg *segs, hipStream_t stream) {
  return launch_behind(behind, mx_gemm_kernel<SH>, (unsigned)n, NT_THREADS, SH::LDS, stream, items, segs);
}

static_assert(MxBlock<false>::COLS == mx_block_cols(false) && MxBlock<true>::COLS == mx_block_cols(true), "blocks along the columns");

}  // namespace

hipError_t mx_allow_lds() {
  hipError_t e = hipFuncSetAttribute((const void *)mx_gemm_kernel<Mx256>, hipFuncAttributeMaxDynamicSharedMemorySize, Mx256::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)mx_gemm_kernel<Mx128>, hipFuncAttributeMaxDynamicSharedMemorySize, Mx128::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)mx_gemm_kernel<Mx128Deep>, hipFuncAttributeMaxDynamicSharedMemorySize, Mx128Deep::LDS);
  return e;
}

bool mx_launch(hipEvent_t behind, int shape, const MxItem *items, int n_items, const NtSeg *segs, const MxJoin *joins, int n_joins, int cus, hipStream_t stream) {
  const hipEvent_t last = n_joins ? nullptr : behind;
  bool marked = false;
  switch (shape) {
    case MX_256: marked = launch<Mx256>(last, items, n_items, segs, stream); break;
    case MX_128: marked = n_items <= cus ? launch<Mx128Deep>(last, items, n_items, segs, stream) : launch<Mx128>(last, items, n_items, segs, stream); break;
    case MX_SKINNY_16: marked = launch_behind(last, mx_skinny_kernel<1, 1>, (unsigned)n_items, NT_THREADS, 0, stream, items, segs); break;
    case MX_SKINNY_32: marked = launch_behind(last, mx_skinny_kernel<2, 2>, (unsigned)n_items, NT_THREADS, 0, stream, items, segs); break;
    default: marked = launch_behind(last, mx_skinny_kernel<4, 2>, (unsigned)n_items, NT_THREADS, 0, stream, items, segs); break;
  }
  if (!n_joins || hipPeekAtLastError() != hipSuccess) return marked;
  const int per = (kMxShape[shape].tm * kMxShape[shape].tn + 1023) / 1024;
  return launch_behind(behind, mx_join_kernel, (unsigned)(n_joins * per), 256, 0, stream, joins, per);
}

int mx_rows_per_unit(int64_t units) { return units >= 16384 ? 4 : 1; }

void mx_quantize_launch(const MxTileArgs &args, int blocks, bool f32, int along, int rows_per_unit, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (along == MX_ALONG_ROWS) {
    if (f32) rows_per_unit == 4 ? mx_rows_kernel<true, 4><<<grid, block, 0, stream>>>(args) : mx_rows_kernel<true, 1><<<grid, block, 0, stream>>>(args);
    else rows_per_unit == 4 ? mx_rows_kernel<false, 4><<<grid, block, 0, stream>>>(args) : mx_rows_kernel<false, 1><<<grid, block, 0, stream>>>(args);
  } else if (along == MX_ALONG_COLS) {
    if (f32) mx_cols_kernel<true, false><<<grid, block, 0, stream>>>(args);
    else mx_cols_kernel<false, false><<<grid, block, 0, stream>>>(args);
  } else {
    if (f32) mx_cols_kernel<true, true><<<grid, block, 0, stream>>>(args);
    else mx_cols_kernel<false, true><<<grid, block, 0, stream>>>(args);
  }
}

void mx_values_launch(const MxTileArgs &args, int blocks, bool f32, int along, int rows_per_unit, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (along == MX_ALONG_ROWS) {
    if (f32) rows_per_unit == 4 ? mx_row_values_kernel<true, 4><<<grid, block, 0, stream>>>(args) : mx_row_values_kernel<true, 1><<<grid, block, 0, stream>>>(args);
    else rows_per_unit == 4 ? mx_row_values_kernel<false, 4><<<grid, block, 0, stream>>>(args) : mx_row_values_kernel<false, 1><<<grid, block, 0, stream>>>(args);
  } else {
    if (f32) mx_col_values_kernel<true><<<grid, block, 0, stream>>>(args);
    else mx_col_values_kernel<false><<<grid, block, 0, stream>>>(args);
  }
}

}  // namespace dmm
