// The kernels for 4-bit microscaled matrices (mx_kernel.hpp) and the host functions that launch them.
#include "mx_kernel.hpp"

namespace dmm {
namespace {

using Mx256 = NtShape<true, 256>;
using Mx128 = NtShape<true, 128>;            // two workgroups on a CU
using Mx128Deep = NtShape<true, 128, 128, 4>;     // one, which then has three steps on their way
using Mx64 = NtShape<true, 64, 128, 2>;          // few rows: bound by the bytes of B
using Mx32 = NtShape<true, 32, 128, 3, 1>;
template <class SH>
constexpr bool same(int shape) { return kMxShape[shape].tm == SH::TM && kMxShape[shape].tn == SH::TN; }
static_assert(same<Mx256>(MX_256) && same<Mx128>(MX_128) && same<Mx64>(MX_64) && same<Mx32>(MX_32) && kMxShape[MX_SKINNY].tn == 16,
              "the host cuts tiles as the kernels expect them");

template <class SH>
hipError_t allow() {
  return hipFuncSetAttribute((const void *)mx_gemm_kernel<SH>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
}

template <class SH>
bool launch(hipEvent_t behind, const MxItem *items, int n, const NtSeg *segs, hipStream_t stream) {
  return launch_behind(behind, mx_gemm_kernel<SH>, (unsigned)n, NT_THREADS, SH::LDS, stream, items, segs);
}

static_assert(MxBlock<false>::COLS == mx_block_cols(false) && MxBlock<true>::COLS == mx_block_cols(true), "blocks along the columns");

}  // namespace

hipError_t mx_allow_lds() {
  hipError_t e = allow<Mx256>();
  if (e == hipSuccess) e = allow<Mx128>();
  if (e == hipSuccess) e = allow<Mx128Deep>();
  if (e == hipSuccess) e = allow<Mx64>();
  if (e == hipSuccess) e = allow<Mx32>();
  return e;
}

bool mx_launch(hipEvent_t behind, int shape, const MxItem *items, int n_items, const NtSeg *segs, const MxJoin *joins, int n_joins, int cus, hipStream_t stream) {
  const hipEvent_t last = n_joins ? nullptr : behind;
  bool marked = false;
  switch (shape) {
    case MX_256: marked = launch<Mx256>(last, items, n_items, segs, stream); break;
    case MX_128: marked = n_items <= cus ? launch<Mx128Deep>(last, items, n_items, segs, stream) : launch<Mx128>(last, items, n_items, segs, stream); break;
    case MX_64: marked = launch<Mx64>(last, items, n_items, segs, stream); break;
    case MX_32: marked = launch<Mx32>(last, items, n_items, segs, stream); break;
    default: marked = launch_behind(last, mx_skinny_kernel, (unsigned)n_items, NT_THREADS, 0, stream, items, segs); break;
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
