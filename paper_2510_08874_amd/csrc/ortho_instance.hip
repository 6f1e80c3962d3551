// The kernels that orthogonalise a matrix (ortho_kernel.hpp) and the host functions that launch them.
#include "ortho_kernel.hpp"

namespace dmm {
namespace {

using Ortho256 = NtShape<false, 256>;
using Ortho128 = NtShape<false, 128>;            // two workgroups on a CU
using Ortho128Deep = NtShape<false, 128, 128, 4>;     // one, which then has three steps on their way

using Ortho64 = NtShape<false, 64, 64, 4>;            // two
using Ortho64Three = NtShape<false, 64, 64, 3>;       // three

template <class SH>
void launch(const OrthoProduct &g, hipStream_t stream) {
  const int cut = g.count * g.tiles - g.whole;
  ortho_product_kernel<SH><<<dim3((unsigned)(g.whole + cut * g.runs)), dim3(NT_THREADS), SH::LDS, stream>>>(g);
  if (cut) ortho_join_kernel<SH::TM><<<dim3((unsigned)(cut * (SH::TM / 16))), dim3(256), 0, stream>>>(g);
}

}  // namespace

hipError_t ortho_allow_lds() {
  hipError_t e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho256>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho256::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho128>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho128::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho128Deep>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho128Deep::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho64>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho64::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho64Three>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho64Three::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * ORTHO_AREA);
  return e;
}

void ortho_norm_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_norm_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_split_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_split_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_store_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_store_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_product_launch(const OrthoProduct &g, int edge, hipStream_t stream) {
  if (edge == 256) launch<Ortho256>(g, stream);
  else if (edge == 64 && g.whole + (g.count * g.tiles - g.whole) * g.runs <= 512) launch<Ortho64>(g, stream);
  else if (edge == 64) launch<Ortho64Three>(g, stream);
  else if (g.whole + (g.count * g.tiles - g.whole) * g.runs <= 256) launch<Ortho128Deep>(g, stream);
  else launch<Ortho128>(g, stream);
}

void ortho_small_launch(const OrthoSmall &args, int count, hipStream_t stream) {
  ortho_small_kernel<<<dim3((unsigned)count), dim3(ORTHO_SMALL_THREADS), 2 * ORTHO_AREA, stream>>>(args);
}

}  // namespace dmm
