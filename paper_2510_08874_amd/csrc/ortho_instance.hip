// The kernels that orthogonalise a matrix (ortho_kernel.hpp) and the host functions that launch them.
#include "ortho_kernel.hpp"

namespace dmm {
namespace {

using Ortho256 = NtShape<false, 256, 256>;
using Ortho128 = NtShape<false, 128, 128>;

template <class SH>
void launch(const OrthoProduct &g, hipStream_t stream) {
  const unsigned tiles = (unsigned)(g.count * g.tiles);
  ortho_product_kernel<SH><<<dim3(tiles * (unsigned)g.runs), dim3(NT_THREADS), SH::LDS, stream>>>(g);
  if (g.runs > 1) ortho_join_kernel<SH::TM><<<dim3(tiles * (SH::TM / 64)), dim3(256), 64 * (SH::TN + 4) * 4, stream>>>(g);
}

}  // namespace

hipError_t ortho_allow_lds() {
  hipError_t e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho256>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho256::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_product_kernel<Ortho128>, hipFuncAttributeMaxDynamicSharedMemorySize, Ortho128::LDS);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void *)ortho_join_kernel<256>, hipFuncAttributeMaxDynamicSharedMemorySize, 64 * 260 * 4);
  return e;
}

void ortho_norm_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_norm_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_split_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_split_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_store_launch(const OrthoTiles &args, int blocks, hipStream_t stream) { ortho_store_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void ortho_product_launch(const OrthoProduct &g, int edge, hipStream_t stream) {
  if (edge == 256) launch<Ortho256>(g, stream);
  else launch<Ortho128>(g, stream);
}

}  // namespace dmm
