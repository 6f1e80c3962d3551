// The kernels for the layers around a product and the host functions that launch them: one kind of product per object file
// (DMM_INSTANCE = LAYER_*), what goes element by element in one of its own (DMM_INSTANCE = LAYER_KINDS).
#if DMM_INSTANCE < 5
#include "layer_kernel.hpp"
#else
#include "layer_point_kernel.hpp"
#endif

namespace dmm {

#define DMM_CAT_(a, b) a##b
#define DMM_CAT(a, b) DMM_CAT_(a, b)

#if DMM_INSTANCE < 5
namespace {

constexpr int KIND = DMM_INSTANCE;
constexpr bool DUAL = layer_gated(KIND);
using L256 = LayerShape<KIND, 256, 256, 2, 2>;
using L128 = LayerShape<KIND, 128, DUAL ? 256 : 128, DUAL ? 3 : 2, 2>;   // (not gated: two workgroups on a CU)
using L64 = LayerShape<KIND == LAYER_TN ? LAYER_NT : KIND, 64, DUAL ? 256 : 128, 3, 2>;
using L32 = LayerShape<KIND == LAYER_TN ? LAYER_NT : KIND, 32, DUAL ? 256 : 128, DUAL ? 4 : 3, 1>;
constexpr bool SMALL = KIND != LAYER_TN;
// not gated, where every workgroup has a CU to itself: more steps on their way
using D128 = LayerShape<DUAL ? LAYER_NT : KIND, 128, 128, 4, 2>;
using D64 = LayerShape<SMALL && !DUAL ? KIND : LAYER_NT, 64, 128, 6, 2>;
using D32 = LayerShape<SMALL && !DUAL ? KIND : LAYER_NT, 32, 128, 7, 1>;
// gated, two workgroups on a CU
using L2 = LayerShape<DUAL ? KIND : LAYER_I8_GATED, KIND == LAYER_GATED ? 64 : 128, KIND == LAYER_GATED ? 256 : 128, 2, 2>;
template <class SH>
constexpr bool same(int shape) { return kLayerTile[KIND][shape].tm == SH::TM && kLayerTile[KIND][shape].tn == SH::OUT; }
static_assert(same<L256>(LAYER_256) && same<L128>(LAYER_128) && (!SMALL || (same<L64>(LAYER_64) && same<L32>(LAYER_32))) && (!DUAL || same<L2>(LAYER_TWO)),
              "the host cuts tiles as the kernels expect them");

template <class SH, int ACT>
hipError_t allow() {
  return hipFuncSetAttribute((const void *)layer_gemm_kernel<SH, ACT>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
}
template <int ACT>
hipError_t allow_all() {
  hipError_t e = allow<L256, ACT>();
  if (e == hipSuccess) e = allow<L128, ACT>();
  if constexpr (SMALL) {
    if (e == hipSuccess) e = allow<L64, ACT>();
    if (e == hipSuccess) e = allow<L32, ACT>();
  }
  if constexpr (DUAL)
    if (e == hipSuccess) e = allow<L2, ACT>();
  if constexpr (!DUAL) {
    if (e == hipSuccess) e = allow<D128, ACT>();
    if constexpr (SMALL) {
      if (e == hipSuccess) e = allow<D64, ACT>();
      if (e == hipSuccess) e = allow<D32, ACT>();
    }
  }
  return e;
}
template <class SH, int ACT>
bool launch_as(hipEvent_t behind, const LayerItem *items, int n, const LayerSeg *segs, hipStream_t stream) {
  return launch_behind(behind, layer_gemm_kernel<SH, ACT>, (unsigned)n, LAYER_THREADS, SH::LDS, stream, items, segs);
}
template <int ACT>
bool launch(hipEvent_t behind, int shape, int cus, const LayerItem *items, int n, const LayerSeg *segs, hipStream_t stream) {
  if (shape == LAYER_256) return launch_as<L256, ACT>(behind, items, n, segs, stream);
  if constexpr (DUAL)
    if (shape == LAYER_TWO) return launch_as<L2, ACT>(behind, items, n, segs, stream);
  if constexpr (!DUAL)
    if (n <= cus) {
      if constexpr (SMALL) {
        if (shape == LAYER_64) return launch_as<D64, ACT>(behind, items, n, segs, stream);
        if (shape == LAYER_32) return launch_as<D32, ACT>(behind, items, n, segs, stream);
      }
      return launch_as<D128, ACT>(behind, items, n, segs, stream);
    }
  if constexpr (SMALL) {
    if (shape == LAYER_64) return launch_as<L64, ACT>(behind, items, n, segs, stream);
    if (shape == LAYER_32) return launch_as<L32, ACT>(behind, items, n, segs, stream);
  }
  return launch_as<L128, ACT>(behind, items, n, segs, stream);
}

}  // namespace

#if DMM_INSTANCE == 4
namespace {
using N128 = LayerShape<LAYER_NT, 128, 128, 2, 2>;
using ND128 = LayerShape<LAYER_NT, 128, 128, 4, 2>;
template <class SA, class SB>
hipError_t allow_pair() {
  return hipFuncSetAttribute((const void *)layer_pair_kernel<SA, SB>, hipFuncAttributeMaxDynamicSharedMemorySize, SA::LDS);
}
}  // namespace
bool layer_launch_pair(hipEvent_t behind, int cus, const LayerItem *items, int n, const LayerSeg *segs, hipStream_t stream) {
  if (n <= cus) return launch_behind(behind, layer_pair_kernel<ND128, D128>, (unsigned)n, LAYER_THREADS, D128::LDS, stream, items, segs);
  return launch_behind(behind, layer_pair_kernel<N128, L128>, (unsigned)n, LAYER_THREADS, L128::LDS, stream, items, segs);
}
#endif

hipError_t DMM_CAT(layer_allow_lds_, DMM_INSTANCE)() {
  hipError_t e = allow_all<DMM_SILU>();
#if DMM_INSTANCE == 4
  if (e == hipSuccess) e = allow_pair<N128, L128>();
  if (e == hipSuccess) e = allow_pair<ND128, D128>();
#endif
  if constexpr (DUAL) {
    if (e == hipSuccess) e = allow_all<DMM_GELU>();
    if (e == hipSuccess) e = allow_all<DMM_GELU_TANH>();
  }
  return e;
}
bool DMM_CAT(layer_launch_, DMM_INSTANCE)(hipEvent_t behind, int shape, int act, int cus, const LayerItem *items, int n, const LayerSeg *segs,
                                          hipStream_t stream) {
  if constexpr (DUAL) {
    if (act == DMM_GELU) return launch<DMM_GELU>(behind, shape, cus, items, n, segs, stream);
    if (act == DMM_GELU_TANH) return launch<DMM_GELU_TANH>(behind, shape, cus, items, n, segs, stream);
  }
  return launch<DMM_SILU>(behind, shape, cus, items, n, segs, stream);
}

#else

hipError_t layer_allow_lds() {
  hipError_t e = layer_allow_lds_0();
  if (e == hipSuccess) e = layer_allow_lds_1();
  if (e == hipSuccess) e = layer_allow_lds_2();
  if (e == hipSuccess) e = layer_allow_lds_3();
  if (e == hipSuccess) e = layer_allow_lds_4();
  return e;
}

namespace {
template <int KIND>
bool join(hipEvent_t behind, int act, const LayerJoin *joins, int n, int per, hipStream_t stream) {
  if constexpr (layer_gated(KIND)) {
    if (act == DMM_GELU) return launch_behind(behind, layer_join_kernel<KIND, DMM_GELU>, (unsigned)(n * per), 256, 0, stream, joins, per);
    if (act == DMM_GELU_TANH) return launch_behind(behind, layer_join_kernel<KIND, DMM_GELU_TANH>, (unsigned)(n * per), 256, 0, stream, joins, per);
  }
  return launch_behind(behind, layer_join_kernel<KIND, DMM_SILU>, (unsigned)(n * per), 256, 0, stream, joins, per);
}
}  // namespace

bool layer_launch(hipEvent_t behind, int kind, int shape, int act, int cus, const LayerItem *items, int n_items, const LayerSeg *segs, const LayerJoin *joins,
                  int n_joins, hipStream_t stream) {
  const hipEvent_t last = n_joins ? nullptr : behind;
  bool marked = false;
  switch (kind) {
    case LAYER_I8: marked = layer_launch_0(last, shape, act, cus, items, n_items, segs, stream); break;
    case LAYER_I8_GATED: marked = layer_launch_1(last, shape, act, cus, items, n_items, segs, stream); break;
    case LAYER_GATED: marked = layer_launch_2(last, shape, act, cus, items, n_items, segs, stream); break;
    case LAYER_PAIR: marked = layer_launch_pair(last, cus, items, n_items, segs, stream); break;
    case LAYER_NT: marked = layer_launch_3(last, shape, act, cus, items, n_items, segs, stream); break;
    default: marked = layer_launch_4(last, shape, act, cus, items, n_items, segs, stream); break;
  }
  if (!n_joins || hipPeekAtLastError() != hipSuccess) return marked;
  const LayerTile tile = kLayerTile[kind == LAYER_PAIR ? LAYER_NT : kind][shape];
  const int per = (tile.tm * tile.tn + 1023) / 1024;
  switch (kind) {
    case LAYER_I8: return join<LAYER_I8>(behind, act, joins, n_joins, per, stream);
    case LAYER_I8_GATED: return join<LAYER_I8_GATED>(behind, act, joins, n_joins, per, stream);
    case LAYER_GATED: return join<LAYER_GATED>(behind, act, joins, n_joins, per, stream);
    default: return join<LAYER_NT>(behind, act, joins, n_joins, per, stream);
  }
}

void layer_copy_launch(const LayerCopy *jobs, int n, int blocks, hipStream_t stream) {
  layer_copy_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(jobs, n);
}
void slope_launch(const SlopeArgs &args, int blocks, hipStream_t stream) { layer_slope_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args); }
void i8_scales_launch(const I8ScaleArgs &args, int blocks, int what, hipStream_t stream) {
  i8_scales_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(args, what);
}
void i8_amax_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (f32) cols ? i8_amax_kernel<true, true><<<grid, block, 0, stream>>>(args) : i8_amax_kernel<true, false><<<grid, block, 0, stream>>>(args);
  else cols ? i8_amax_kernel<false, true><<<grid, block, 0, stream>>>(args) : i8_amax_kernel<false, false><<<grid, block, 0, stream>>>(args);
}
void i8_quantize_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (f32) cols ? i8_cols_kernel<true, false><<<grid, block, 0, stream>>>(args) : i8_rows_kernel<true><<<grid, block, 0, stream>>>(args);
  else cols ? i8_cols_kernel<false, false><<<grid, block, 0, stream>>>(args) : i8_rows_kernel<false><<<grid, block, 0, stream>>>(args);
}
void i8_whole_cols_launch(const I8Args &args, int blocks, bool f32, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (f32) i8_cols_kernel<true, true><<<grid, block, 0, stream>>>(args);
  else i8_cols_kernel<false, true><<<grid, block, 0, stream>>>(args);
}
void i8_values_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block(256);
  if (f32) cols ? i8_col_values_kernel<true><<<grid, block, 0, stream>>>(args) : i8_row_values_kernel<true><<<grid, block, 0, stream>>>(args);
  else cols ? i8_col_values_kernel<false><<<grid, block, 0, stream>>>(args) : i8_row_values_kernel<false><<<grid, block, 0, stream>>>(args);
}
template <bool F32>
static void whole_rows(const I8RowArgs &args, const dim3 &grid, const dim3 &block, hipStream_t stream) {
  if (args.groups > 1) args.n > 1 ? i8_whole_rows_kernel<F32, true, true><<<grid, block, 0, stream>>>(args) : i8_whole_rows_kernel<F32, false, true><<<grid, block, 0, stream>>>(args);
  else args.n > 1 ? i8_whole_rows_kernel<F32, true, false><<<grid, block, 0, stream>>>(args) : i8_whole_rows_kernel<F32, false, false><<<grid, block, 0, stream>>>(args);
}
void i8_whole_rows_launch(const I8RowArgs &args, int blocks, int threads, bool f32, hipStream_t stream) {
  const dim3 grid((unsigned)blocks), block((unsigned)threads);
  if (f32) whole_rows<true>(args, grid, block, stream);
  else whole_rows<false>(args, grid, block, stream);
}

#endif

}  // namespace dmm
