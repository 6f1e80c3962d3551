// Kernels of the layers around a product (gfx950, device code only): products of 8-bit integers with a scale for every row and
// column, the gated block H = act(A Wg) * (A Wu), and the gradients of bf16 products, all on the macro-tiles of layer_tile.hpp.
//
// Sums, scales, activations and the product of both projections are fp32 (integers: int32 sums, converted once); a result is rounded once, on its
// way out.  The activation is applied where the sums are: G and U of 8192 x 49152 would be 3.2 GB written and read again, 1.3 ms beside 14.6.
#pragma once

#include "dmm.h"
#include "gemm_launch.hpp"
#include "layer_launch.hpp"
#include "layer_tile.hpp"

namespace dmm {

typedef __bf16 layer_bf16x2 __attribute__((ext_vector_type(2)));
typedef float layer_f32x2 __attribute__((ext_vector_type(2)));
typedef int layer_i32_any __attribute__((aligned(2)));        // (two bf16 at any address of one)
__device__ __forceinline__ unsigned short layer_bf16(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }

// ---- activations ------------------------------------------------------------------------------------

// 256 / (1 + e^-x): the instruction for 1 / x gives zero instead of results below the normal range, and 1 / (1 + e^87.4) is one; e^88.8 is past the range, its
// root is not.  (x / (1 + e^-x) then reaches down to the end of the normal range, x = -92.)
constexpr float kSigmoidUnit = 1.f / 256;
__device__ __forceinline__ float layer_sigmoid256(float x) {
  const float root = __builtin_amdgcn_exp2f(-0.7213475204f * x);
  return __builtin_amdgcn_rcpf(__builtin_fmaf(kSigmoidUnit * root, root, kSigmoidUnit));
}
constexpr float kTanhIn = 1.595769122f, kTanhCube = 0.044715f;   // 2 sqrt(2 / pi): (1 + tanh y) / 2 = 1 / (1 + e^-2y)

// The normal distribution's (1 + erf(g / sqrt 2)) / 2, to 5 units in the last place down to g = -2 and, where little is left of it, to 1.5 for every unit of the
// exponential's argument g^2 / 2, which is rounded to fp32 (12 units at -4, 126 at -13; 1 + erf would lose it altogether): with x = |g| / sqrt 2 and t = 1 / (1 + x / 2), erfc(x) e^(x^2) / t is a smooth function of t, here by the polynomial of degree 8
// whose largest relative error over x <= 14 is the least (2^-24; beyond, e^(-x^2) is zero).
__device__ __forceinline__ float layer_normal(float g) {
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3535533906f * __builtin_fabsf(g));
  float p = -0.0593864769f;
  p = __builtin_fmaf(p, t, 0.28612408f);
  p = __builtin_fmaf(p, t, -0.490406662f);
  p = __builtin_fmaf(p, t, 0.281733721f);
  p = __builtin_fmaf(p, t, -0.0291489121f);
  p = __builtin_fmaf(p, t, 0.203752726f);
  p = __builtin_fmaf(p, t, 0.24283506f);
  p = __builtin_fmaf(p, t, 0.282412112f);
  p = __builtin_fmaf(p, t, 0.282084316f);
  const float half = 0.5f * t * p * __builtin_amdgcn_exp2f(-0.7213475204f * g * g);
  return g < 0.f ? half : 1.f - half;
}

template <int ACT>
__device__ __forceinline__ float layer_act(float g) {
  if constexpr (ACT == DMM_SILU) return kSigmoidUnit * g * layer_sigmoid256(g);
  if constexpr (ACT == DMM_GELU) return g * layer_normal(g);
  return kSigmoidUnit * g * layer_sigmoid256(kTanhIn * (g + kTanhCube * g * g * g));
}
// act and its slope
__device__ __forceinline__ void layer_slope(int act, float g, float *value, float *slope) {
  if (act == DMM_SILU) {
    const float s256 = layer_sigmoid256(g), s = kSigmoidUnit * s256;
    *value = kSigmoidUnit * g * s256;
    *slope = s256 * (kSigmoidUnit * (1.f + g * (1.f - s)));
  } else if (act == DMM_GELU) {
    const float p = layer_normal(g);
    *value = g * p;
    *slope = p + g * 0.3989422804f * __builtin_amdgcn_exp2f(-0.7213475204f * g * g);
  } else {
    const float s256 = layer_sigmoid256(kTanhIn * (g + kTanhCube * g * g * g)), s = kSigmoidUnit * s256;
    *value = kSigmoidUnit * g * s256;
    // (g^2 past the range times no slope would be NaN; from |g| = 20 on s is 0 or 1 and the product zero)
    *slope = s + *value * (1.f - s) * kTanhIn * (1.f + 3.f * kTanhCube * __builtin_fminf(g * g, 1e30f));
  }
}

// A sum of integers times the scales of its row and its column, each given as m 2^e: no product on the way passes the range of fp32.
struct LayerScale {
  float m;
  int e;
};
__device__ __forceinline__ LayerScale layer_scale(float s) { return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }
__device__ __forceinline__ float layer_scaled(float v, LayerScale a, LayerScale b) { return __builtin_amdgcn_ldexpf(v * a.m * b.m, a.e + b.e); }

// ---- storing a tile -----------------------------------------------------------------------------------

// NJ tiles of 32 columns of a wave's part, `get(I, J, X)` the value of tile (I, J) in element X of the accumulators' layout.  fp32: half a wave stores 32
// neighbouring columns of a row.  bf16: the halves of a wave exchange two tiles of 32 columns, and lanes of an even and an odd column
// halves of these, so that a wave stores 64 columns of two rows, whole lines.  INSIDE: the whole part is; otherwise `rows` x `cols` of it.
template <class SH, int NJ, bool F32, bool INSIDE, class Get>
__device__ __forceinline__ void layer_store(char *c, int64_t ldc, int rows_left, int cols_left, Get &&get) {
  constexpr bool LINES = !F32 && NJ % 2 == 0;
  constexpr int ES = F32 ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const unsigned pitch = (unsigned)ldc * (unsigned)ES;
  const int row0 = (LINES ? 0 : 4 * (lane >> 5)) + (F32 ? 0 : lane & 1), col0 = F32 ? lane & 31 : LINES ? lane & 62 : lane & 30;
  const unsigned mine = (unsigned)row0 * pitch + (unsigned)col0 * (unsigned)ES;
  const unsigned pick = lane & 1 ? 0x07060302 : 0x01000504;   // bf16: the high halves of both lanes, or the low ones
  const int rows = rows_left - row0, cols = cols_left - col0; // below which the lane's are inside
  const char *at = (const char *)nt_uniform(c);
  // two rows of a column in each lane, one column on in the other of two lanes: two columns of one row, from row `row` and column `col` on
  auto pair = [&](unsigned own, const char *to, int row, int col) {
    const unsigned other = (unsigned)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true);   // lane ^ 1
    const int both = (int)__builtin_amdgcn_perm(own, other, pick);
    if (INSIDE || (row < rows && col + 1 < cols)) __builtin_nontemporal_store(both, (layer_i32_any *)(to + mine + col * 2));
    else if (row < rows && col < cols) *(unsigned short *)(to + mine + col * 2) = (unsigned short)both;
  };
  nt_for<SH::MI>([&](auto ic) {
    constexpr int I = decltype(ic)::value;
    nt_for<16>([&](auto xc) {
      constexpr int X = decltype(xc)::value, ROW = 32 * I + 8 * (X / 4) + X % 4;
      if constexpr (F32) {
        nt_for<NJ>([&](auto jc) {
          constexpr int J = decltype(jc)::value;
          if (INSIDE || (ROW < rows && 32 * J < cols)) __builtin_nontemporal_store(get(ic, jc, xc), (float *)(at + mine) + 32 * J);
        });
      } else if constexpr (X % 2 == 0) {
        auto two = [&](auto jc) {
          const layer_f32x2 v = {get(ic, jc, xc), get(ic, jc, std::integral_constant<int, X + 1>{})};
          return __builtin_bit_cast(unsigned, __builtin_convertvector(v, layer_bf16x2));
        };
        if constexpr (LINES) {
          nt_for<NJ / 2>([&](auto jc) {
            constexpr int J = 2 * decltype(jc)::value;
            // {first's lower half, second's lower half}: rows ROW, ROW + 1; {the upper halves}: four rows on
            const unsigned first = two(std::integral_constant<int, J>{});
            __builtin_amdgcn_sched_barrier(0);                // (registers)
            const auto r = __builtin_amdgcn_permlane32_swap(first, two(std::integral_constant<int, J + 1>{}), false, false);
            pair(r[0], at, ROW, 32 * J);
            pair(r[1], at + 4 * (int64_t)pitch, ROW + 4, 32 * J);
          });
        } else {
          nt_for<NJ>([&](auto jc) { pair(two(jc), at, ROW, 32 * decltype(jc)::value); });
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      at += X % 4 == 3 ? 5 * (int64_t)pitch : (int64_t)pitch;
    });
  });
}

template <class SH, int ACT>
__device__ __forceinline__ void layer_finish(const LayerTileSums<SH> &tile, const LayerItem &it, char *lds) {
  constexpr int NI = SH::NI, NJ = SH::DUAL ? NI / 2 : NI;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave_row = wave / SH::WN * (SH::TM / SH::WM);
  const int wave_col = wave % SH::WN * (SH::OUT / SH::WN);
  if (it.what == LAYER_PARTS) {
    // sums as they are: a slot's columns are the stage's (gated: those of the second right operand behind those of the first)
    auto bits = [&](auto ic, auto jc, auto xc) {
      const auto v = tile.acc[decltype(ic)::value][decltype(jc)::value][decltype(xc)::value];
      return __builtin_bit_cast(float, v);
    };
    char *const slot = it.c + (wave_row * SH::TN + wave_col) * 4;
    if constexpr (SH::DUAL) {
      layer_store<SH, NJ, true, true>(slot, SH::TN, 0, 0, [&](auto ic, auto jc, auto xc) { return bits(ic, std::integral_constant<int, 2 * decltype(jc)::value>{}, xc); });
      layer_store<SH, NJ, true, true>(slot + SH::OUT * 4, SH::TN, 0, 0,
                                      [&](auto ic, auto jc, auto xc) { return bits(ic, std::integral_constant<int, 2 * decltype(jc)::value + 1>{}, xc); });
    } else {
      layer_store<SH, NJ, true, true>(slot, SH::TN, 0, 0, bits);
    }
    return;
  }
  const int rows = it.m_ext - wave_row, cols = it.n_ext - wave_col;
  const bool inside = it.m_ext == SH::TM && it.n_ext == SH::OUT;
  // scales of the wave's rows are read four at a time from LDS, those of its columns once
  const __attribute__((address_space(3))) nt_f32x4 *row_scales = nullptr;
  LayerScale sb[SH::I8 ? NI : 1], sa[4];
  if constexpr (SH::I8) {
    __syncthreads();
    for (int x = threadIdx.x; x < SH::TM; x += LAYER_THREADS)
      ((__attribute__((address_space(3))) float *)(nt_lptr)lds)[x] = it.sa[min(x, it.m_ext - 1)];
    __syncthreads();
    row_scales = (const __attribute__((address_space(3))) nt_f32x4 *)((nt_lptr)lds + (wave_row + 4 * (lane >> 5)) * 4);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int col = min(wave_col + (SH::DUAL ? j / 2 : j) * 32 + (lane & 31), it.n_ext - 1);
      sb[j] = layer_scale((SH::DUAL && (j & 1) ? it.sb2 : it.sb)[col]);
    }
  }
  auto sum = [&](auto ic, auto jc, auto xc) {
    constexpr int I = decltype(ic)::value, J = decltype(jc)::value, X = decltype(xc)::value;
    if constexpr (SH::I8) return layer_scaled((float)tile.acc[I][J][X], sa[X % 4], sb[J]);
    else return tile.acc[I][J][X];
  };
  // (the stores ask for tiles in ascending order of rows)
  auto at_row = [&](auto ic, auto xc) {
    if constexpr (SH::I8 && decltype(xc)::value % 4 == 0) {
      const nt_f32x4 v = row_scales[decltype(ic)::value * 8 + decltype(xc)::value / 4 * 2];
#pragma unroll
      for (int y = 0; y < 4; ++y) sa[y] = layer_scale(v[y]);
    }
  };
  auto store = [&](char *c, int64_t ldc, int es, auto get) {
    auto with = [&](auto ic, auto jc, auto xc) {
      if constexpr (decltype(jc)::value == 0) at_row(ic, xc);
      return get(ic, jc, xc);
    };
    char *const mine = c + (int64_t)wave_row * ldc * es + wave_col * es;
    if (!SH::DUAL && es == 4) {
      if (inside) layer_store<SH, NJ, true, true>(mine, ldc, rows, cols, with);
      else layer_store<SH, NJ, true, false>(mine, ldc, rows, cols, with);
    } else {
      if (inside) layer_store<SH, NJ, false, true>(mine, ldc, rows, cols, with);
      else layer_store<SH, NJ, false, false>(mine, ldc, rows, cols, with);
    }
  };
  if constexpr (SH::DUAL) {
    auto gate = [&](auto ic, auto jc, auto xc) { return sum(ic, std::integral_constant<int, 2 * decltype(jc)::value>{}, xc); };
    auto up = [&](auto ic, auto jc, auto xc) { return sum(ic, std::integral_constant<int, 2 * decltype(jc)::value + 1>{}, xc); };
    if (it.g) store(it.g, it.ldg, 2, gate);
    if (it.u) store(it.u, it.ldu, 2, up);
    store(it.c, it.ldc, 2, [&](auto ic, auto jc, auto xc) { return layer_act<ACT>(gate(ic, jc, xc)) * up(ic, jc, xc); });
  } else {
    store(it.c, it.ldc, it.c_es, sum);
  }
}

// A region of C that no op writes.
__device__ __forceinline__ void layer_zeros(const LayerItem &it) {
  for (int x = threadIdx.x; x < it.m_ext * it.n_ext; x += LAYER_THREADS) {
    const int64_t row = x / it.n_ext, col = x % it.n_ext;
    if (it.c_es == 4) ((float *)it.c)[row * it.ldc + col] = 0.f;
    else ((unsigned short *)it.c)[row * it.ldc + col] = 0;
    if (it.g) ((unsigned short *)it.g)[row * it.ldg + col] = 0;
    if (it.u) ((unsigned short *)it.u)[row * it.ldu + col] = 0;
  }
}

template <class SH, int ACT>
__global__ __launch_bounds__(LAYER_THREADS, SH::LDS > 80 * 1024 ? 1 : 2) void layer_gemm_kernel(const LayerItem *__restrict__ items,
                                                                                               const LayerSeg *__restrict__ segs) {
  extern __shared__ char lds[];
  const LayerItem it = items[blockIdx.x];
  if (it.what == LAYER_ZERO) {
    layer_zeros(it);
    return;
  }
  LayerTileSums<SH> tile;
  tile.run(it, segs + it.seg, segs + it.tail_seg, lds);
  tile.pin();
  layer_finish<SH, ACT>(tile, it, lds);
}

// Macro-tiles of two kinds in one launch, of the same size: the gradients of a product, which wait for nothing of each other.  Each alone leaves places empty
// in its last round, or fills none.  (Gradients of 381 x 720 x 1112 uneven, copies included: 29 us in two launches, 20.5 in one.)
template <class SA, class SB>
__global__ __launch_bounds__(LAYER_THREADS, SA::LDS > 80 * 1024 ? 1 : 2) void layer_pair_kernel(const LayerItem *__restrict__ items,
                                                                                               const LayerSeg *__restrict__ segs) {
  static_assert(SA::LDS == SB::LDS && !SA::DUAL && !SB::DUAL, "one size of LDS, one epilogue");
  extern __shared__ char lds[];
  const LayerItem it = items[blockIdx.x];
  if (it.what == LAYER_ZERO) {
    layer_zeros(it);
    return;
  }
  auto multiply = [&](auto *sums) {
    using SH = std::remove_reference_t<decltype(*sums)>;
    LayerTileSums<SH> tile;
    tile.run(it, segs + it.seg, segs + it.tail_seg, lds);
    tile.pin();
    layer_finish<SH, DMM_SILU>(tile, it, lds);
  };
  if (it.kind == SA::KIND) multiply((SA *)nullptr);
  else multiply((SB *)nullptr);
}

// Sums of partial tiles, in ascending k: four columns a thread.  Integers are added in 64 bits: a run's sum fits 32, all together need not.
template <int KIND, int ACT>
__global__ __launch_bounds__(256) void layer_join_kernel(const LayerJoin *__restrict__ joins, int blocks_per_join) {
  constexpr bool I8 = layer_i8(KIND), DUAL = layer_gated(KIND);
  const LayerJoin jn = joins[blockIdx.x / blocks_per_join];
  const int out = DUAL ? jn.tn / 2 : jn.tn;
  const int at = ((blockIdx.x % blocks_per_join) * 256 + threadIdx.x) * 4;
  const int row = at / out, col = at % out;
  if (row >= jn.m_ext || col >= jn.n_ext) return;
  const int64_t slot = (int64_t)jn.tm * jn.tn * 4;
  auto total = [&](const char *p, const float *scales, float v[4]) {
    if constexpr (I8) {
      int64_t sum[4] = {0, 0, 0, 0};
      for (int r = 0; r < jn.runs; ++r) {
        const nt_i32x4 x = *(const nt_i32x4 *)(p + r * slot);
#pragma unroll
        for (int y = 0; y < 4; ++y) sum[y] += x[y];
      }
      const LayerScale a = layer_scale(jn.sa[row]);
#pragma unroll
      for (int y = 0; y < 4; ++y) v[y] = layer_scaled((float)sum[y], a, layer_scale(scales[min(col + y, jn.n_ext - 1)]));
    } else {
      nt_f32x4 sum = *(const nt_f32x4 *)p;
      for (int r = 1; r < jn.runs; ++r) sum += *(const nt_f32x4 *)(p + r * slot);
#pragma unroll
      for (int y = 0; y < 4; ++y) v[y] = sum[y];
    }
  };
  float v[4], w[4];
  const char *const p = jn.parts + ((int64_t)row * jn.tn + col) * 4;
  total(p, jn.sb, v);
  auto put = [&](char *c, int64_t ldc, int es, const float *x) {
#pragma unroll
    for (int y = 0; y < 4; ++y)
      if (col + y < jn.n_ext) {
        const int64_t o = (int64_t)row * ldc + col + y;
        if (es == 4) ((float *)c)[o] = x[y];
        else ((unsigned short *)c)[o] = layer_bf16(x[y]);
      }
  };
  if constexpr (DUAL) {
    total(p + out * 4, jn.sb2, w);
    if (jn.g) put(jn.g, jn.ldg, 2, v);
    if (jn.u) put(jn.u, jn.ldu, 2, w);
#pragma unroll
    for (int y = 0; y < 4; ++y) v[y] = layer_act<ACT>(v[y]) * w[y];
  }
  put(jn.c, jn.ldc, jn.c_es, v);
}

}  // namespace dmm
