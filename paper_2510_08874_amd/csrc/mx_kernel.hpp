// Matrices in 4-bit microscaled floating point (gfx950, device code only): quantisation, its inverse, and
// the products of two such matrices.
//
// A block of 32 elements along one axis has the scale 2^e, e = floor(log2(largest magnitude)) - 2 kept to [-127, 127],
// stored as the byte e + 127 (255: the block holds an infinity or a NaN, all of it stands for NaN); an element
// is a 4-bit code: sign, two bits of exponent, one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6).  The instruction that
// converts rounds to nearest, half-way values to the even code, and keeps what is larger than 6 at 6: checked against
// every bf16 value.
#pragma once

#include "gemm_launch.hpp"
#include "mx_launch.hpp"
#include "nt_kernel.hpp"

namespace dmm {

// ---- products -------------------------------------------------------------------------------------

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef int mx_i32_any __attribute__((aligned(2)));           // (two bf16 at any address of one)
__device__ __forceinline__ unsigned short mx_bf16(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }

// fp32: half a wave stores 32 neighbouring columns of a row.  bf16: the halves of a wave exchange two tiles of 32 columns, so that all lanes
// have neighbouring columns of the same two rows, and lanes of an even and an odd column halves of these: a wave stores 64 columns of
// two rows, whole lines.  Straight from the registers, 9300 cycles; by way of LDS, 64 rows at a time and 16 bytes a thread, the end of a tile took
// 11800 (19000 with one read of LDS after the other), half lines as many as whole ones but a layer's step 2 % more.  Addresses are a row's, the same for the wave, and a lane's, the same for
// all rows.  INSIDE: the whole macro-tile is.  (The host sees to it that a macro-tile's rows lie within 2^32 bytes.)
template <class SH, bool F32, bool INSIDE>
__device__ __forceinline__ void mx_store(const NtTile<SH> &tile, const MxItem &it) {
  constexpr bool LINES = !F32 && SH::NI % 2 == 0;             // (of one tile of 32 columns: half of a line)
  constexpr int ES = F32 ? 4 : 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave_row = wave / SH::WN * (SH::TM / SH::WM), wave_col = wave % SH::WN * (SH::TN / SH::WN);
  const unsigned pitch = (unsigned)it.ldc * (unsigned)ES;
  const int row0 = (LINES ? 0 : 4 * (lane >> 5)) + (F32 ? 0 : lane & 1), col0 = F32 ? lane & 31 : LINES ? lane & 62 : lane & 30;
  const unsigned mine = (unsigned)row0 * pitch + (unsigned)col0 * (unsigned)ES;
  const unsigned pick = lane & 1 ? 0x07060302 : 0x01000504;   // bf16: the high halves of both lanes, or the low ones
  const int rows = it.m_ext - wave_row - row0, cols = it.n_ext - wave_col - col0;   // below which the lane's are inside
  const char *at = (const char *)nt_uniform(it.c + (int64_t)wave_row * pitch + wave_col * ES);
  // two rows of a column in each lane, one column on in the other of two lanes: two columns of one row, from row `row` and column `col` on
  auto pair = [&](unsigned own, const char *to, int row, int col) {
    const unsigned other = (unsigned)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true);   // lane ^ 1
    const int both = (int)__builtin_amdgcn_perm(own, other, pick);
    if (INSIDE || (row < rows && col + 1 < cols)) __builtin_nontemporal_store(both, (mx_i32_any *)(to + mine + col * 2));
    else if (row < rows && col < cols) *(unsigned short *)(to + mine + col * 2) = (unsigned short)both;
  };
  nt_for<SH::MI>([&](auto ic) {
    constexpr int I = decltype(ic)::value;
    nt_for<16>([&](auto xc) {
      constexpr int X = decltype(xc)::value, ROW = 32 * I + 8 * (X / 4) + X % 4;
      if constexpr (F32) {
        nt_for<SH::NI>([&](auto jc) {
          constexpr int J = decltype(jc)::value;
          if (INSIDE || (ROW < rows && 32 * J < cols)) __builtin_nontemporal_store(tile.acc[I][J][X], (float *)(at + mine) + 32 * J);
        });
      } else if constexpr (X % 2 == 0) {
        auto two = [&](const nt_f32x16 &v) {
          return __builtin_bit_cast(unsigned, __builtin_convertvector((mx_f32x2){v[X], v[X + 1]}, mx_bf16x2));
        };
        if constexpr (LINES) {
          nt_for<SH::NI / 2>([&](auto jc) {
            constexpr int J = 2 * decltype(jc)::value;
            // {first's lower half, second's lower half}: rows ROW, ROW + 1; {the upper halves}: four rows on
            const auto r = __builtin_amdgcn_permlane32_swap(two(tile.acc[I][J]), two(tile.acc[I][J + 1]), false, false);
            pair(r[0], at, ROW, 32 * J);
            pair(r[1], at + 4 * (int64_t)pitch, ROW + 4, 32 * J);
          });
        } else {
          nt_for<SH::NI>([&](auto jc) { pair(two(tile.acc[I][decltype(jc)::value]), at, ROW, 32 * decltype(jc)::value); });
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      at += X % 4 == 3 ? 5 * (int64_t)pitch : (int64_t)pitch;
    });
  });
}

// A region of C that no op writes.
__device__ __forceinline__ void mx_zeros(const MxItem &it) {
  for (int x = threadIdx.x; x < it.m_ext * it.n_ext; x += NT_THREADS) {
    const int64_t at = (int64_t)(x / it.n_ext) * it.ldc + x % it.n_ext;
    if (it.c_es == 4) ((float *)it.c)[at] = 0.f;
    else ((unsigned short *)it.c)[at] = 0;
  }
}

// Macro-tiles.
template <class SH>
__global__ __launch_bounds__(NT_THREADS, SH::LDS > 80 * 1024 ? 1 : 2) void mx_gemm_kernel(const MxItem *__restrict__ items, const NtSeg *__restrict__ segs) {
  extern __shared__ char lds[];
  const MxItem it = items[blockIdx.x];
  if (it.steps == 0) {
    mx_zeros(it);
    return;
  }
  NtTile<SH> tile;
  tile.run(it.front, segs + it.seg, it.n_segs, it.first, it.steps, it.m_off, it.m_ext, it.n_off, it.n_ext, lds);
  tile.pin();
  const bool inside = it.m_ext == SH::TM && it.n_ext == SH::TN;
  if (it.c_es == 4) {
    if (inside) mx_store<SH, true, true>(tile, it);
    else mx_store<SH, true, false>(tile, it);
  } else {
    if (inside) mx_store<SH, false, true>(tile, it);
    else mx_store<SH, false, false>(tile, it);
  }
}

// Sums of partial tiles, in ascending k.
__global__ __launch_bounds__(256) void mx_join_kernel(const MxJoin *__restrict__ joins, int blocks_per_join) {
  const MxJoin jn = joins[blockIdx.x / blocks_per_join];
  const int at = ((blockIdx.x % blocks_per_join) * 256 + threadIdx.x) * 4;
  const int row = at / jn.tn, col = at % jn.tn;
  if (row >= jn.m_ext || col >= jn.n_ext) return;
  const int64_t slot = (int64_t)jn.tm * jn.tn;
  const float *p = jn.parts + at;
  nt_f32x4 sum = *(const nt_f32x4 *)p;
  for (int r = 1; r < jn.runs; ++r) sum += *(const nt_f32x4 *)(p + r * slot);
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (col + x < jn.n_ext) {
      const int64_t o = (int64_t)row * jn.ldc + col + x;
      if (jn.c_es == 4) ((float *)jn.c)[o] = sum[x];
      else ((unsigned short *)jn.c)[o] = mx_bf16(sum[x]);
    }
}

// Up to 32 rows against little B, 16 a workgroup: every wave reads B straight into registers.  A workgroup owns 16 columns; its four waves
// take every fourth 512 elements of K each and add up through LDS, so that there are enough waves on the way to memory without partial
// sums in memory.  (Calls one after another, bf16: 1 x 4096 x 4096 5.7 us, tiles of 32 x 128 8.5; 1 x 16384 x 2048 9.8, those cut into eight 14.8.  125 MB
// of B that no cache holds at 4.5 TB/s with one row, 3.2 with 16, the tiles at 4.6.)
__global__ __launch_bounds__(NT_THREADS) void mx_skinny_kernel(const MxItem *__restrict__ items, const NtSeg *__restrict__ segs) {
  constexpr int Q = 4;                                        // chunks (128 of k) at a time
  __shared__ nt_f32x4 sums[4][64];
  const MxItem it = items[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  nt_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  int todo = it.steps, skip = it.first;
  for (int sg = 0; todo > 0; ++sg) {
    const NtSeg s = sg ? segs[it.seg + sg] : it.front;
    const int n = min(s.chunks - 2 * skip, 2 * todo);
    const int64_t row_a = it.m_off + min(r, it.m_ext - 1), row_b = it.n_off + min(r, it.n_ext - 1);
    const char *const pa = s.a + row_a * s.a_pitch + (int64_t)skip * NT_ROW + g * 16, *const sa = s.a_scale + row_a * s.a_scale_pitch + (int64_t)skip * 8;
    const char *const pb = s.b + row_b * s.b_pitch + (int64_t)skip * NT_ROW + g * 16, *const sb = s.b_scale + row_b * s.b_scale_pitch + (int64_t)skip * 8;
    auto multiply = [&](nt_i32x4 a, nt_i32x4 b, int as, int bs) {
      const nt_i32x8 x = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
      const nt_i32x8 y = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, (int)((unsigned)bs >> (8 * g)), 0, (int)((unsigned)as >> (8 * g)));
    };
    int t = wave * Q;
    for (; t + Q <= n; t += 4 * Q) {
      nt_i32x4 a[Q], b[Q], as, bs;
      __builtin_memcpy(&bs, sb + t * 4, 16);
#pragma unroll
      for (int q = 0; q < Q; ++q) b[q] = __builtin_nontemporal_load((const nt_i32x4 *)(pb + (t + q) * NT_CHUNK));
      __builtin_memcpy(&as, sa + t * 4, 16);
#pragma unroll
      for (int q = 0; q < Q; ++q) a[q] = *(const nt_i32x4 *)(pa + (t + q) * NT_CHUNK);
#pragma unroll
      for (int q = 0; q < Q; ++q) multiply(a[q], b[q], as[q], bs[q]);
    }
    // the last, incomplete 512 elements: one wave's t ends in front of them, the others' behind
    for (; t < n; ++t)
      multiply(*(const nt_i32x4 *)(pa + t * NT_CHUNK), *(const nt_i32x4 *)(pb + t * NT_CHUNK), *(const int *)(sa + t * 4), *(const int *)(sb + t * 4));
    todo -= (n + 1) >> 1;
    skip = 0;
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
  const nt_f32x4 v = ((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane];
  const int col = 4 * g;                                      // row r, columns 4 g ...
  if (r < it.m_ext) {
#pragma unroll
    for (int y = 0; y < 4; ++y)
      if (col + y < it.n_ext) {
        const int64_t at = (int64_t)r * it.ldc + col + y;
        if (it.c_es == 4) ((float *)it.c)[at] = v[y];
        else ((unsigned short *)it.c)[at] = mx_bf16(v[y]);
      }
  }
}

// ---- quantisation -----------------------------------------------------------------------------------

typedef unsigned short mx_u16x2 __attribute__((ext_vector_type(2)));

// Eight (2 N) neighbouring elements of a tile as they came: words of two bf16, or fp32.
template <bool F32>
struct MxVec {
  static constexpr int WORDS = F32 ? 8 : 4;
  unsigned w[WORDS];
};

// largest magnitude, as bits that compare like the values
__device__ __forceinline__ unsigned mx_abs_max(const MxVec<true> &v) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, v.w[i] & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ unsigned mx_abs_max(const MxVec<false> &v) {
  mx_u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(mx_u16x2, v.w[i] & 0x7fff7fffu));
  return (unsigned)max(m[0], m[1]) << 16;
}
// the scale's byte of a block whose largest magnitude has these bits
__device__ __forceinline__ unsigned mx_scale(unsigned amax) {
  const int e = (int)(amax >> 23);                            // 255: infinity or NaN; 0: below 2^-126
  return e == 255 ? 255u : (unsigned)max(e - 2, 0);
}
// eight codes.  The instruction takes the scale from the exponent's bits alone, so 2^-127 (all of them zero) needs no care, nor
// do elements below 2^-126; what it makes of a block without a scale counts for nothing.
__device__ __forceinline__ unsigned mx_codes(const MxVec<true> &v, unsigned scale) {
  const float s = __builtin_bit_cast(float, scale << 23);
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __builtin_bit_cast(float, v.w[0]), __builtin_bit_cast(float, v.w[1]), s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __builtin_bit_cast(float, v.w[2]), __builtin_bit_cast(float, v.w[3]), s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __builtin_bit_cast(float, v.w[4]), __builtin_bit_cast(float, v.w[5]), s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __builtin_bit_cast(float, v.w[6]), __builtin_bit_cast(float, v.w[7]), s, 3);
  return r;
}
__device__ __forceinline__ unsigned mx_codes(const MxVec<false> &v, unsigned scale) {
  const float s = __builtin_bit_cast(float, scale << 23);
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, v.w[0]), s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, v.w[1]), s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, v.w[2]), s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, v.w[3]), s, 3);
  return r;
}

// Eight elements of a row from column `col` on, zeros behind column w.  Rows may begin anywhere: the loads and stores of 16
// bytes take any address (element by element 4099 x 2731 fp32 took 29 us along the columns, and its values 32).
template <bool F32>
__device__ __forceinline__ MxVec<F32> mx_load8(const char *row, int col, int w) {
  MxVec<F32> v;
  if (col + 8 <= w) {
    __builtin_memcpy(v.w, row + (int64_t)col * (F32 ? 4 : 2), sizeof v.w);
  } else {
#pragma unroll
    for (int i = 0; i < MxVec<F32>::WORDS; ++i) {
      if constexpr (F32) {
        v.w[i] = col + i < w ? ((const unsigned *)row)[col + i] : 0u;
      } else {
        const unsigned lo = col + 2 * i < w ? ((const unsigned short *)row)[col + 2 * i] : 0u;
        const unsigned hi = col + 2 * i + 1 < w ? ((const unsigned short *)row)[col + 2 * i + 1] : 0u;
        v.w[i] = lo | hi << 16;
      }
    }
  }
  return v;
}

// the largest of four neighbouring lanes
__device__ __forceinline__ unsigned mx_max4(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // lane ^ 2
}

// the tile that workgroup `block` belongs to, and the workgroup's number inside it
__device__ __forceinline__ const MxTile &mx_find(const MxTileArgs &args, int block, int *inside) {
  int x = 0;
  while (x + 1 < args.n && block >= args.tile[x + 1].first_block) ++x;
  *inside = block - args.tile[x].first_block;
  return args.tile[x];
}

// Along the rows alone: a wave takes 512 columns of R rows, all loads first.
template <bool F32, int R>
__global__ __launch_bounds__(256) void mx_rows_kernel(MxTileArgs) {
  const auto &args = *(const MxTileArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const MxTile &T = mx_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63;
  const int unit = block * 4 + (threadIdx.x >> 6), across = T.blocks_across;   // 512-column pieces of a row
  const int col = (unit % across) * 512 + lane * 8, row0 = unit / across * R;
  const int wide_cols = (T.w + 127) & ~127;
  if (col >= wide_cols) return;
  MxVec<F32> v[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (row0 + i < T.h) v[i] = mx_load8<F32>((const char *)T.x + (int64_t)(row0 + i) * T.x_pitch, col, T.w);
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (row0 + i < T.h) {
      const unsigned scale = mx_scale(mx_max4(mx_abs_max(v[i])));
      *(unsigned *)(T.row_codes + (int64_t)(row0 + i) * T.row_pitch + col / 2) = mx_codes(v[i], scale);
      if ((lane & 3) == 0) T.row_scales[(int64_t)(row0 + i) * T.row_scale_pitch + col / 32] = (unsigned char)scale;
    }
}

// Along the columns, and along the rows too if ROWS: a workgroup takes 128 rows of 256 bytes, reads them along the rows and leaves
// them in LDS (33 KB: four workgroups on a CU), where each thread then finds its 32 rows of one or two columns.  Four threads
// make the 64 bytes of a column's 128 codes.
// 8192 x 8192 bf16 both ways: 54 us for 205 MB (3.8 TB/s; 4.6 is what a large copy makes).  A workgroup that goes on to other blocks
// and loads them ahead made 53, blocks ordered so that lines of codes and scales are completed in one L2 55.
template <bool F32>
struct MxBlock {
  static constexpr int ES = F32 ? 4 : 2, COLS = 256 / ES;     // 64 or 128 columns
  static constexpr int PITCH = 256 + 4;                       // bytes (one word more: rows start in other banks)
  static constexpr int LDS = 128 * PITCH + 3 * 64;
  // byte that a row starts at: 16 words further on every 32 rows, which four neighbouring threads have in hand at a time
  static __device__ __forceinline__ int at(int row) { return row * PITCH + (row >> 5) * 64; }
  static constexpr int ACROSS = COLS / 8, DOWN = 256 / ACROSS, PASSES = 128 / DOWN;   // threads to a row of a pass, rows of a pass
  static constexpr int OWN = COLS / 64;                       // columns of a thread
};
template <bool F32, bool ROWS>
__global__ __launch_bounds__(256) void mx_cols_kernel(MxTileArgs) {
  using B = MxBlock<F32>;
  __shared__ __attribute__((aligned(16))) char lds[B::LDS];
  const auto &args = *(const MxTileArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const MxTile &T = mx_find(args, blockIdx.x, &block);
  const int col0 = (block % T.blocks_across) * B::COLS, row0 = block / T.blocks_across * 128;
  const int tid = threadIdx.x;
  {
    const int col = col0 + tid % B::ACROSS * 8, r0 = tid / B::ACROSS;
    MxVec<F32> v[B::PASSES];
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x) {
      const int row = row0 + x * B::DOWN + r0;
      v[x] = row < T.h ? mx_load8<F32>((const char *)T.x + (int64_t)row * T.x_pitch, col, T.w) : MxVec<F32>{};
    }
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x) {
      const int r = x * B::DOWN + r0;
      unsigned *p = (unsigned *)(lds + B::at(r) + tid % B::ACROSS * 8 * B::ES);
#pragma unroll
      for (int i = 0; i < MxVec<F32>::WORDS; ++i) p[i] = v[x].w[i];
      if constexpr (ROWS) {
        const unsigned scale = mx_scale(mx_max4(mx_abs_max(v[x])));
        // (with 64 columns a block may lie behind the last chunk)
        if (row0 + r < T.h && col < ((T.w + 127) & ~127)) {
          *(unsigned *)(T.row_codes + (int64_t)(row0 + r) * T.row_pitch + col / 2) = mx_codes(v[x], scale);
          if ((tid & 3) == 0) T.row_scales[(int64_t)(row0 + r) * T.row_scale_pitch + col / 32] = (unsigned char)scale;
        }
      }
    }
  }
  __syncthreads();
  // thread: rows 32 b ..., its columns
  const int b = tid & 3, p = tid >> 2;
  unsigned words[B::OWN][F32 ? 32 : 16];                      // a column: 32 fp32, or 32 bf16 in pairs
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const char *q = lds + B::at(32 * b + i) + p * 4;
    const unsigned x = *(const unsigned *)q, y = *(const unsigned *)(q + B::PITCH);
    if constexpr (F32) {
      words[0][i] = x;
      words[0][i + 1] = y;
    } else {
      words[0][i / 2] = __builtin_amdgcn_perm(y, x, 0x05040100);   // low halves
      words[1][i / 2] = __builtin_amdgcn_perm(y, x, 0x07060302);   // high halves
    }
  }
#pragma unroll
  for (int c = 0; c < B::OWN; ++c) {
    const int col = col0 + B::OWN * p + c;
    MxVec<F32> v[4];
    unsigned amax = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int i = 0; i < MxVec<F32>::WORDS; ++i) v[k].w[i] = words[c][k * MxVec<F32>::WORDS + i];
      amax = max(amax, mx_abs_max(v[k]));
    }
    if (col < T.w) {
      const unsigned scale = mx_scale(amax);
      nt_i32x4 codes;
#pragma unroll
      for (int k = 0; k < 4; ++k) codes[k] = (int)mx_codes(v[k], scale);
      *(nt_i32x4 *)(T.col_codes + (int64_t)col * T.col_pitch + (row0 / 32 + b) * 16) = codes;
      T.col_scales[(int64_t)col * T.col_scale_pitch + row0 / 32 + b] = (unsigned char)scale;
    }
  }
}

// ---- values -------------------------------------------------------------------------------------------

// Eight values of a block as they are stored in the tile.
template <bool F32>
__device__ __forceinline__ MxVec<F32> mx_values(unsigned codes, unsigned scale) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const int e = (int)scale - 127;
  float f[8];
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 1);
  const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, 3);
  f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1], f[4] = c[0], f[5] = c[1], f[6] = d[0], f[7] = d[1];
  MxVec<F32> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // (bf16 holds every such value: two significant bits, 2^-128 at least)
    const unsigned bits = scale == 255u ? 0x7fc00000u : __builtin_bit_cast(unsigned, ldexpf(f[i], e));
    if constexpr (F32) v.w[i] = bits;
    else if (i & 1) v.w[i / 2] |= bits & 0xffff0000u;
    else v.w[i / 2] = bits >> 16;
  }
  return v;
}
template <bool F32>
__device__ __forceinline__ void mx_store8(char *row, int col, int w, const MxVec<F32> &v) {
  if (col + 8 <= w) {
    __builtin_memcpy(row + (int64_t)col * (F32 ? 4 : 2), v.w, sizeof v.w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < w) {
        if constexpr (F32) ((unsigned *)row)[col + i] = v.w[i];
        else ((unsigned short *)row)[col + i] = (unsigned short)(v.w[i / 2] >> (16 * (i & 1)));
      }
  }
}

template <bool F32, int R>
__global__ __launch_bounds__(256) void mx_row_values_kernel(MxTileArgs) {
  const auto &args = *(const MxTileArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const MxTile &T = mx_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63;
  const int unit = block * 4 + (threadIdx.x >> 6), across = T.blocks_across;
  const int col = (unit % across) * 512 + lane * 8, row0 = unit / across * R;
  if (col >= T.w) return;
  unsigned codes[R], scale[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (row0 + i < T.h) {
      codes[i] = *(const unsigned *)(T.row_codes + (int64_t)(row0 + i) * T.row_pitch + col / 2);
      scale[i] = T.row_scales[(int64_t)(row0 + i) * T.row_scale_pitch + col / 32];
    }
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (row0 + i < T.h) mx_store8<F32>((char *)T.x + (int64_t)(row0 + i) * T.x_pitch, col, T.w, mx_values<F32>(codes[i], scale[i]));
}

// 128 rows of 64 or 128 columns, turned through LDS the other way.
template <bool F32>
__global__ __launch_bounds__(256) void mx_col_values_kernel(MxTileArgs) {
  using B = MxBlock<F32>;
  __shared__ __attribute__((aligned(16))) char lds[B::LDS];
  const auto &args = *(const MxTileArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const MxTile &T = mx_find(args, blockIdx.x, &block);
  const int col0 = (block % T.blocks_across) * B::COLS, row0 = block / T.blocks_across * 128;
  const int tid = threadIdx.x, b = tid & 3, p = tid >> 2;
  nt_i32x4 codes[B::OWN];
  unsigned scale[B::OWN];
#pragma unroll
  for (int c = 0; c < B::OWN; ++c) {
    const int col = min(col0 + B::OWN * p + c, T.w - 1);
    codes[c] = *(const nt_i32x4 *)(T.col_codes + (int64_t)col * T.col_pitch + (row0 / 32 + b) * 16);
    scale[c] = T.col_scales[(int64_t)col * T.col_scale_pitch + row0 / 32 + b];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const MxVec<F32> x = mx_values<F32>((unsigned)codes[0][k], scale[0]), y = mx_values<F32>((unsigned)codes[B::OWN - 1][k], scale[B::OWN - 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned *const q = (unsigned *)(lds + B::at(32 * b + 8 * k + i) + p * 4);
      if constexpr (F32) *q = x.w[i];
      else *q = __builtin_amdgcn_perm(y.w[i / 2], x.w[i / 2], i & 1 ? 0x07060302 : 0x05040100);
    }
  }
  __syncthreads();
  const int col = col0 + tid % B::ACROSS * 8, r0 = tid / B::ACROSS;
#pragma unroll
  for (int pass = 0; pass < B::PASSES; ++pass) {
    const int r = pass * B::DOWN + r0;
    if (row0 + r >= T.h) continue;
    MxVec<F32> v;
    const unsigned *q = (const unsigned *)(lds + B::at(r) + tid % B::ACROSS * 8 * B::ES);
#pragma unroll
    for (int i = 0; i < MxVec<F32>::WORDS; ++i) v.w[i] = q[i];
    mx_store8<F32>((char *)T.x + (int64_t)(row0 + r) * T.x_pitch, col, T.w, v);
  }
}

}  // namespace dmm
