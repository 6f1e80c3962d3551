// What the layers around a product do element by element (gfx950, device code only): the gated block's slopes, and
// matrices to 8-bit integers and back.
#pragma once

#include "layer_kernel.hpp"

namespace dmm {

// The last of `n` entries that does not begin behind workgroup `block`: 64 of them are looked at together (one after the other each costs the
// workgroup a read that it waits for).
template <class Entry>
__device__ __forceinline__ int layer_last(const Entry *entries, int n, int block) {
  int count = 0;
  for (int x = 0; x < n; x += 64) {
    const int i = x + (int)(threadIdx.x & 63);
    const int mine = __builtin_popcountll(__ballot(i < n && entries[min(i, n - 1)].first_block <= block));
    count += mine;
    if (mine < 64) break;
  }
  return __builtin_amdgcn_readfirstlane(count) - 1;
}
// the tile that workgroup `block` belongs to, and the workgroup's number inside it
template <class Args>
__device__ __forceinline__ const auto &layer_find(const Args &args, int block, int *inside) {
  const int x = layer_last(args.tile, args.n, block);
  *inside = block - args.tile[x].first_block;
  return args.tile[x];
}

// Eight neighbouring elements of a row from column `col` on, zeros behind column w; rows may begin anywhere.  (Where others write elements in front of
// `col` at the same time, what is read of them counts for nothing.)
template <bool F32>
struct LayerVec {
  static constexpr int WORDS = F32 ? 8 : 4;
  unsigned w[WORDS];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (F32) return __builtin_bit_cast(float, w[i]);
    else return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(int i, float v) {
    if constexpr (F32) {
      w[i] = __builtin_bit_cast(unsigned, v);
    } else {
      const unsigned b = layer_bf16(v);
      w[i / 2] = i & 1 ? w[i / 2] | b << 16 : b;              // (in ascending order)
    }
  }
};
template <bool F32>
__device__ __forceinline__ LayerVec<F32> layer_load8(const char *row, int col, int w) {
  LayerVec<F32> v;
  if (col + 8 <= w) {
    __builtin_memcpy(v.w, row + (int64_t)col * (F32 ? 4 : 2), sizeof v.w);
  } else if (!F32 && w >= 8) {
    // the row's last eight, moved to the front (one by one they keep the wave waiting eight times, and almost every wave meets a row's end)
    unsigned __int128 all;
    __builtin_memcpy(&all, row + (int64_t)(w - 8) * 2, 16);
    const int back = min(col + 8 - w, 8);
    all = back < 8 ? all >> (16 * back) : 0;
    __builtin_memcpy(v.w, &all, sizeof v.w);
  } else {
#pragma unroll
    for (int i = 0; i < LayerVec<F32>::WORDS; ++i) {
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
template <bool F32>
__device__ __forceinline__ void layer_store8(char *row, int col, int w, const LayerVec<F32> &v) {
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

// Tiles whose rows are misaligned or finely cut, into dense rows: 16 bytes a thread at a time, eight of them on their way together.  The last 16 bytes
// of a row are moved as such, over some of those in front of them: a part of 16 bytes would be moved one by one, and every wave meets one.
// Bound: HBM or the caches (21 MB of integers in 15 uneven blocks 10.2 us with the launch, 4.1 TB/s read and written).
__global__ __launch_bounds__(256) void layer_copy_kernel(const LayerCopy *__restrict__ jobs, int n) {
  const LayerCopy j = jobs[layer_last(jobs, n, (int)blockIdx.x)];
  const unsigned across = (unsigned)(j.bytes + 15) / 16;      // chunks of a row
  const uint64_t all = (uint64_t)across * (unsigned)j.rows, first = (uint64_t)((int)blockIdx.x - j.first_block) * LAYER_COPY_CHUNKS;
  constexpr int N = LAYER_COPY_CHUNKS / 256;
  const unsigned row0 = (unsigned)(first / across), col0 = (unsigned)(first % across);
  typedef __attribute__((address_space(1))) char *gptr;
  typedef const __attribute__((address_space(1))) char *cgptr;
  if (j.bytes < 16) {
    for (int i = 0; i < N; ++i) {
      const uint64_t row = first + i * 256 + threadIdx.x;     // (one chunk a row)
      if (row >= all) break;
      for (int b = 0; b < j.bytes; ++b) ((gptr)j.dst)[(int64_t)row * j.dst_pitch + b] = j.src ? ((cgptr)j.src)[(int64_t)row * j.src_pitch + b] : 0;
    }
    return;
  }
  nt_i32x4 v[N];
  gptr to[N];
  bool mine[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const unsigned on = col0 + i * 256 + threadIdx.x, row = row0 + on / across, at = min(on % across * 16, (unsigned)j.bytes - 16);
    mine[i] = first + i * 256 + threadIdx.x < all;
    to[i] = (gptr)j.dst + ((int64_t)row * j.dst_pitch + at);
    v[i] = nt_i32x4{0, 0, 0, 0};
    if (j.src && mine[i]) __builtin_memcpy(&v[i], (cgptr)j.src + ((int64_t)row * j.src_pitch + at), 16);
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (mine[i]) __builtin_memcpy(to[i], &v[i], 16);
}

// dU = dH act(G), dG = dH U act'(G): a thread has four pieces of eight neighbouring elements, whatever rows they are of.  Every element is read and written
// by one thread, in this order, so dG and dU may be G and U themselves.  Bound: HBM (4096 x 8192: 335 MB in 62 us, 5.4 TB/s; 2501 x 1777 in 15 uneven blocks,
// 44 MB with rows at any address, 17.7).
__global__ __launch_bounds__(256) void layer_slope_kernel(SlopeArgs) {
  const auto &args = *(const SlopeArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int N = SLOPE_CHUNKS / 256;
  int block;
  const SlopeTile &T = layer_find(args, blockIdx.x, &block);
  const unsigned across = (unsigned)(T.w + 7) / 8;
  const uint64_t first = (uint64_t)block * SLOPE_CHUNKS;
  const unsigned row0 = (unsigned)(first / across), col0 = (unsigned)(first % across);
  LayerVec<false> g[N], u[N], h[N];
  int row[N], col[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const unsigned on = col0 + i * 256 + threadIdx.x;
    row[i] = (int)(row0 + on / across);
    col[i] = (int)(on % across) * 8;
    if (row[i] < T.h) {
      g[i] = layer_load8<false>(T.g + row[i] * T.pg, col[i], T.w);
      u[i] = layer_load8<false>(T.u + row[i] * T.pu, col[i], T.w);
      h[i] = layer_load8<false>(T.dh + row[i] * T.ph, col[i], T.w);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (row[i] < T.h) {
      LayerVec<false> dg, du;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        float value, slope;
        layer_slope(args.act, g[i].at(x), &value, &slope);
        const float dh = h[i].at(x);
        dg.set(x, dh * u[i].at(x) * slope);
        du.set(x, dh * value);
      }
      layer_store8<false>(T.dg + row[i] * T.pdg, col[i], T.w, dg);
      layer_store8<false>(T.du + row[i] * T.pdu, col[i], T.w, du);
    }
}

// ---- 8-bit integers -------------------------------------------------------------------------------------
//
// A row's (column's) scale is its largest magnitude over 127, rounded to fp32; an element is the integer nearest to 127 x / (largest
// magnitude), both taken exactly, half-way values to the even one.  A row with an infinity or a NaN has the scale NaN.
//
// Bound: HBM.  A row's scale is known only when all of it has been read; along the rows a workgroup keeps what it has read in registers, along the columns the
// matrix is read twice (4099 x 11003 fp32 in uneven blocks: magnitudes 47 us, 3.8 TB/s; integers 46, 4.9; values back 56, 4.0; scales cleared and finished
// 4.8 each).

// bits of |x|, which compare like the values (NaN above infinity)
template <bool F32>
__device__ __forceinline__ unsigned i8_abs_max(const LayerVec<F32> &v, unsigned m) {
#pragma unroll
  for (int i = 0; i < LayerVec<F32>::WORDS; ++i) {
    if constexpr (F32) m = max(m, v.w[i] & 0x7fffffffu);
    else m = max(m, max(v.w[i] << 16 & 0x7fffffffu, v.w[i] & 0x7fff0000u));
  }
  return m;
}

// What turns elements of a row into integers: |x| and the largest magnitude are brought to [1, 2) by a power of two, so that nothing leaves the
// range of fp32 on the way.
struct I8Row {
  float top, over;              // the largest magnitude in [1, 2); 127 / top
  int e;
  unsigned bits;
};
__device__ __forceinline__ I8Row i8_row(unsigned bits) {
  I8Row r;
  r.bits = bits;
  const float v = __builtin_bit_cast(float, bits);
  r.e = 1 - __builtin_amdgcn_frexp_expf(v);
  r.top = bits ? __builtin_amdgcn_ldexpf(v, r.e) : 1.f;
  r.over = 127.f / r.top;
  if (bits == 0 || bits >= 0x7f800000u) r.over = 0.f, r.e = 0;
  return r;
}
__device__ __forceinline__ float i8_scale(unsigned bits) {
  return bits >= 0x7f800000u ? __builtin_bit_cast(float, 0x7fc00000u) : __builtin_bit_cast(float, bits) / 127.f;
}
// x (127 / top) is off by less than 2^-16; where that could matter the exact products decide (they fit 53 bits).
__device__ __forceinline__ int i8_code(const I8Row &r, float x) {
  if (r.bits >= 0x7f800000u) return 0;
  const float y = __builtin_amdgcn_ldexpf(x, r.e), q = y * r.over;
  float t = __builtin_rintf(q);
  const float off = q - t;
  if (__builtin_fabsf(__builtin_fabsf(off) - 0.5f) < 0x1p-14f) {
    const float low = off < 0.f ? t - 1.f : t;                // the integer below
    const double twice = 254.0 * (double)y, border = (2.0 * (double)low + 1.0) * (double)r.top;
    const bool odd = ((int)low & 1) != 0;
    t = twice > border || (twice == border && odd) ? low + 1.f : low;
  }
  return (int)t;
}
__device__ __forceinline__ unsigned i8_four(const I8Row &r, float a, float b, float c, float d) {
  return (unsigned)(i8_code(r, a) & 255) | (unsigned)(i8_code(r, b) & 255) << 8 | (unsigned)(i8_code(r, c) & 255) << 16 | (unsigned)i8_code(r, d) << 24;
}
// `n` of the bytes of N words, to any address
template <int N>
__device__ __forceinline__ void i8_put(char *p, const unsigned *w, int n) {
  if (n >= 4 * N) {
    __builtin_memcpy(p, w, 4 * N);
  } else {
#pragma unroll
    for (int i = 0; i < 4 * N; ++i)
      if (i < n) p[i] = (char)(w[i / 4] >> (8 * (i & 3)));
  }
}
// Eight integers of a row from column `col` on, zeros behind column w (a row's end as in layer_load8).
__device__ __forceinline__ void i8_load8(const char *row, int col, int w, unsigned out[2]) {
  uint64_t all = 0;
  if (col + 8 <= w) {
    __builtin_memcpy(&all, row + col, 8);
  } else if (w >= 8) {
    const int back = min(col + 8 - w, 8);
    __builtin_memcpy(&all, row + w - 8, 8);
    all = back < 8 ? all >> (8 * back) : 0;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < w) all |= (uint64_t)*(const unsigned char *)(row + col + i) << (8 * i);
  }
  out[0] = (unsigned)all;
  out[1] = (unsigned)(all >> 32);
}
template <int N>
__device__ __forceinline__ void i8_get(const char *p, unsigned *w, int n) {
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = 0;
  if (n >= 4 * N) {
    __builtin_memcpy(w, p, 4 * N);
  } else {
#pragma unroll
    for (int i = 0; i < 4 * N; ++i)
      if (i < n) w[i / 4] |= (unsigned)*(const unsigned char *)(p + i) << (8 * (i & 3));
  }
}

__device__ __forceinline__ unsigned i8_wave_max(unsigned v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}

__global__ __launch_bounds__(256) void i8_scales_kernel(I8ScaleArgs, int what) {
  const auto &args = *(const I8ScaleArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  const int x = layer_last(args.piece, args.n, (int)blockIdx.x);
  const int i = ((int)blockIdx.x - args.piece[x].first_block) * 256 + threadIdx.x;
  if (i >= args.piece[x].n) return;
  float *const at = args.piece[x].at + i;
  *at = what == I8_CLEAR ? 0.f : i8_scale(__builtin_bit_cast(unsigned, *at));
}

// A workgroup's place in a tile.  Neighbours share lines, of the matrix where rows are not aligned and of the integers along the columns, so every XCD (workgroup
// w runs on XCD w % 8) has a run of the blocks, four side by side and then down the tile.  (`all` workgroups in the launch.)
struct I8Place {
  int row0, col0;
};
__device__ __forceinline__ int i8_in_order(int all) {
  const int xcd = (int)blockIdx.x % 8, each = all / 8, more = all % 8;
  return xcd * each + min(xcd, more) + (int)blockIdx.x / 8;
}
template <int ROWS, int COLS>
__device__ __forceinline__ I8Place i8_place(const I8Tile &T, int block) {
  const int down = (T.h + ROWS - 1) / ROWS, strip = block / (4 * down), in = block % (4 * down);
  const int wide = min(4, T.blocks_across - 4 * strip);
  return {in / wide * ROWS, (4 * strip + in % wide) * COLS};
}

// A workgroup's 128 rows of 64 (128) columns: threads to a row of a pass, rows of a pass.
template <bool F32>
struct I8Block {
  static constexpr int ES = F32 ? 4 : 2, COLS = i8_block_cols(F32), ACROSS = COLS / 8, DOWN = 256 / ACROSS, PASSES = 128 / DOWN;
  static constexpr int PITCH = 256 + 4;                       // bytes of a row in LDS (one word more: rows start in other banks)
};

// Largest magnitudes of rows or columns so far, as bits, in the scales' place.  (The largest of integers does not depend on the order of the atomics.)
template <bool F32, bool ALONG_COLS>
__global__ __launch_bounds__(256) void i8_amax_kernel(I8Args) {
  using B = I8Block<F32>;
  __shared__ unsigned tops[128];
  const auto &args = *(const I8Args *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const I8Tile &T = layer_find(args, i8_in_order(gridDim.x), &block);
  const I8Place place0 = i8_place<128, B::COLS>(T, block);
  const int col0 = place0.col0, row0 = place0.row0;
  const int tid = threadIdx.x, col = col0 + tid % B::ACROSS * 8, r0 = tid / B::ACROSS;
  LayerVec<F32> v[B::PASSES];
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int row = row0 + x * B::DOWN + r0;
    v[x] = row < T.h ? layer_load8<F32>(T.x + (int64_t)row * T.x_pitch, col, T.w) : LayerVec<F32>{};
  }
  if (tid < 128) tops[tid] = 0;
  __syncthreads();
  if constexpr (ALONG_COLS) {
    unsigned m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x)
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = max(m[i], __builtin_bit_cast(unsigned, v[x].at(i)) & 0x7fffffffu);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int d = B::ACROSS; d < 64; d *= 2) m[i] = max(m[i], (unsigned)__shfl_xor((int)m[i], d));
      if ((tid & 63) < B::ACROSS) atomicMax(&tops[tid % B::ACROSS * 8 + i], m[i]);
    }
    __syncthreads();
    if (tid < B::COLS && col0 + tid < T.w) atomicMax((unsigned *)T.scale + col0 + tid, tops[tid]);
  } else {
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x) {
      unsigned m = i8_abs_max(v[x], 0);
#pragma unroll
      for (int d = 1; d < B::ACROSS; d *= 2) m = max(m, (unsigned)__shfl_xor((int)m, d));
      if (tid % B::ACROSS == 0) tops[x * B::DOWN + r0] = m;
    }
    __syncthreads();
    if (tid < 128 && row0 + tid < T.h) atomicMax((unsigned *)T.scale + row0 + tid, tops[tid]);
  }
}

// Integers along the rows: the same blocks, eight bytes a thread and row.
template <bool F32>
__global__ __launch_bounds__(256) void i8_rows_kernel(I8Args) {
  using B = I8Block<F32>;
  const auto &args = *(const I8Args *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const I8Tile &T = layer_find(args, i8_in_order(gridDim.x), &block);
  const I8Place place0 = i8_place<128, B::COLS>(T, block);
  const int col0 = place0.col0, row0 = place0.row0;
  const int col = col0 + threadIdx.x % B::ACROSS * 8, r0 = threadIdx.x / B::ACROSS;
  if (col >= T.w) return;
  LayerVec<F32> v[B::PASSES];
  unsigned top[B::PASSES];
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int row = min(row0 + x * B::DOWN + r0, T.h - 1);    // (rows past the last read that one again: loads that wait for no branch)
    v[x] = layer_load8<F32>(T.x + (int64_t)row * T.x_pitch, col, T.w);
    top[x] = ((const unsigned *)T.scale)[row];
  }
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int row = row0 + x * B::DOWN + r0;
    if (row >= T.h) break;
    const I8Row r = i8_row(top[x]);
    const unsigned w[2] = {i8_four(r, v[x].at(0), v[x].at(1), v[x].at(2), v[x].at(3)), i8_four(r, v[x].at(4), v[x].at(5), v[x].at(6), v[x].at(7))};
    i8_put<2>(T.q + (int64_t)row * T.q_pitch + col, w, T.w - col);
  }
}

// Integers along the columns: the block is left in LDS, where every thread finds 32 rows of one or two columns.  ALL: a block has all rows of its columns, and
// finds their largest magnitudes there as well (one launch for four: 16 x 8192, and back, bf16 23 us and 15, fp32 20 and 9.6).
template <bool F32, bool ALL>
__global__ __launch_bounds__(256) void i8_cols_kernel(I8Args) {
  using B = I8Block<F32>;
  __shared__ __attribute__((aligned(16))) char lds[128 * B::PITCH + 3 * 64];
  auto place = [](int row) { return row * B::PITCH + (row >> 5) * 64; };   // (16 words on every 32 rows: four threads read these side by side)
  const auto &args = *(const I8Args *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const I8Tile &T = layer_find(args, i8_in_order(gridDim.x), &block);
  const I8Place place0 = i8_place<128, B::COLS>(T, block);
  const int col0 = place0.col0, row0 = place0.row0;
  const int tid = threadIdx.x;
  {
    const int col = col0 + tid % B::ACROSS * 8, r0 = tid / B::ACROSS;
    LayerVec<F32> v[B::PASSES];
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x) {
      const int row = row0 + x * B::DOWN + r0;
      v[x] = row < T.h ? layer_load8<F32>(T.x + (int64_t)row * T.x_pitch, col, T.w) : LayerVec<F32>{};
    }
#pragma unroll
    for (int x = 0; x < B::PASSES; ++x) {
      unsigned *p = (unsigned *)(lds + place(x * B::DOWN + r0) + tid % B::ACROSS * 8 * B::ES);
#pragma unroll
      for (int i = 0; i < LayerVec<F32>::WORDS; ++i) p[i] = v[x].w[i];
    }
  }
  __syncthreads();
  const int b = tid & 3, p = tid >> 2;                        // rows 32 b ..., a word of each row
  constexpr int OWN = F32 ? 1 : 2;
  I8Row r[OWN];
#pragma unroll
  for (int c = 0; c < OWN; ++c) {
    const int col = col0 + OWN * p + c;
    if constexpr (ALL) {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const unsigned w = *(const unsigned *)(lds + place(32 * b + i) + p * 4);
        m = max(m, (F32 ? w : c ? w & 0xffff0000u : w << 16) & 0x7fffffffu);
      }
      m = max(m, (unsigned)__shfl_xor((int)m, 1));
      m = max(m, (unsigned)__shfl_xor((int)m, 2));
      if (b == 0 && col < T.w) T.scale[col] = i8_scale(m);
      r[c] = i8_row(m);
    } else {
      r[c] = i8_row(col < T.w ? ((const unsigned *)T.scale)[col] : 0u);
    }
  }
  unsigned out[OWN][8];
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    unsigned w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) w[y] = *(const unsigned *)(lds + place(32 * b + i + y) + p * 4);
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      float f[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) f[y] = __builtin_bit_cast(float, F32 ? w[y] : c ? w[y] & 0xffff0000u : w[y] << 16);
      out[c][i / 4] = i8_four(r[c], f[0], f[1], f[2], f[3]);
    }
  }
  const int row = row0 + 32 * b;
#pragma unroll
  for (int c = 0; c < OWN; ++c) {
    const int col = col0 + OWN * p + c;
    if (col < T.w && row < T.h) i8_put<8>(T.q + (int64_t)col * T.q_pitch + row, out[c], T.h - row);
  }
}

// Rows over all tiles that they are cut into, a workgroup each, scales and integers.  The vectors of eight elements of all tiles are counted through, so that every thread has
// its own on their way at once whatever the tiles' widths, and the first I8_ROW_KEPT of each thread stay in registers between the two passes over a row.  (16
// rows of 8192: 256 threads with four vectors each 7 us, 1024 threads 4.3; 115 x 715 in eight tiles, and back, 22 us
// one tile after the other, now 11.  4096 x 8192, and back: 36 us with 256 threads and four vectors each, 50 with 1024 and one.)
// CUT: several tiles side by side, MANY: several rows of tiles (without, there is no search, and the one tile's numbers stay in scalar registers).
template <bool F32, bool CUT, bool MANY>
__global__ __launch_bounds__(I8_ROW_THREADS) void i8_whole_rows_kernel(I8RowArgs) {
  __shared__ unsigned tops[I8_ROW_THREADS / 64];
  __shared__ int firsts[I8_ROW_CUTS];
  const auto &args = *(const I8RowArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  const I8RowGroup &group = args.group[MANY ? layer_last(args.group, args.groups, (int)blockIdx.x) : 0];
  const I8RowPiece *const pieces = args.piece + (MANY ? group.first_piece : 0);
  const int row = (int)blockIdx.x - (MANY ? group.first_block : 0), tid = threadIdx.x, threads = blockDim.x;
  if constexpr (CUT) {
    if (tid < args.n) firsts[tid] = pieces[tid].first;
    __syncthreads();
  }
  // the tile of vector `at`
  auto piece_of = [&](int at) -> const I8RowPiece & {
    if constexpr (!CUT) return pieces[0];
    int lo = 0, hi = args.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (firsts[mid] <= at) lo = mid;
      else hi = mid - 1;
    }
    return pieces[lo];
  };
  auto load = [&](int at) {
    const I8RowPiece &P = piece_of(at);
    return layer_load8<F32>(P.x + (int64_t)row * P.x_pitch, (at - P.first) * 8, P.w);
  };
  LayerVec<F32> kept[I8_ROW_KEPT];
#pragma unroll
  for (int y = 0; y < I8_ROW_KEPT; ++y) {
    kept[y] = LayerVec<F32>{};
    if (y * threads + tid < args.vectors) kept[y] = load(y * threads + tid);
  }
  unsigned m = 0;
#pragma unroll
  for (int y = 0; y < I8_ROW_KEPT; ++y) m = i8_abs_max(kept[y], m);
  for (int64_t at = I8_ROW_KEPT * threads + tid; at < args.vectors; at += threads) m = i8_abs_max(load((int)at), m);
  m = i8_wave_max(m);
  if ((tid & 63) == 0) tops[tid >> 6] = m;
  __syncthreads();
  m = 0;
  for (int x = 0; x < threads / 64; ++x) m = max(m, tops[x]);
  if (tid == 0) group.scale[row] = i8_scale(m);
  const I8Row r = i8_row(m);
  auto codes = [&](int at, const LayerVec<F32> &v) {
    const I8RowPiece &P = piece_of(at);
    const int col = (at - P.first) * 8;
    const unsigned w[2] = {i8_four(r, v.at(0), v.at(1), v.at(2), v.at(3)), i8_four(r, v.at(4), v.at(5), v.at(6), v.at(7))};
    i8_put<2>(P.q + (int64_t)row * P.q_pitch + col, w, P.w - col);
  };
#pragma unroll
  for (int y = 0; y < I8_ROW_KEPT; ++y)
    if (y * threads + tid < args.vectors) codes(y * threads + tid, kept[y]);
  for (int64_t at = I8_ROW_KEPT * threads + tid; at < args.vectors; at += threads) codes((int)at, load((int)at));
}

// Values, integer times scale, along the rows.
template <bool F32>
__global__ __launch_bounds__(256) void i8_row_values_kernel(I8Args) {
  using B = I8Block<F32>;
  const auto &args = *(const I8Args *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const I8Tile &T = layer_find(args, i8_in_order(gridDim.x), &block);
  const I8Place place0 = i8_place<128, B::COLS>(T, block);
  const int col = place0.col0 + threadIdx.x % B::ACROSS * 8, row0 = place0.row0 + threadIdx.x / B::ACROSS;
  if (col >= T.w) return;
  unsigned w[B::PASSES][2];
  float s[B::PASSES];
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int row = min(row0 + x * B::DOWN, T.h - 1);
    i8_load8(T.q + (int64_t)row * T.q_pitch, col, T.w, w[x]);
    s[x] = T.scale[row];
  }
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int row = row0 + x * B::DOWN;
    if (row >= T.h) break;
    LayerVec<F32> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.set(i, (float)(signed char)(w[x][i / 4] >> (8 * (i & 3))) * s[x]);
    layer_store8<F32>(T.x + (int64_t)row * T.x_pitch, col, T.w, v);
  }
}

// ... along the columns, turned through LDS the other way.
template <bool F32>
__global__ __launch_bounds__(256) void i8_col_values_kernel(I8Args) {
  using B = I8Block<F32>;
  __shared__ __attribute__((aligned(16))) char lds[128 * B::PITCH + 3 * 64];
  auto place = [](int row) { return row * B::PITCH + (row >> 5) * 64; };
  const auto &args = *(const I8Args *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const I8Tile &T = layer_find(args, i8_in_order(gridDim.x), &block);
  const I8Place place0 = i8_place<128, B::COLS>(T, block);
  const int col0 = place0.col0, row0 = place0.row0;
  const int tid = threadIdx.x, b = tid & 3, p = tid >> 2;
  constexpr int OWN = F32 ? 1 : 2;
  unsigned w[OWN][8];
  float s[OWN];
#pragma unroll
  for (int c = 0; c < OWN; ++c) {
    const int col = col0 + OWN * p + c, row = row0 + 32 * b;
    i8_get<8>(T.q + (int64_t)col * T.q_pitch + row, w[c], col < T.w ? T.h - row : 0);
    s[c] = col < T.w ? T.scale[col] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    float f[OWN];
#pragma unroll
    for (int c = 0; c < OWN; ++c) f[c] = (float)(signed char)(w[c][i / 4] >> (8 * (i & 3))) * s[c];
    *(unsigned *)(lds + place(32 * b + i) + p * 4) =
        F32 ? __builtin_bit_cast(unsigned, f[0]) : (unsigned)layer_bf16(f[0]) | (unsigned)layer_bf16(f[OWN - 1]) << 16;
  }
  __syncthreads();
  const int col = col0 + tid % B::ACROSS * 8, r0 = tid / B::ACROSS;
  if (col >= T.w) return;
#pragma unroll
  for (int x = 0; x < B::PASSES; ++x) {
    const int r = x * B::DOWN + r0;
    if (row0 + r >= T.h) continue;
    LayerVec<F32> v;
    const unsigned *const q = (const unsigned *)(lds + place(r) + tid % B::ACROSS * 8 * B::ES);
#pragma unroll
    for (int i = 0; i < LayerVec<F32>::WORDS; ++i) v.w[i] = q[i];
    layer_store8<F32>(T.x + (int64_t)(row0 + r) * T.x_pitch, col, T.w, v);
  }
}

}  // namespace dmm
