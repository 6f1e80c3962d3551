// Newton-Schulz steps that bring the singular values of a matrix near 1 (gfx950, device code only):
//   X_0 = G / |G|,   S = X X^T,   X <- a X + (b S + c S S) X
// with X the matrix or its transpose, whichever has fewer rows.
//
// Every matrix is kept as pairs of fp16, v 2^12 = high + low with low the rounded rest: 22 bits of a value, and
// a product of two is low high + high low + high high, three matrix instructions (what is left out is 2^-22 of it).  Singular
// values far below the largest grow by 3.4 each step, and so do errors: rounded to bf16 once per step a matrix with a few
// strong directions comes out 28 % off (512 x 512, rank 16 over 1 % of noise), in fp16 4 %, in pairs 7e-6, in plain fp32 2e-5.
// The factor 2^12: no value reaches 16 (|X| <= 1.2 and |b S + c S S| < 5 in every element, checked by the host for the coefficients
// given), and the low part of one of 2^-13, the size of an element of a normalised 8192 x 8192 matrix, still is
// a multiple of 2^-24 / 2^12.
#pragma once

#include "nt_kernel.hpp"
#include "ortho_launch.hpp"

namespace dmm {

constexpr float ORTHO_SCALE = 4096.f;

struct OrthoPair {
  _Float16 high, low;
};
// where the high part of an element lies in a matrix of `pitch` elements a row; the low part is 64 bytes on
__device__ __forceinline__ int64_t ortho_at(int row, int col, unsigned pitch) {
  return (int64_t)row * (pitch * 4u) + (col >> 5) * 128 + (col & 31) * 2;
}
__device__ __forceinline__ OrthoPair ortho_split(float v) {
  OrthoPair p;
  p.high = (_Float16)v;
  p.low = (_Float16)(v - (float)p.high);
  return p;
}

__device__ __forceinline__ const OrthoTile &ortho_find(const OrthoTiles &args, int block, int *inside) {
  int x = 0;
  while (x + 1 < args.n && block >= args.tile[x + 1].first_block) ++x;
  *inside = block - args.tile[x].first_block;
  return args.tile[x];
}
__device__ __forceinline__ float ortho_load(const char *p, bool f32, int64_t i) {
  return f32 ? ((const float *)p)[i] : __builtin_bit_cast(float, (unsigned)((const unsigned short *)p)[i] << 16);
}

// Sums of squares, in 64 bits (an fp32 square may not have a place in fp32), added up in a fixed order: every workgroup has a
// place of its own among its matrix' sums, and takes 64 x 64 elements of its tile at a time.  16 loads of a wave on the way.
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoTiles) {
  __shared__ double part[4];
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pieces_c = (T.w + 63) >> 6, pieces = ((T.h + 63) >> 6) * pieces_c;
  const bool f32 = args.f32;
  double sum = 0.0;
  for (int p = block; p < pieces; p += T.across) {
    const int col = min((p % pieces_c) * 64 + lane, T.w - 1), row0 = p / pieces_c * 64 + wave * 16;
    const bool in = (p % pieces_c) * 64 + lane < T.w;
    float v[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = ortho_load(T.p + (int64_t)min(row0 + r, T.h - 1) * T.pitch, f32, col);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (in && row0 + r < T.h) sum += (double)v[r] * (double)v[r];
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) args.sums[(int64_t)T.matrix * args.sums_of_launch + T.pad + block] = ((part[0] + part[1]) + part[2]) + part[3];
}

// 1 / |G|; 0 for a matrix of zeros, NaN where an element is no finite number
__device__ __forceinline__ double ortho_inverse_norm(const double *sums, int n) {
  double s = 0.0;
  for (int i = threadIdx.x & 63; i < n; i += 64) s += sums[i];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if (!(s <= 1.7976931348623157e308)) return __builtin_nan("");
  return s > 0.0 ? 1.0 / sqrt(s) : 0.0;
}

// G / |G| as pairs, by rows and by columns: 64 x 64 elements a workgroup, turned through LDS.
__global__ __launch_bounds__(256) void ortho_split_kernel(OrthoTiles) {
  __shared__ float turn[64][65];
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  const double inv = ortho_inverse_norm(args.sums + (int64_t)T.matrix * args.sums_of_launch, args.sums_of_launch) * ORTHO_SCALE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col0 = (block % T.across) * 64, row0 = block / T.across * 64;
  // the last tiles of a matrix also clear what fills its rows and columns up
  const int w = T.col0 + T.w == args.cols ? args.row_pitch - T.col0 : T.w;
  const int h = T.row0 + T.h == args.rows ? args.col_pitch - T.row0 : T.h;
  char *const ws = args.ws + T.matrix * args.stride;
  char *const by_rows = ws + args.by_rows, *const by_cols = ws + args.by_cols;
  for (int r = wave; r < 64; r += 4) {
    const int row = row0 + r, col = col0 + lane;
    const float v = row < T.h && col < T.w ? (float)((double)ortho_load(T.p + (int64_t)row * T.pitch, args.f32, col) * inv) : 0.f;
    turn[r][lane] = v;
    if (row < T.h && col < w) {
      const OrthoPair p = ortho_split(v);
      char *const at = by_rows + ortho_at(T.row0 + row, T.col0 + col, args.row_pitch);
      *(_Float16 *)at = p.high;
      *(_Float16 *)(at + 64) = p.low;
    }
  }
  __syncthreads();
  for (int c = wave; c < 64; c += 4) {
    const int row = row0 + lane, col = col0 + c;
    if (col < T.w && row < h) {
      const OrthoPair p = ortho_split(turn[lane][c]);
      char *const at = by_cols + ortho_at(T.col0 + col, T.row0 + row, args.col_pitch);
      *(_Float16 *)at = p.high;
      *(_Float16 *)(at + 64) = p.low;
    }
  }
}

// The result, fp32 and dense, into the tiles.
__global__ __launch_bounds__(256) void ortho_store_kernel(OrthoTiles) {
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = (block % T.across) * 64 + lane, row0 = block / T.across * 64;
  const float *const y = (const float *)(args.ws + T.matrix * args.stride + args.by_rows);
  if (col >= T.w) return;
  for (int r = row0 + wave; r < min(row0 + 64, T.h); r += 4) {
    const float v = y[(int64_t)(T.row0 + r) * args.cols + T.col0 + col];
    char *const row = T.p + (int64_t)r * T.pitch;
    if (args.f32) ((float *)row)[col] = v;
    else ((__bf16 *)row)[col] = (__bf16)v;
  }
}

typedef _Float16 ortho_h8 __attribute__((ext_vector_type(8)));

// Eight neighbouring elements of a row of out: their sums to what they hold (zero outside of the matrix), stored row by
// row; the values replace the sums.
__device__ __forceinline__ void ortho_rows8(const OrthoProduct &g, char *ws, int row, int col, float *v) {
  const int64_t at = ortho_at(row, col, g.out_pitch);
  if (row >= g.m || (unsigned)col >= g.out_pitch) {           // (out_pitch is a multiple of 32)
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = 0.f;
    return;
  }
  ortho_h8 high = {}, low = {};
  if (g.old >= 0) {
    high = *(const ortho_h8 *)(ws + g.old + at);
    low = *(const ortho_h8 *)(ws + g.old + at + 64);
  }
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    v[x] = col + x < g.n ? g.alpha * ((float)high[x] + (float)low[x]) + g.beta * v[x] : 0.f;
    const OrthoPair p = ortho_split(v[x]);
    high[x] = p.high;
    low[x] = p.low;
  }
  if (g.y >= 0) return;
  *(ortho_h8 *)(ws + g.out + at) = high;
  *(ortho_h8 *)(ws + g.out + at + 64) = low;
}
// Eight neighbouring elements of a column of out, into its transpose.
__device__ __forceinline__ void ortho_cols8(const OrthoProduct &g, char *ws, int row, int col, const float *v) {
  if (col >= g.n || (unsigned)row >= g.turned_pitch) return;
  ortho_h8 high, low;
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const OrthoPair p = ortho_split(v[x]);
    high[x] = p.high;
    low[x] = p.low;
  }
  char *const at = ws + g.turned + ortho_at(col, row, g.turned_pitch);
  *(ortho_h8 *)at = high;
  *(ortho_h8 *)(at + 64) = low;
}

// ROWS rows of a tile in LDS, `pitch` floats each: half of them are rows row0 ... of out, the others lie `apart` further on.
template <int TN, int ROWS>
__device__ __forceinline__ void ortho_finish(const OrthoProduct &g, char *ws, float *values, int pitch, int row0, int apart, int col0, bool mirror) {
  constexpr int PER = TN / 8, HALF = ROWS / 2;
  auto row_of = [&](int r) { return row0 + r % HALF + r / HALF * apart; };
  for (int x = threadIdx.x; x < ROWS * PER; x += NT_THREADS) {
    const int r = x / PER, c = x % PER * 8;
    float *const p = values + r * pitch + c;
    float v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) v[y] = p[y];
    ortho_rows8(g, ws, row_of(r), col0 + c, v);
#pragma unroll
    for (int y = 0; y < 8; ++y) p[y] = v[y];
  }
  if (g.y >= 0) {
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * TN; x += NT_THREADS) {
      // (lanes run along the rows of Y)
      const int r = g.y_turned ? x % ROWS : x / TN, c = g.y_turned ? x / ROWS : x % TN;
      const int row = row_of(r), col = col0 + c;
      if (row < g.m && col < g.n) ((float *)(ws + g.y))[g.y_turned ? (int64_t)col * g.m + row : (int64_t)row * g.n + col] = values[r * pitch + c] * (1.f / ORTHO_SCALE);
    }
  } else if (mirror) {
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS / 8 * TN; x += NT_THREADS) {
      const int r = x % (ROWS / 8) * 8, c = x / (ROWS / 8);
      float v[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) v[y] = values[(r + y) * pitch + c];
      ortho_cols8(g, ws, row_of(r), col0 + c, v);
    }
  }
}

struct OrthoPlace {
  int matrix, row, col;         // row and column of tiles
};
// Bands of eight tile rows, column by column: the tiles that run on an XCD at a time share operands.  Of a symmetric
// result the tiles on and above the diagonal.
__device__ __forceinline__ OrthoPlace ortho_place(const OrthoProduct &g, int t) {
  OrthoPlace p;
  p.matrix = t / g.tiles;
  t %= g.tiles;
  int row0 = 0;
  for (;; row0 += 8) {
    const int rows = min(8, g.tiles_m - row0);
    const int n = g.symmetric ? (g.tiles_n - row0) * rows - rows * (rows - 1) / 2 : g.tiles_n * rows;
    if (t >= n) {
      t -= n;
      continue;
    }
    if (g.symmetric) {
      // columns row0, row0 + 1, ... of 1, 2, ..., rows, rows, ... tiles
      int c = 0;
      while (c < rows && t > c) t -= ++c;
      if (c == rows) {
        c = rows + t / rows;
        t %= rows;
      }
      p.row = row0 + t;
      p.col = row0 + c;
    } else {
      p.row = row0 + t % rows;
      p.col = t / rows;
    }
    return p;
  }
}

template <class SH>
__global__ __launch_bounds__(NT_THREADS, SH::LDS > 80 * 1024 ? 1 : 2) void ortho_product_kernel(const OrthoProduct g) {
  extern __shared__ char lds[];
  // workgroup w runs on XCD w % 8: every XCD gets a run of the whole tiles, and of the list of all first ranges of the others, all
  // second ones, ... (it then reads a range of K of all rows)
  const bool cut = (int)blockIdx.x >= g.whole;
  const int w = cut ? (int)blockIdx.x - g.whole : (int)blockIdx.x, rest = g.count * g.tiles - g.whole, n = cut ? rest * g.runs : g.whole;
  const int in_list = (w & 7) * (n >> 3) + min(w & 7, n & 7) + (w >> 3);
  const int run = cut ? in_list / rest : 0, piece = in_list - run * rest;
  const OrthoPlace at = ortho_place(g, cut ? g.whole + piece : in_list);
  char *const ws = g.ws + at.matrix * g.stride;
  struct Seg {
    NtSeg s;
    __device__ __forceinline__ NtSeg operator[](int) const { return s; }
  };
  const int begin = run * g.per, end = cut ? min(begin + g.per, g.steps) : g.steps;
  const int m0 = at.row * SH::TM, n0 = at.col * SH::TN;
  NtTile<SH> tile;
  const Seg seg = {{ws + g.a, ws + g.b, nullptr, nullptr, g.k_pitch_a, g.k_pitch_b, 0, 0, 2 * g.steps, 0}};
  tile.run(seg, 1, begin, end - begin, m0, min(SH::TM, g.m - m0), n0, min(SH::TN, g.n - n0), lds);
  tile.pin();
  const bool mirror = g.turned >= 0 && !(g.symmetric && at.row == at.col);
  if (cut) {
    float *const part = g.parts + ((int64_t)piece * g.runs + run) * (SH::TM * SH::TN);
    tile.slices(lds, [&](const float *values, int base) {
      for (int x = threadIdx.x; x < 64 * SH::TN / 4; x += NT_THREADS) {
        const int r = x / (SH::TN / 4), c = x % (SH::TN / 4) * 4;
        *(nt_f32x4 *)(part + (base + (r & 31) + (r >> 5) * (SH::TM / 2)) * SH::TN + c) = *(const nt_f32x4 *)(values + r * NtTile<SH>::PITCH + c);
      }
    });
  } else {
    tile.slices(lds, [&](float *values, int base) {
      ortho_finish<SH::TN, 64>(g, ws, values, NtTile<SH>::PITCH, m0 + base, SH::TM / 2, n0, mirror);
    });
  }
}

// Tiles cut along K: the sums of their runs, in ascending order.  16 rows of a tile a workgroup.
template <int EDGE>
__global__ __launch_bounds__(256) void ortho_join_kernel(const OrthoProduct g) {
  constexpr int BLOCKS = EDGE / 16, PITCH = EDGE + 4;
  __shared__ float values[16 * PITCH];
  const int t = blockIdx.x / BLOCKS, rows0 = blockIdx.x % BLOCKS * 16;
  const OrthoPlace at = ortho_place(g, g.whole + t);
  const float *const p = g.parts + (int64_t)t * g.runs * (EDGE * EDGE) + rows0 * EDGE;
  constexpr int N = 16 * EDGE / 4 / 256;                      // four columns at a time
  nt_f32x4 sum[N];
#pragma unroll
  for (int y = 0; y < N; ++y) sum[y] = ((const nt_f32x4 *)p)[y * 256 + threadIdx.x];
#pragma unroll 4
  for (int r = 1; r < g.runs; ++r)
#pragma unroll
    for (int y = 0; y < N; ++y) sum[y] += ((const nt_f32x4 *)(p + (int64_t)r * (EDGE * EDGE)))[y * 256 + threadIdx.x];
#pragma unroll
  for (int y = 0; y < N; ++y) {
    const int x = y * 256 + threadIdx.x;
    *(nt_f32x4 *)(values + x / (EDGE / 4) * PITCH + x % (EDGE / 4) * 4) = sum[y];
  }
  __syncthreads();
  ortho_finish<EDGE, 16>(g, g.ws + at.matrix * g.stride, values, PITCH, at.row * EDGE + rows0, 8, at.col * EDGE,
                         g.turned >= 0 && !(g.symmetric && at.row == at.col));
}

}  // namespace dmm
