// Newton-Schulz steps that bring the singular values of a matrix near 1 (gfx950, device code only):
//   X_0 = G / |G|,   S = X X^T,   X <- a X + (b S + c S S) X
// with X the matrix or its transpose, whichever has fewer rows.
//
// Every matrix is kept as two fp16 planes, v 2^12 = high + low with low the rounded rest: 22 bits of a value, and
// a product of two is high low + low high + high high, three matrix instructions (what is left out is 2^-22 of it).  Singular
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

// Sum of squares of 64 x 64 elements of a tile, in 64 bits (an fp32 square may not have a place in fp32), added up in a fixed order:
// every block has a place of its own among its matrix' sums.
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoTiles) {
  __shared__ double part[4];
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  // (a tile's blocks share its places: block b takes the pieces b, b + across, ...)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pieces_c = (T.w + 63) >> 6, pieces = ((T.h + 63) >> 6) * pieces_c;
  double sum = 0.0;
  for (int p = block; p < pieces; p += T.across) {
    const int col = (p % pieces_c) * 64 + lane, row0 = p / pieces_c * 64;
    if (col < T.w)
      for (int r = row0 + wave; r < min(row0 + 64, T.h); r += 4) {
        const double v = ortho_load(T.p + (int64_t)r * T.pitch, args.f32, col);
        sum += v * v;
      }
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
  _Float16 *const by_rows = (_Float16 *)(ws + args.by_rows), *const by_cols = (_Float16 *)(ws + args.by_cols);
  const int64_t rows_plane = (int64_t)args.rows * args.row_pitch, cols_plane = (int64_t)args.cols * args.col_pitch;
  for (int r = wave; r < 64; r += 4) {
    const int row = row0 + r, col = col0 + lane;
    const float v = row < T.h && col < T.w ? (float)((double)ortho_load(T.p + (int64_t)row * T.pitch, args.f32, col) * inv) : 0.f;
    turn[r][lane] = v;
    if (row < T.h && col < w) {
      const OrthoPair p = ortho_split(v);
      const int64_t at = (int64_t)(T.row0 + row) * args.row_pitch + T.col0 + col;
      by_rows[at] = p.high;
      by_rows[rows_plane + at] = p.low;
    }
  }
  __syncthreads();
  for (int c = wave; c < 64; c += 4) {
    const int row = row0 + lane, col = col0 + c;
    if (col < T.w && row < h) {
      const OrthoPair p = ortho_split(turn[lane][c]);
      const int64_t at = (int64_t)(T.col0 + col) * args.col_pitch + T.row0 + row;
      by_cols[at] = p.high;
      by_cols[cols_plane + at] = p.low;
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

// Eight neighbouring elements of a row of out: their sums to what they hold (zero outside of the matrix), stored in the
// row-wise planes; the values replace the sums.
__device__ __forceinline__ void ortho_rows8(const OrthoProduct &g, char *ws, int row, int col, float *v) {
  const int64_t at = (int64_t)row * g.out_pitch + col;
  if (row >= g.m || (unsigned)col >= g.out_pitch) {           // (out_pitch is a multiple of 64)
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = 0.f;
    return;
  }
  ortho_h8 high = {}, low = {};
  if (g.old >= 0) {
    high = *(const ortho_h8 *)((const _Float16 *)(ws + g.old) + at);
    low = *(const ortho_h8 *)((const _Float16 *)(ws + g.old_low) + at);
  }
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    v[x] = col + x < g.n ? g.alpha * ((float)high[x] + (float)low[x]) + g.beta * v[x] : 0.f;
    const OrthoPair p = ortho_split(v[x]);
    high[x] = p.high;
    low[x] = p.low;
  }
  if (g.y >= 0) return;
  *(ortho_h8 *)((_Float16 *)(ws + g.out) + at) = high;
  *(ortho_h8 *)((_Float16 *)(ws + g.out_low) + at) = low;
}
// Eight neighbouring elements of a column of out, into the planes of its transpose.
__device__ __forceinline__ void ortho_cols8(const OrthoProduct &g, char *ws, int row, int col, const float *v) {
  if (col >= g.n || (unsigned)row >= g.turned_pitch) return;
  ortho_h8 high, low;
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const OrthoPair p = ortho_split(v[x]);
    high[x] = p.high;
    low[x] = p.low;
  }
  const int64_t at = (int64_t)col * g.turned_pitch + row;
  *(ortho_h8 *)((_Float16 *)(ws + g.turned) + at) = high;
  *(ortho_h8 *)((_Float16 *)(ws + g.turned_low) + at) = low;
}

// 64 rows of a tile in LDS, `pitch` floats each: rows row0 .. row0 + 31 of out, and `apart` further on 32 more.
template <int TN>
__device__ __forceinline__ void ortho_finish(const OrthoProduct &g, char *ws, float *values, int pitch, int row0, int apart, int col0, bool mirror) {
  constexpr int PER = TN / 8;
  for (int x = threadIdx.x; x < 64 * PER; x += NT_THREADS) {
    const int r = x / PER, c = x % PER * 8;
    float *const p = values + r * pitch + c;
    float v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) v[y] = p[y];
    ortho_rows8(g, ws, row0 + (r & 31) + (r >> 5) * apart, col0 + c, v);
#pragma unroll
    for (int y = 0; y < 8; ++y) p[y] = v[y];
  }
  if (g.y >= 0) {
    __syncthreads();
    for (int x = threadIdx.x; x < 64 * TN; x += NT_THREADS) {
      // (lanes run along the rows of Y)
      const int r = g.y_turned ? x % 64 : x / TN, c = g.y_turned ? x / 64 : x % TN;
      const int row = row0 + (r & 31) + (r >> 5) * apart, col = col0 + c;
      if (row < g.m && col < g.n) ((float *)(ws + g.y))[g.y_turned ? (int64_t)col * g.m + row : (int64_t)row * g.n + col] = values[r * pitch + c] * (1.f / ORTHO_SCALE);
    }
  } else if (mirror) {
    __syncthreads();
    for (int x = threadIdx.x; x < 8 * TN; x += NT_THREADS) {
      const int r = x % 8 * 8, c = x / 8;
      float v[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) v[y] = values[(r + y) * pitch + c];
      ortho_cols8(g, ws, row0 + (r & 31) + (r >> 5) * apart, col0 + c, v);
    }
  }
}

struct OrthoPlace {
  int matrix, row, col, run;    // row and column of tiles
};
__device__ __forceinline__ OrthoPlace ortho_place(const OrthoProduct &g, int block) {
  OrthoPlace p;
  // workgroup w runs on XCD w % 8: every XCD gets a run of the list
  const int n = g.count * g.tiles * g.runs, xcd = block & 7;
  int t = xcd * (n >> 3) + min(xcd, n & 7) + (block >> 3);
  p.run = t % g.runs;
  t /= g.runs;
  p.matrix = t / g.tiles;
  t %= g.tiles;
  if (g.symmetric) {            // tiles on and above the diagonal, row by row
    p.row = 0;
    while (t >= g.tiles_n - p.row) t -= g.tiles_n - p.row++;
    p.col = p.row + t;
  } else {                      // bands of eight tile rows, column by column
    const int band = t / (8 * g.tiles_n), rows = min(8, g.tiles_m - band * 8), in = t - band * 8 * g.tiles_n;
    p.row = band * 8 + in % rows;
    p.col = in / rows;
  }
  return p;
}

template <class SH>
__global__ __launch_bounds__(NT_THREADS, SH::TM == 256 ? 1 : 2) void ortho_product_kernel(const OrthoProduct g) {
  extern __shared__ char lds[];
  const OrthoPlace at = ortho_place(g, blockIdx.x);
  char *const ws = g.ws + at.matrix * g.stride;
  struct Segs {                 // low high, high low, high high
    const OrthoProduct &g;
    const char *ws;
    __device__ __forceinline__ NtSeg operator[](int i) const {
      NtSeg s;
      s.a = ws + (i == 0 ? g.a_low : g.a);
      s.b = ws + (i == 1 ? g.b_low : g.b);
      s.a_scale = s.b_scale = nullptr;
      s.a_pitch = g.k_pitch_a;
      s.b_pitch = g.k_pitch_b;
      s.a_scale_pitch = s.b_scale_pitch = 0;
      s.chunks = 2 * g.steps;
      s.pad = 0;
      return s;
    }
  };
  struct From {
    Segs s;
    int first;
    __device__ __forceinline__ NtSeg operator[](int i) const { return s[first + i]; }
  };
  const int begin = at.run * g.per, end = min(begin + g.per, 3 * g.steps);
  const int first = begin / g.steps;
  const int m0 = at.row * SH::TM, n0 = at.col * SH::TN;
  NtTile<SH> tile;
  tile.run(From{{g, ws}, first}, 3 - first, begin - first * g.steps, end - begin, m0, min(SH::TM, g.m - m0), n0, min(SH::TN, g.n - n0), lds);
  tile.pin();
  const bool mirror = g.turned >= 0 && !(g.symmetric && at.row == at.col);
  if (g.runs > 1) {
    const int t = g.symmetric ? at.row * g.tiles_n - at.row * (at.row - 1) / 2 + at.col - at.row : at.row * g.tiles_n + at.col;
    float *const part = g.parts + ((int64_t)(at.matrix * g.tiles + t) * g.runs + at.run) * (SH::TM * SH::TN);
    tile.slices(lds, [&](const float *values, int base) {
      for (int x = threadIdx.x; x < 64 * SH::TN / 4; x += NT_THREADS) {
        const int r = x / (SH::TN / 4), c = x % (SH::TN / 4) * 4;
        *(nt_f32x4 *)(part + (base + (r & 31) + (r >> 5) * (SH::TM / 2)) * SH::TN + c) = *(const nt_f32x4 *)(values + r * NtTile<SH>::PITCH + c);
      }
    });
  } else {
    tile.slices(lds, [&](float *values, int base) {
      ortho_finish<SH::TN>(g, ws, values, NtTile<SH>::PITCH, m0 + base, SH::TM / 2, n0, mirror);
    });
  }
}

// Tiles cut along K: the sums of their runs, in ascending order.  64 rows of a tile a workgroup.
template <int EDGE>
__global__ __launch_bounds__(256) void ortho_join_kernel(const OrthoProduct g) {
  constexpr int BLOCKS = EDGE / 64, PITCH = EDGE + 4;
  extern __shared__ char lds[];
  float *const values = (float *)lds;
  const int t = blockIdx.x / BLOCKS, row64 = blockIdx.x % BLOCKS * 64;
  const int matrix = t / g.tiles;
  int in = t % g.tiles, row = 0, col;
  if (g.symmetric) {
    while (in >= g.tiles_n - row) in -= g.tiles_n - row++;
    col = row + in;
  } else {
    row = in / g.tiles_n;
    col = in % g.tiles_n;
  }
  const float *const p = g.parts + (int64_t)t * g.runs * (EDGE * EDGE) + row64 * EDGE;
  for (int x = threadIdx.x; x < 64 * EDGE / 4; x += 256) {
    nt_f32x4 sum = ((const nt_f32x4 *)p)[x];
    for (int r = 1; r < g.runs; ++r) sum += *(const nt_f32x4 *)(p + (int64_t)r * (EDGE * EDGE) + x * 4);
    *(nt_f32x4 *)(values + x / (EDGE / 4) * PITCH + x % (EDGE / 4) * 4) = sum;
  }
  __syncthreads();
  ortho_finish<EDGE>(g, g.ws + matrix * g.stride, values, PITCH, row * EDGE + row64, 32, col * EDGE, g.turned >= 0 && !(g.symmetric && row == col));
}

}  // namespace dmm
