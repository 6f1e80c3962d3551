// Newton-Schulz steps that bring the singular values of a matrix near 1 (gfx950, device code only):
//   X_0 = G / |G|,   S = X X^T,   X <- (a I + b S + c S S) X
// with X the matrix or its transpose, whichever has fewer rows.
//
// Every matrix is kept as pairs of fp16, v 2^12 = high + low with low the rounded rest: 22 bits of a value, and
// a product of two is low high + high low + high high, three matrix instructions (what is left out is 2^-22 of it).  Singular
// values far below the largest grow by 3.4 each step, and so do errors: rounded to bf16 once per step a matrix with a few
// strong directions comes out 28 % off (512 x 512, rank 16 over 1 % of noise), in fp16 4 %, in pairs 7e-6, in plain fp32 2e-5.
// (Frobenius norms.)
// The factor 2^12: no value reaches 16 (the host refuses coefficients with which one could pass 15; the default ones leave |X| <= 1.21
// and |b S + c S S| < 3), and the low part of one of 2^-13, the size of an element of a normalised 8192 x 8192 matrix, still is
// a multiple of 2^-24 / 2^12.  Rows smaller than the matrix by 10^6 and more lose digits to that step (256 x 1024: 10^6 4e-4
// of themselves, 10^8 4e-2).
#pragma once

#include "nt_kernel.hpp"
#include "ortho_launch.hpp"

namespace dmm {

constexpr float ORTHO_SCALE = 4096.f;

typedef _Float16 ortho_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 ortho_h4 __attribute__((ext_vector_type(4)));
typedef _Float16 ortho_h8 __attribute__((ext_vector_type(8)));
typedef float ortho_f2 __attribute__((ext_vector_type(2)));
// where the high part of an element lies in a matrix of `pitch` elements a row; the low part is 64 bytes on
__device__ __forceinline__ int64_t ortho_at(int row, int col, unsigned pitch) {
  return (int64_t)row * (pitch * 4u) + (col >> 5) * 128 + (col & 31) * 2;
}
// Two values as pairs: four instructions (v - high in one, of a half that is not taken out first).
struct OrthoPairs {
  ortho_h2 high, low;
};
__device__ __forceinline__ OrthoPairs ortho_split(float v0, float v1) {
  OrthoPairs p;
  p.high = __builtin_convertvector((ortho_f2){v0, v1}, ortho_h2);
  ortho_f2 rest;
  float r0, r1;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(p.high), "v"(v0));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(p.high), "v"(v1));
  rest = (ortho_f2){r0, r1};
  p.low = __builtin_convertvector(rest, ortho_h2);
  return p;
}
__device__ __forceinline__ void ortho_split8(const float *v, ortho_h8 &high, ortho_h8 &low) {
#pragma unroll
  for (int x = 0; x < 8; x += 2) {
    const OrthoPairs p = ortho_split(v[x], v[x + 1]);
    high[x] = p.high[0], high[x + 1] = p.high[1];
    low[x] = p.low[0], low[x + 1] = p.low[1];
  }
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

// G / |G| as pairs, by rows and by columns: 64 x 64 elements a workgroup, turned through LDS, from multiples of 8 on so that eight
// neighbours are stored together, 16 bytes high and 16 low parts; element by element where a tile begins or ends inside of
// them.  (Stores of two bytes took 1021 x 4090 21 us, these take 17; 50 MB.)
__global__ __launch_bounds__(256) void ortho_split_kernel(OrthoTiles) {
  __shared__ float turn[64][65];
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // rows and columns of the tile; those in front of it are negative
  const int col0 = (block % T.across) * 64 - (T.col0 & 7), row0 = block / T.across * 64 - (T.row0 & 7);
  float v[16];
#pragma unroll
  for (int x = 0; x < 16; ++x)
    v[x] = ortho_load(T.p + (int64_t)min(max(row0 + 16 * wave + x, 0), T.h - 1) * T.pitch, args.f32, min(max(col0 + lane, 0), T.w - 1));
  const double inv = ortho_inverse_norm(args.sums + (int64_t)T.matrix * args.sums_of_launch, args.sums_of_launch) * ORTHO_SCALE;
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    const int row = row0 + 16 * wave + x, col = col0 + lane;
    turn[16 * wave + x][lane] = row >= 0 && row < T.h && col >= 0 && col < T.w ? (float)((double)v[x] * inv) : 0.f;
  }
  __syncthreads();
  // the last tiles of a matrix also clear what fills its rows and columns up
  const int w = T.col0 + T.w == args.cols ? args.row_pitch - T.col0 : T.w;
  const int h = T.row0 + T.h == args.rows ? args.col_pitch - T.row0 : T.h;
  char *const ws = args.ws + T.matrix * args.stride;
  // elements `line`, `at` ... at + 7 of a matrix whose tile has lines 0 ... lines - 1 and elements 0 ... n - 1 of them
  auto put = [&](char *to, int line, int lines, int line0, int at, int n, int at0, unsigned pitch, const float *f) {
    if (line < 0 || line >= lines) return;
    ortho_h8 high, low;
    ortho_split8(f, high, low);
    char *const out = to + ortho_at(line0 + line, at0 + at, pitch);
    if (at >= 0 && at + 8 <= n) {
      *(ortho_h8 *)out = high;
      *(ortho_h8 *)(out + 64) = low;
      return;
    }
#pragma unroll
    for (int x = 0; x < 8; ++x)
      if (at + x >= 0 && at + x < n) {
        ((_Float16 *)out)[x] = high[x];
        ((_Float16 *)(out + 64))[x] = low[x];
      }
  };
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int line = 32 * x + 8 * wave + (lane >> 3), at = (lane & 7) * 8;
    float f[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) f[y] = turn[line][at + y];
    put(ws + args.by_rows, row0 + line, T.h, T.row0, col0 + at, w, T.col0, args.row_pitch, f);
#pragma unroll
    for (int y = 0; y < 8; ++y) f[y] = turn[at + y][line];
    put(ws + args.by_cols, col0 + line, T.w, T.col0, row0 + at, h, T.row0, args.col_pitch, f);
  }
}

// The result, fp32 and dense, into the tiles.
__global__ __launch_bounds__(256) void ortho_store_kernel(OrthoTiles) {
  const auto &args = *(const OrthoTiles *)__builtin_amdgcn_kernarg_segment_ptr();
  int block;
  const OrthoTile &T = ortho_find(args, blockIdx.x, &block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = (block % T.across) * 64 + lane, row0 = block / T.across * 64 + wave * 16;
  const float *const y = (const float *)(args.ws + T.matrix * args.stride + args.by_rows) + T.col0 + col;
  if (col >= T.w) return;
  float v[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = y[(int64_t)(T.row0 + min(row0 + r, T.h - 1)) * args.cols];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (row0 + r >= T.h) return;
    char *const row = T.p + (int64_t)(row0 + r) * T.pitch;
    if (args.f32) ((float *)row)[col] = v[r];
    else ((__bf16 *)row)[col] = (__bf16)v[r];
  }
}

// What eight neighbouring elements of a row of out are added to.
__device__ __forceinline__ void ortho_old8(const OrthoProduct &g, const char *ws, int row, int col, ortho_h8 &high, ortho_h8 &low) {
  high = low = ortho_h8{};
  if (g.old < 0 || row >= g.m || (unsigned)col >= g.out_pitch) return;   // (out_pitch is a multiple of 32)
  const char *const at = ws + g.old + ortho_at(row, col, g.out_pitch);
  high = *(const ortho_h8 *)at;
  low = *(const ortho_h8 *)(at + 64);
}
// Their sums to what they hold (zero outside of the matrix), stored row by row; the values replace the sums.
__device__ __forceinline__ void ortho_rows8(const OrthoProduct &g, char *ws, int row, int col, ortho_h8 high, ortho_h8 low, float *v) {
  if (row >= g.m || (unsigned)col >= g.out_pitch) {
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = 0.f;
    return;
  }
#pragma unroll
  for (int x = 0; x < 8; ++x)
    v[x] = col + x < g.n ? g.alpha * ((float)high[x] + (float)low[x]) + g.beta * v[x] : 0.f;
  if (g.y >= 0) return;
  ortho_split8(v, high, low);
  const int64_t at = ortho_at(row, col, g.out_pitch);
  *(ortho_h8 *)(ws + g.out + at) = high;
  *(ortho_h8 *)(ws + g.out + at + 64) = low;
}
// Eight neighbouring elements of a column of out, into its transpose.
__device__ __forceinline__ void ortho_cols8(const OrthoProduct &g, char *ws, int row, int col, const float *v) {
  if (col >= g.n || (unsigned)row >= g.turned_pitch) return;
  ortho_h8 high, low;
  ortho_split8(v, high, low);
  char *const at = ws + g.turned + ortho_at(col, row, g.turned_pitch);
  *(ortho_h8 *)at = high;
  *(ortho_h8 *)(at + 64) = low;
}

// ROWS rows of a tile in LDS, `pitch` floats each: half of them are rows row0 ... of out, the others lie `apart` further on.
template <int TN, int ROWS>
__device__ __forceinline__ void ortho_finish(const OrthoProduct &g, char *ws, float *values, int pitch, int row0, int apart, int col0, bool mirror) {
  constexpr int PER = TN / 8, HALF = ROWS / 2;
  auto row_of = [&](int r) { return row0 + r % HALF + r / HALF * apart; };
  // (what a thread reads is read at once: one after the other every read waits out its latency)
  constexpr int N = (ROWS * PER + NT_THREADS - 1) / NT_THREADS;
  float v[N][8];
  ortho_h8 high[N], low[N];
  const bool all = ROWS * PER % NT_THREADS == 0 || (int)threadIdx.x < ROWS * PER;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = i * NT_THREADS + threadIdx.x;
    if (all) ortho_old8(g, ws, row_of(x / PER), col0 + x % PER * 8, high[i], low[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = i * NT_THREADS + threadIdx.x;
    const float *const p = values + nt_value(all ? x / PER : 0, x % PER * 8, pitch);
#pragma unroll
    for (int y = 0; y < 8; ++y) v[i][y] = p[y];
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = i * NT_THREADS + threadIdx.x, r = x / PER, c = x % PER * 8;
    if (!all) break;
    ortho_rows8(g, ws, row_of(r), col0 + c, high[i], low[i], v[i]);
    float *const p = values + nt_value(r, c, pitch);
#pragma unroll
    for (int y = 0; y < 8; ++y) p[y] = v[i][y];
  }
  if (g.y >= 0) {
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * TN; x += NT_THREADS) {
      // (lanes run along the rows of Y)
      const int r = g.y_turned ? x % ROWS : x / TN, c = g.y_turned ? x / ROWS : x % TN;
      const int row = row_of(r), col = col0 + c;
      if (row < g.m && col < g.n) ((float *)(ws + g.y))[g.y_turned ? (int64_t)col * g.m + row : (int64_t)row * g.n + col] = values[nt_value(r, c, pitch)] * (1.f / ORTHO_SCALE);
    }
  } else if (mirror) {
    __syncthreads();
    constexpr int M = (ROWS / 8 * TN + NT_THREADS - 1) / NT_THREADS;
    const bool some = ROWS / 8 * TN % NT_THREADS == 0 || (int)threadIdx.x < ROWS / 8 * TN;
    float u[M][8];
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int x = i * NT_THREADS + threadIdx.x, r = some ? x % (ROWS / 8) * 8 : 0, c = some ? x / (ROWS / 8) : 0;
#pragma unroll
      for (int y = 0; y < 8; ++y) u[i][y] = values[nt_value(r + y, c, pitch)];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int x = i * NT_THREADS + threadIdx.x;
      if (some) ortho_cols8(g, ws, row_of(x % (ROWS / 8) * 8), col0 + x / (ROWS / 8), u[i]);
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
__global__ __launch_bounds__(NT_THREADS, SH::LDS > 80 * 1024 ? 1 : SH::TM == 64 ? 3 : 2) void ortho_product_kernel(const OrthoProduct g) {
  extern __shared__ char lds[];
  // workgroup w runs on XCD w % 8: every XCD gets a run of the whole tiles, and of the list of all first ranges of the others, all
  // second ones, ... (it then reads a range of K of all rows)
  const bool cut = (int)blockIdx.x >= g.whole;
  const int w = cut ? (int)blockIdx.x - g.whole : (int)blockIdx.x, rest = g.count * g.tiles - g.whole, n = cut ? rest * g.runs : g.whole;
  const int in_list = (w & 7) * (n >> 3) + min(w & 7, n & 7) + (w >> 3);
  const int run = cut ? in_list / rest : 0, piece = in_list - run * rest;
  const OrthoPlace at = ortho_place(g, cut ? g.whole + piece : in_list);
  char *const ws = g.ws + at.matrix * g.stride;
  const int begin = run * g.per, end = cut ? min(begin + g.per, g.steps) : g.steps;
  const int m0 = at.row * SH::TM, n0 = at.col * SH::TN;
  NtTile<SH> tile;
  const NtSeg seg = {ws + g.a, ws + g.b, nullptr, nullptr, g.k_pitch_a, g.k_pitch_b, 0, 0, 2 * g.steps, 0};
  tile.run(seg, nullptr, 1, begin, end - begin, m0, min(SH::TM, g.m - m0), n0, min(SH::TN, g.n - n0), lds);
  tile.pin();
  const bool mirror = g.turned >= 0 && !(g.symmetric && at.row == at.col);
  if (cut) {
    float *const part = g.parts + ((int64_t)piece * g.runs + run) * (SH::TM * SH::TN);
    tile.slices(lds, [&](const float *values, int base) {
      for (int x = threadIdx.x; x < 64 * SH::TN / 4; x += NT_THREADS) {
        const int r = x / (SH::TN / 4), c = x % (SH::TN / 4) * 4;
        *(nt_f32x4 *)(part + (base + (r & 31) + (r >> 5) * (SH::TM / 2)) * SH::TN + c) = *(const nt_f32x4 *)(values + nt_value(r, c, NtTile<SH>::PITCH));
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
    *(nt_f32x4 *)(values + nt_value(x / (EDGE / 4), x % (EDGE / 4) * 4, PITCH)) = sum[y];
  }
  __syncthreads();
  ortho_finish<EDGE, 16>(g, g.ws + at.matrix * g.stride, values, PITCH, at.row * EDGE + rows0, 8, at.col * EDGE,
                         g.turned >= 0 && !(g.symmetric && at.row == at.col));
}

// ---- small matrices ---------------------------------------------------------------------------------
//
// X stays in registers in fp32, eight waves of 32 x 64 elements each; what a product reads goes through LDS as pairs, two areas of
// 128 rows: X by rows, then by columns, and S, then P.  Five barriers a step, no memory traffic between the first load and the
// last store.  Bound by one CU: 3 x 384 matrix instructions of 32 cycles a step on its four pipes (9200 cycles), with LDS reads that
// take as long (6 KB for every six of a wave); taking values apart and storing them between the barriers is the other half of 17000 cycles
// a step, 41.6 us a call of five.  In launches of the products above every one of the 18 took 8 to 15 us: 32 matrices of 128 x 128 200 us.
constexpr int ORTHO_SMALL_THREADS = 512;
constexpr int ORTHO_AREA = ORTHO_SMALL * ORTHO_SMALL * 4;    // bytes

// Byte of an area that holds the high part of (row, k), the low part 64 further on (^ 64: it is the fourth bit of the slot's number);
// 16-byte slots are exchanged by row so that 16 rows of one slot lie in different banks.
__device__ __forceinline__ int ortho_area(int row, int k) {
  const int slot = (k >> 5) * 8 + ((k & 31) >> 3);
  return row * (ORTHO_SMALL * 4) + ((slot ^ (row & 15)) << 4) + (k & 7) * 2;
}

__global__ __launch_bounds__(ORTHO_SMALL_THREADS) void ortho_small_kernel(OrthoSmall) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  double *const part = (double *)lds;  // (for the norm, before the areas are used)
  const auto &args = *(const OrthoSmall *)__builtin_amdgcn_kernarg_segment_ptr();
  auto M = args.matrix[args.even ? 0 : blockIdx.x];
  if (args.even) {
    M.x += (int64_t)blockIdx.x * (args.matrix[1].x - M.x);
    M.y += (int64_t)blockIdx.x * (args.matrix[1].y - M.y);
  }
  const int64_t x_pitch = (int64_t)M.x_ld * (args.x_f32 ? 4 : 2), y_pitch = (int64_t)M.y_ld * (args.y_f32 ? 4 : 2);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int r = lane & 31, g = lane >> 5;
  const bool flip = args.rows > args.cols;
  const int s = flip ? args.cols : args.rows, l = flip ? args.rows : args.cols;   // X is s x l
  const int row0 = (wave >> 1) * 32, col0 = (wave & 1) * 64;
  const unsigned area1 = (unsigned)(uintptr_t)(nt_lptr)lds, area2 = area1 + ORTHO_AREA;
  auto row_of = [&](int x) { return row0 + 8 * (x / 4) + 4 * g + x % 4; };
  nt_f32x16 X[2], S[2];

  // ---- G / |G| -----------------------------------------------------------------------------
  double sum = 0.0;
  // (all loads first, whatever lies outside from the nearest element)
  const char *const from = M.x;
  const int64_t to_row = flip ? (args.x_f32 ? 4 : 2) : x_pitch, to_col = flip ? x_pitch : (args.x_f32 ? 4 : 2);
  auto load = [&](auto fc) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x)
        X[j][x] = ortho_load(from + min(row_of(x), s - 1) * to_row + min(col0 + 32 * j + r, l - 1) * to_col, decltype(fc)::value, 0);
  };
  if (args.x_f32) load(std::true_type{});
  else load(std::false_type{});
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) X[j][x] = row_of(x) < s && col0 + 32 * j + r < l ? X[j][x] : 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) sum += (double)X[j][x] * (double)X[j][x];
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += part[w];
  __syncthreads();
  const double inv = !(sum <= 1.7976931348623157e308) ? __builtin_nan("") : sum > 0.0 ? ORTHO_SCALE / sqrt(sum) : 0.0;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int x = 0; x < 16; ++x) X[j][x] = (float)((double)X[j][x] * inv);
  asm volatile("" : "+v"(r), "+v"(g));
  __builtin_amdgcn_sched_barrier(0);

  // ---- between registers and areas -----------------------------------------------------------
  // (addresses are written so that all but a few exclusive ors of constants are offsets of the instructions)
  struct Pairs {
    OrthoPairs p[2][8];                                       // of elements 2 x, 2 x + 1: neighbouring rows of a column
  };
  auto split = [&](const nt_f32x16 (&v)[2]) {
    Pairs out;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 8; ++x) out.p[j][x] = ortho_split(v[j][2 * x], v[j][2 * x + 1]);
    return out;
  };
  // Lanes of an even and an odd column exchange halves of two rows, so that each stores two columns of one of them.
  auto put_rows = [&](unsigned area, const Pairs &v) {
    const unsigned base = area + ortho_area(row0 + 4 * g + (r & 1), col0 + (r & 30)), pick = r & 1 ? 0x07060302 : 0x01000504;
    auto turned = [&](ortho_h2 h) {
      const unsigned own = __builtin_bit_cast(unsigned, h);
      return __builtin_amdgcn_perm(own, (unsigned)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true), pick);   // lane ^ 1
    };
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 16; x += 2) {
        const OrthoPairs &p = v.p[j][x / 2];
        const int row = 8 * (x / 4) + x % 4, turn = ((row & 15) ^ (8 * j)) << 4;   // (32 columns on are 8 slots on)
        *(__attribute__((address_space(3))) unsigned *)((nt_lptr)(uintptr_t)(base ^ turn) + row * (ORTHO_SMALL * 4)) = turned(p.high);
        *(__attribute__((address_space(3))) unsigned *)((nt_lptr)(uintptr_t)(base ^ turn ^ 64) + row * (ORTHO_SMALL * 4)) = turned(p.low);
        if (x % 4 == 2) __builtin_amdgcn_sched_barrier(0);
      }
  };
  // (the transpose; four neighbouring rows of a column at a time)
  auto put_cols = [&](unsigned area, const Pairs &v) {
    const unsigned base = area + ortho_area(col0 + r, row0 + 4 * g);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const OrthoPairs &p = v.p[j][2 * x], &q = v.p[j][2 * x + 1];
        const ortho_h4 high = {p.high[0], p.high[1], q.high[0], q.high[1]}, low = {p.low[0], p.low[1], q.low[0], q.low[1]};
        *(__attribute__((address_space(3))) ortho_h4 *)((nt_lptr)(uintptr_t)(base ^ (x << 4)) + 32 * j * (ORTHO_SMALL * 4)) = high;
        *(__attribute__((address_space(3))) ortho_h4 *)((nt_lptr)(uintptr_t)(base ^ (x << 4) ^ 64) + 32 * j * (ORTHO_SMALL * 4)) = low;
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // rows row0 ... of `a` times rows col0 ... of `b`, inner length 64 or 128
  auto product = [&](unsigned a, unsigned b, int k, nt_f32x16 (&acc)[2]) {
    acc[0] = nt_f32x16{};
    acc[1] = nt_f32x16{};
    const unsigned base_a = a + ortho_area(row0 + r, 8 * g), base_b = b + ortho_area(col0 + r, 8 * g);
    auto get = [](unsigned at, int on) { return *(const __attribute__((address_space(3))) nt_f16x8 *)((nt_lptr)(uintptr_t)at + on); };
    struct Frag {
      nt_f16x8 ah, al, bh[2], bl[2];
    };
    auto read = [&](Frag &f, auto ac) {
      constexpr int AT = decltype(ac)::value * 16, SLOT = (AT >> 5) * 8 + ((AT & 31) >> 3), TURN = (SLOT & 15) << 4, ON = (SLOT & 16) << 4;
      f.al = get(base_a ^ TURN ^ 64, ON);
#pragma unroll
      for (int j = 0; j < 2; ++j) f.bh[j] = get(base_b ^ TURN, ON + 32 * j * (ORTHO_SMALL * 4));
      f.ah = get(base_a ^ TURN, ON);
#pragma unroll
      for (int j = 0; j < 2; ++j) f.bl[j] = get(base_b ^ TURN ^ 64, ON + 32 * j * (ORTHO_SMALL * 4));
    };
    // the fragments of 16 k are read while those in front of them are multiplied
    auto all = [&](auto nc) {
      constexpr int N = decltype(nc)::value;
      Frag f[2];
      read(f[0], std::integral_constant<int, 0>{});
      nt_for<N>([&](auto ac) {
        constexpr int I = decltype(ac)::value;
        const Frag &now = f[I & 1];
        if constexpr (I + 1 < N) read(f[(I + 1) & 1], std::integral_constant<int, I + 1>{});
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now.al, now.bh[j], acc[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now.ah, now.bl[j], acc[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now.ah, now.bh[j], acc[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    if (k > 64) all(std::integral_constant<int, 8>{});
    else all(std::integral_constant<int, 4>{});
  };

  // ---- the steps -------------------------------------------------------------------------------
  constexpr float UNIT = 1.f / ORTHO_SCALE;
  for (int step = 0; step < args.steps; ++step) {
    const float a = args.coefficients[3 * step], b = args.coefficients[3 * step + 1], c = args.coefficients[3 * step + 2];
    nt_f32x16 acc[2];
    // (behind every barrier the lane's number is new to the compiler, which else keeps 100 addresses from step to step)
    auto sync = [&]() {
      __syncthreads();
      asm volatile("" : "+v"(r), "+v"(g));
      __builtin_amdgcn_sched_barrier(0);
    };
    const Pairs x_pairs = split(X);
    put_rows(area1, x_pairs);
    sync();
    product(area1, area1, l, S);
#pragma unroll
    for (int j = 0; j < 2; ++j) S[j] *= UNIT;
    __builtin_amdgcn_sched_barrier(0);
    put_cols(area2, split(S));         // (symmetric)
    sync();
    put_cols(area1, x_pairs);
    product(area2, area2, s, acc);
    sync();
#pragma unroll
    for (int j = 0; j < 2; ++j) S[j] = b * S[j] + c * UNIT * acc[j];
    __builtin_amdgcn_sched_barrier(0);
    put_cols(area2, split(S));
    sync();
    product(area2, area1, s, acc);
#pragma unroll
    for (int j = 0; j < 2; ++j) X[j] = a * X[j] + UNIT * acc[j];
    sync();
  }
  char *const out = M.y;
  const int64_t out_row = flip ? (args.y_f32 ? 4 : 2) : y_pitch, out_col = flip ? y_pitch : (args.y_f32 ? 4 : 2);
  auto store = [&](auto fc) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int row = row_of(x), col = col0 + 32 * j + r;
        char *const to = out + row * out_row + col * out_col;
        if (row < s && col < l) {
          if constexpr (decltype(fc)::value) *(float *)to = X[j][x] * UNIT;
          else *(__bf16 *)to = (__bf16)(X[j][x] * UNIT);
        }
      }
  };
  if (args.y_f32) store(std::true_type{});
  else store(std::false_type{});
}

}  // namespace dmm
