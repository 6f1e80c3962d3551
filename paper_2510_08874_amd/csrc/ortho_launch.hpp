// Arguments and host-side doors of the kernels that orthogonalise a matrix (ortho_kernel.hpp), compiled in an
// object file of their own (ortho_instance.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dmm {

// A tile of an input or an output; travels with the launch.
struct OrthoTile {
  char *p;
  int64_t pitch;                // bytes
  int32_t row0, col0, h, w;     // where it lies in its matrix
  int32_t matrix;
  int32_t first_block, across;  // its workgroups begin here; as many side by side
  int32_t pad;                  // the norm: workgroups of the matrix' tiles in front of this one
};
constexpr int ORTHO_TILES = 64;
struct OrthoTiles {
  int32_t n, f32;               // tiles; fp32 or bf16
  int32_t rows, cols;
  int32_t row_pitch, col_pitch; // elements of a row of the two layouts: columns (rows) up to a multiple of 32
  int64_t stride;               // bytes from one matrix' buffers to the next
  char *ws;
  int64_t by_rows, by_cols;     // byte offsets: pairs [rows][row_pitch] and [cols][col_pitch]
  double *sums;                 // of squares, so many per matrix
  int32_t sums_of_launch, pad;
  OrthoTile tile[ORTHO_TILES];
};

// out = alpha old + beta sum over k of A[m][k] B[n][k].  All matrices are pairs of fp16: 32 values of a row are 64 bytes
// of high parts and 64 bytes of low parts.
struct OrthoProduct {
  char *ws;                     // what follows are byte offsets in a matrix' buffers
  int64_t stride;
  int64_t a, b;
  int64_t old;                  // out's rows and pitch; none: < 0
  int64_t out;
  int64_t turned;               // out transposed, none: < 0
  int64_t y;                    // the last product: out goes here alone, in fp32; else < 0
  uint32_t k_pitch_a, k_pitch_b;   // bytes
  uint32_t out_pitch, turned_pitch;   // elements (4 bytes)
  int32_t m, n;                 // out: m x n (columns up to out_pitch are zero, and rows up to turned_pitch)
  int32_t steps;                // 32 of k each
  int32_t y_turned;             // ... transposed
  int32_t symmetric;            // out is: tiles below the diagonal come from those above
  int32_t count, tiles, tiles_m, tiles_n;   // matrices; tiles of each, in rows and columns
  int32_t whole;                // tiles (of all matrices) that are not cut; the others in `runs` ranges of K,
  int32_t runs, per;            // steps of each
  float *parts;
  float alpha, beta;
};

// Matrices of up to 128 x 128, one workgroup each, whole in registers and LDS.
constexpr int ORTHO_SMALL = 128;
constexpr int ORTHO_MATRICES = 144, ORTHO_STEPS = 32;
struct OrthoSmall {
  int32_t rows, cols, steps;
  int32_t x_f32, y_f32;
  float coefficients[3 * ORTHO_STEPS];
  int32_t even;                 // matrices lie at even distances: matrix[0] tells where the first is, matrix[1] the second
  struct {
    const char *x;
    char *y;
    uint32_t x_ld, y_ld;        // elements
  } matrix[ORTHO_MATRICES];
};
void ortho_small_launch(const OrthoSmall &args, int count, hipStream_t stream);

hipError_t ortho_allow_lds();
void ortho_norm_launch(const OrthoTiles &args, int blocks, hipStream_t stream);
void ortho_split_launch(const OrthoTiles &args, int blocks, hipStream_t stream);
// y: fp32 matrices one behind another in by_rows' place -> the tiles
void ortho_store_launch(const OrthoTiles &args, int blocks, hipStream_t stream);
void ortho_product_launch(const OrthoProduct &args, int edge, hipStream_t stream);   // edge of a tile: 64, 128 or 256

}  // namespace dmm
