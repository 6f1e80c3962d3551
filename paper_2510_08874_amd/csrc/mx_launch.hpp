// Tables and host-side doors of the kernels for 4-bit microscaled matrices (mx_kernel.hpp), compiled in an
// object file of their own (mx_instance.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dmm {

// A run of K on which both operands lie in one piece.  The pointers name row 0 of the product's rows (columns) at
// the run's first chunk (64 bytes of a row); scales only where there are any (4 bytes of a row and chunk).
struct NtSeg {
  const char *a, *b, *a_scale, *b_scale;
  uint32_t a_pitch, b_pitch, a_scale_pitch, b_scale_pitch;   // bytes
  int32_t chunks;
  int32_t pad;
};

// A macro-tile of a product, or a run of its K whose partial sums go to a slot of scratch memory.
struct MxItem {
  NtSeg front;                  // segment `seg`, so that the first loads wait for one read of a table and not for two
  char *c;                      // its corner
  int64_t ldc;                  // elements
  int32_t m_off, n_off;         // first row and column inside the output sub-tile that the segments are given for
  int32_t m_ext, n_ext;
  int32_t seg, n_segs;          // from the segment that holds its first step; none: zeros
  int32_t first, steps;         // first step (two chunks, 256 of k) in that segment; how many in all
  int32_t c_es;                 // bytes of an element of C: 4, or 2 for bf16
  int32_t pad;
};

struct MxJoin {
  char *c;
  int64_t ldc;
  const float *parts;           // `runs` slots of tm x tn
  int32_t runs, tm, tn, m_ext, n_ext, c_es;
};

// A tile that is quantised, or whose values are written.
struct MxTile {
  char *x;
  int64_t x_pitch;              // bytes, like the others
  char *row_codes, *col_codes;
  unsigned char *row_scales, *col_scales;
  int64_t row_pitch, col_pitch, row_scale_pitch, col_scale_pitch;
  int32_t h, w;
  int32_t first_block, blocks_across;   // its workgroups begin here; as many side by side
};
// Travels as the kernel's argument: the call needs no memory of its own and no copy.
constexpr int MX_TILES = 32;
struct MxTileArgs {
  int32_t n, pad;
  MxTile tile[MX_TILES];
};

enum { MX_256, MX_128, MX_64, MX_32, MX_SKINNY, MX_SHAPES };
struct MxShape {
  int tm, tn;
};
constexpr MxShape kMxShape[MX_SHAPES] = {{256, 256}, {128, 128}, {64, 128}, {32, 128}, {16, 16}};

enum { MX_ALONG_ROWS = 1, MX_ALONG_COLS = 2 };
constexpr int mx_block_cols(bool f32) { return f32 ? 64 : 128; }   // 128 rows of so many columns a workgroup, along the columns

hipError_t mx_allow_lds();
bool mx_launch(hipEvent_t behind, int shape, const MxItem *items, int n_items, const NtSeg *segs, const MxJoin *joins, int n_joins, int cus, hipStream_t stream);
// rows that a wave takes at a time, when there are `units` pieces of 512 columns of a row in all
int mx_rows_per_unit(int64_t units);
void mx_quantize_launch(const MxTileArgs &args, int blocks, bool f32, int along, int rows_per_unit, hipStream_t stream);
void mx_values_launch(const MxTileArgs &args, int blocks, bool f32, int along, int rows_per_unit, hipStream_t stream);

}  // namespace dmm
