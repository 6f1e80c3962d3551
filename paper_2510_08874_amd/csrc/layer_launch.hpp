// Tables and host-side doors of the kernels for the layers around a product (layer_kernel.hpp): products of 8-bit
// integers, the gated block, the gradients of bf16 products.  Compiled in object files of their own (layer_instance.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dmm {

// A run of K on which both operands lie in one piece.  An operand that lies along K ("direct") is named by its row 0 at the run's
// first k; one that lies across K ("turned") by its first k row at the product's row (column) 0.  b2: the second right operand of a
// gated product.  Pitches in bytes, below 2^24.
struct LayerSeg {
  const char *a, *b, *b2;
  uint32_t a_pitch, b_pitch, b2_pitch;
  int32_t steps;                // whole steps of K: 128 bytes of a direct row, i.e. 64 bf16 or 128 integers
  int32_t tail;                 // elements behind them, up to a step's; read one by one where they end
  int32_t pad;
};

// What becomes of a finished tile.
enum { LAYER_STORE, LAYER_PARTS, LAYER_ZERO };

// A macro-tile of a product, or a run of its K whose partial sums go to a slot of scratch memory.
struct LayerItem {
  LayerSeg front;               // segment `seg`, so that the first loads wait for one read of a table and not for two
  char *c;                      // its corner (LAYER_PARTS: its slot)
  int64_t ldc;                  // elements
  char *g, *u;                  // gated: corners of what is kept of both products (none: null)
  int64_t ldg, ldu;
  const float *sa, *sb, *sb2;   // integers: scales of its rows and columns
  int32_t m_off, n_off;         // first row and column inside the output sub-tile that the segments are given for
  int32_t m_ext, n_ext;
  int32_t seg, n_segs;          // from the segment that holds its first whole step
  int32_t first, steps;         // first whole step in that segment; how many in all
  int32_t tail_seg, n_tails;    // segments whose tails it adds
  int32_t c_es;                 // bytes of an element of C: 4, or 2 for bf16
  int32_t what;                 // LAYER_*
  int32_t kind, pad;            // of product, where a launch has two
};

struct LayerJoin {
  char *c;
  int64_t ldc;
  char *g, *u;
  int64_t ldg, ldu;
  const float *sa, *sb, *sb2;
  const char *parts;            // `runs` slots of tm x tn
  int32_t runs, tm, tn, m_ext, n_ext, c_es;
};

// Rows of a tile on their way into a dense copy of its matrix; without a source, zeros.
struct LayerCopy {
  const char *src;
  char *dst;
  int64_t src_pitch, dst_pitch; // bytes
  int32_t rows, bytes;          // of a row
  int32_t first_block, pad;
};
constexpr int LAYER_COPY_CHUNKS = 2048;   // of 16 bytes, a workgroup
void layer_copy_launch(const LayerCopy *jobs, int n, int blocks, hipStream_t stream);

// Elements and operands of a product.
enum {
  LAYER_I8,                     // C = A B, both direct
  LAYER_I8_GATED,
  LAYER_GATED,                  // bf16, A direct, both right operands turned
  LAYER_NT,                     // bf16, both direct
  LAYER_TN,                     // bf16, both turned
  LAYER_KINDS,
  LAYER_PAIR = LAYER_KINDS      // a launch of both gradients' macro-tiles of 128 x 128
};
// Macro-tiles of a kind: rows by columns of the result.
enum { LAYER_256, LAYER_128, LAYER_TWO, LAYER_64, LAYER_32, LAYER_SHAPES };   // (TWO: gated, small enough for two on a CU)
struct LayerTile {
  int tm, tn;
};
constexpr LayerTile kLayerTile[LAYER_KINDS][LAYER_SHAPES] = {
    {{256, 256}, {128, 128}, {0, 0}, {64, 128}, {32, 128}},
    {{256, 128}, {128, 128}, {128, 64}, {64, 128}, {32, 128}},
    {{256, 128}, {128, 128}, {64, 128}, {64, 128}, {32, 128}},
    {{256, 256}, {128, 128}, {0, 0}, {64, 128}, {32, 128}},
    {{256, 256}, {128, 128}, {0, 0}, {0, 0}, {0, 0}},
};
constexpr bool layer_gated(int kind) { return kind == LAYER_I8_GATED || kind == LAYER_GATED; }
constexpr bool layer_i8(int kind) { return kind == LAYER_I8 || kind == LAYER_I8_GATED; }
constexpr int layer_step(int kind) { return layer_i8(kind) ? 128 : 64; }   // of K

hipError_t layer_allow_lds();
bool layer_launch(hipEvent_t behind, int kind, int shape, int act, int cus, const LayerItem *items, int n_items, const LayerSeg *segs, const LayerJoin *joins,
                  int n_joins, hipStream_t stream);

// per kind, in object files of their own
#define DMM_DECLARE_LAYER(n)      \
  hipError_t layer_allow_lds_##n(); \
  bool layer_launch_##n(hipEvent_t behind, int shape, int act, int cus, const LayerItem *items, int n_items, const LayerSeg *segs, hipStream_t stream);
DMM_DECLARE_LAYER(0)
DMM_DECLARE_LAYER(1)
DMM_DECLARE_LAYER(2)
DMM_DECLARE_LAYER(3)
DMM_DECLARE_LAYER(4)
#undef DMM_DECLARE_LAYER
bool layer_launch_pair(hipEvent_t behind, int cus, const LayerItem *items, int n, const LayerSeg *segs, hipStream_t stream);

// ---- element by element ---------------------------------------------------------------------------------

// A tile of G, U, dH, dG and dU.
struct SlopeTile {
  const char *g, *u, *dh;
  char *dg, *du;
  int64_t pg, pu, ph, pdg, pdu;  // bytes from row to row
  int32_t h, w;
  int32_t first_block, pad;
};
constexpr int SLOPE_TILES = 32;
struct SlopeArgs {
  int32_t n, act;
  SlopeTile tile[SLOPE_TILES];
};
constexpr int SLOPE_CHUNKS = 1024;                // of eight elements of a row, a workgroup
void slope_launch(const SlopeArgs &args, int blocks, hipStream_t stream);

// ---- 8-bit integers -------------------------------------------------------------------------------------

// A tile that is quantised, or whose values are written.
struct I8Tile {
  char *x, *q;
  int64_t x_pitch, q_pitch;      // bytes
  float *scale;                  // of its rows, or its columns
  int32_t h, w;
  int32_t first_block, blocks_across;
};
constexpr int I8_TILES = 48;
struct I8Args {
  int32_t n, pad;
  I8Tile tile[I8_TILES];
};
// The scales of a matrix: pieces that are cleared, or turned from magnitudes into scales.
struct I8Scales {
  float *at;
  int32_t n, first_block;
};
constexpr int I8_PIECES = 240;
struct I8ScaleArgs {
  int32_t n, pad;
  I8Scales piece[I8_PIECES];
};
// A tile of such a row of tiles.
struct I8RowPiece {
  const char *x;
  char *q;
  int64_t x_pitch, q_pitch;
  int32_t w, first;              // columns; vectors of eight of the tiles in front
};
// A row of tiles whose rows are quantised whole: its tiles are I8RowArgs::piece[first_piece ...], n of them.
struct I8RowGroup {
  float *scale;
  int32_t first_block, first_piece;
};
constexpr int I8_ROW_GROUPS = 24, I8_ROW_PIECES = 64, I8_ROW_CUTS = 32, I8_ROW_THREADS = 1024, I8_ROW_KEPT = 4;
struct I8RowArgs {
  int32_t groups, n;
  int32_t vectors, pad;          // of a row
  I8RowGroup group[I8_ROW_GROUPS];
  I8RowPiece piece[I8_ROW_PIECES];
};
enum { I8_CLEAR, I8_FINISH };
void i8_scales_launch(const I8ScaleArgs &args, int blocks, int what, hipStream_t stream);
// blocks of 128 rows by 256 bytes (i8_block_cols columns)
constexpr int i8_block_cols(bool f32) { return f32 ? 64 : 128; }
void i8_amax_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream);
void i8_quantize_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream);
void i8_values_launch(const I8Args &args, int blocks, bool f32, bool cols, hipStream_t stream);
void i8_whole_cols_launch(const I8Args &args, int blocks, bool f32, hipStream_t stream);   // columns of no more rows than a block has
void i8_whole_rows_launch(const I8RowArgs &args, int blocks, int threads, bool f32, hipStream_t stream);

}  // namespace dmm
