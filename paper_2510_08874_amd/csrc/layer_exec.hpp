// The entry points for the layers around a product (included by exec.hip): 8-bit integers, the gated block, the gradients of bf16
// products.  Arguments are checked here; what a product reads and writes is laid out as groups (an output sub-tile and its segments of K),
// cut into macro-tiles by one routine whatever the kind.
#pragma once

namespace dmm {
namespace {

constexpr int64_t kLayerBlocks = (1 << 24) - 1;                // workgroups of a launch: 2^32 threads are too many
constexpr int64_t kLayerManyRows = 1024;                           // rows that fill the device with small workgroups
constexpr int64_t kLayerPitch = (int64_t)1 << 24;              // bytes from row to row
constexpr int64_t kLayerRows = 0x7fff0000;                     // kernels count rows and columns in 32 bits, a workgroup's past the last among them
constexpr int64_t kLayerSum = 131071;                          // products of two bytes that an int32 sum holds whatever they are

int allow_layer_lds() {
  static std::mutex mu;
  static bool done[64] = {};
  int device = 0;
  DMM_HIP(hipGetDevice(&device));
  if (device < 0 || device >= 64) return DMM_EINVAL;
  std::lock_guard<std::mutex> g(mu);
  if (!done[device]) {
    DMM_HIP(layer_allow_lds());
    done[device] = true;
  }
  return DMM_OK;
}

// The tiles of a matrix: buffers aligned to their elements, leading dimensions that hold a row and stay below kLayerPitch.
int check_layer_tiles(const Grid &G, const dmm_tiles *t, int es) {
  if (!t->tiles || !t->ld) return DMM_EINVAL;
  int rc;
  if ((rc = check_lds(G, t->ld)) || (rc = check_tiles(G, t->tiles, es))) return rc;
  for (int32_t rep = 0; rep < G.c; ++rep)
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj)
        if (G.rc[ti + 1] > G.rc[ti] && G.cc[tj + 1] > G.cc[tj] && t->ld[G.table_index(rep, ti, tj)] >= kLayerPitch / es) return DMM_ELD;
  return DMM_OK;
}
// One replica's, whatever the matrix has.  (The copy takes host memory.)
int check_layer_single(const Grid &G, const dmm_tiles *t, int es) {
  Grid one = G;
  one.c = 1;
  return check_layer_tiles(one, t, es);
}
int check_sizes(const dmm_plan_t *P) { return std::max({P->A.rows, P->A.cols, P->B.cols}) > kLayerRows ? DMM_ELIMIT : DMM_OK; }
// 8-bit integers along the rows, or along the columns, where a tile lies transposed.
int check_i8(const Grid &G, const dmm_int_tiles *q, bool by_cols) {
  if (!q->codes || !q->code_ld || !q->scales) return DMM_EINVAL;
  for (int32_t rep = 0; rep < G.c; ++rep) {
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t h = G.rc[ti + 1] - G.rc[ti], w = G.cc[tj + 1] - G.cc[tj];
        if (h <= 0 || w <= 0) continue;
        const int64_t i = G.table_index(rep, ti, tj);
        if (!q->codes[i]) return DMM_EINVAL;
        if (q->code_ld[i] < (by_cols ? h : w) || q->code_ld[i] >= kLayerPitch) return DMM_ELD;
      }
    const int32_t n = by_cols ? G.gc : G.gr;
    for (int32_t t = 0; t < n; ++t) {
      const int64_t len = by_cols ? G.cc[t + 1] - G.cc[t] : G.rc[t + 1] - G.rc[t];
      const void *s = q->scales[(int64_t)rep * n + t];
      if (len > 0 && (!s || ((uintptr_t)s & 3))) return DMM_EINVAL;
    }
  }
  return DMM_OK;
}

// ---- groups -------------------------------------------------------------------------------------------

struct LayerGroup {
  int64_t m, n;                        // extents
  size_t seg, n_segs;
  char *c, *g, *u;                     // corners
  int64_t ldc, ldg, ldu;
  const float *sa, *sb, *sb2;
};

struct LayerWork {
  int kind = 0, act = DMM_SILU, c_es = 4;
  int64_t rows = 1;                    // of the whole result
  std::vector<LayerSeg> segs;
  std::vector<LayerGroup> groups;
};

// Of a turned operand whose rows are `ld` elements apart: how many of a tile's last `rows` rows below k1 a read of eight columns at a time could
// take past the end of its buffer, where the columns end with the tile.
int64_t rows_past_end(int64_t tile_rows, int64_t tile_cols, int64_t ld, int64_t k1, int64_t col0, int64_t cols) {
  const int64_t over = col0 + (cols + 7) / 8 * 8 - tile_cols;
  if (over <= 0) return 0;
  return std::max<int64_t>(0, (over + ld - 1) / ld - (tile_rows - k1));
}

// Whole steps of a segment of `len`, and what is left; the last `guard` rows are not to be part of whole steps.
void put_segment(LayerWork *W, LayerSeg s, int64_t len, int64_t guard) {
  const int64_t step = layer_step(W->kind);
  int64_t steps = len / step, tail = len % step;
  s.pad = 0;
  if (tail < guard && steps > 0) {
    s.steps = (int32_t)(steps - 1);
    s.tail = (int32_t)step;
    W->segs.push_back(s);
    if (tail == 0) return;
    // (an operand on a copy is named by its place, which may be 0)
    auto on = [&](const char *p, uint32_t pitch, bool turned) { return (const char *)((uintptr_t)p + (uintptr_t)(turned ? steps * step * (int64_t)pitch : steps * 128)); };
    const bool bt = W->kind == LAYER_TN || W->kind == LAYER_GATED;
    s.a = on(s.a, s.a_pitch, W->kind == LAYER_TN);
    s.b = on(s.b, s.b_pitch, bt);
    if (layer_gated(W->kind)) s.b2 = on(s.b2, s.b2_pitch, bt);
    steps = 0;
  }
  s.steps = (int32_t)steps;
  s.tail = (int32_t)tail;
  W->segs.push_back(s);
}

int64_t up_to(int64_t n, int64_t step) { return (n + step - 1) / step * step; }

struct LayerChoice {
  int shape = LAYER_256;
  int64_t runs = 1;
  double us = 0;
  // what an estimate of two products together needs: steps and tails of a tile's K, macro-tiles of 128 x 128, how long memory takes
  double steps = 0, tails = 0, tiles = 0, memory = 0;
};

// Which operands of a product are read from copies; LAYER_ROWS: the left one, and results go through scratch memory as well.
enum LayerDense { LAYER_IN_PLACE, LAYER_BOTH, LAYER_LEFT, LAYER_ROWS };

// Dense copies of operands whose rows are misaligned or finely cut (8-bit gated 2501 x 1999 x 1777 in 15 uneven blocks: 93 us in place, 42 with 10 for the
// copies; gradients of 1999 x 2731 x 1021 87 and 52): every row starts at a multiple of 128 bytes, K is one segment of whole steps,
// filled up with zeros.  Places are given out from 0 on; the buffer is known later.
struct LayerCopies {
  std::vector<LayerCopy> jobs, back;   // in front of the product, behind it
  size_t size = 0;
  double bytes = 0;
  int64_t blocks = 0, back_blocks = 0;
  bool fits = true;                    // rows are not too long for the kernels
  struct Matrix {
    size_t at;
    int64_t pitch;
  };
  struct Made {
    const void *tiles, *ld;
    const Grid *grid;
    Matrix m;
  };
  std::vector<Made> made;              // two products may read one copy

  // rows x row_bytes bytes from `src` to place `dst`
  void job(const void *src, int64_t src_pitch, size_t dst, int64_t dst_pitch, int64_t rows, int64_t row_bytes) {
    if (rows <= 0 || row_bytes <= 0) return;
    LayerCopy j;
    std::memset(&j, 0, sizeof j);
    j.src = (const char *)src;
    j.dst = (char *)(uintptr_t)dst;
    j.src_pitch = src_pitch;
    j.dst_pitch = dst_pitch;
    j.rows = (int32_t)rows;
    j.bytes = (int32_t)row_bytes;
    j.first_block = (int32_t)blocks;
    blocks += ((row_bytes + 15) / 16 * rows + LAYER_COPY_CHUNKS - 1) / LAYER_COPY_CHUNKS;
    jobs.push_back(j);
    bytes += (double)rows * (double)row_bytes * (src ? 2 : 1);
  }
  // Results of `es` bytes in dense rows, and their way into the tiles from there.
  Matrix results(const Grid &G, const dmm_tiles *t, int es) {
    const Matrix m = {size, (G.cols * es + 127) / 128 * 128 | 128};
    if (m.pitch >= kLayerPitch) fits = false;
    size += (size_t)(G.rows * m.pitch + 4095) / 4096 * 4096;
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t i = G.table_index(0, ti, tj), r0 = G.rc[(size_t)ti], c0 = G.cc[(size_t)tj], rows = G.rc[(size_t)ti + 1] - r0, w = G.cc[(size_t)tj + 1] - c0;
        if (rows <= 0 || w <= 0) continue;
        LayerCopy j;
        std::memset(&j, 0, sizeof j);
        j.src = (const char *)(uintptr_t)(m.at + (size_t)(r0 * m.pitch + c0 * es));
        j.dst = (char *)t->tiles[i];
        j.src_pitch = m.pitch;
        j.dst_pitch = t->ld[i] * es;
        j.rows = (int32_t)rows;
        j.bytes = (int32_t)(w * es);
        j.first_block = (int32_t)back_blocks;
        back_blocks += ((w * es + 15) / 16 * rows + LAYER_COPY_CHUNKS - 1) / LAYER_COPY_CHUNKS;
        back.push_back(j);
        bytes += 2.0 * (double)rows * (double)w * es;
      }
    return m;
  }
  // Where the columns of a matrix lie in its copy: those from every cut on start at a multiple of 128 bytes, so that macro-tiles that begin there read
  // aligned rows.
  struct Axis {
    std::vector<int64_t> cuts, at;
    int64_t total = 0;                 // columns of the copy
    Axis(const std::vector<int64_t> &c, int64_t step) : cuts(merged_cuts({&c})) {
      for (size_t i = 0; i + 1 < cuts.size(); ++i) {
        at.push_back(total);
        total += (cuts[i + 1] - cuts[i] + step - 1) / step * step;
      }
    }
    int64_t place(int64_t col) const {
      const size_t i = (size_t)(std::upper_bound(cuts.begin(), cuts.end(), col) - cuts.begin()) - 1;
      return at[i] + col - cuts[i];
    }
  };
  // Replica 0 of a matrix, `rows` rows and the columns of `axis` to be there in the end, zeros where the matrix has none (`zeros`; otherwise what lies between the
  // columns is left as it is).  `turned`: its tiles lie transposed, and so does the copy.
  Matrix matrix(const Grid &G, const void *const *tiles, const int64_t *ld, int es, bool turned, int64_t rows, const Axis &axis, bool zeros) {
    for (const Made &other : made)
      if (other.tiles == tiles && other.ld == ld && other.grid == &G) return other.m;
    const int64_t have_rows = turned ? G.cols : G.rows;
    const int64_t pitch = (axis.total * es + 127) / 128 * 128 | 128;   // (an odd number of lines: rows start in different channels)
    const Matrix m = {size, pitch};
    if (pitch >= kLayerPitch || rows > 0x7fffff00) fits = false;
    size += (size_t)(rows * pitch + 128 + 4095) / 4096 * 4096;   // (a read of eight columns may pass the last row's end)
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t r0 = turned ? G.cc[(size_t)tj] : G.rc[(size_t)ti], r1 = turned ? G.cc[(size_t)tj + 1] : G.rc[(size_t)ti + 1];
        const int64_t c0 = turned ? G.rc[(size_t)ti] : G.cc[(size_t)tj], c1 = turned ? G.rc[(size_t)ti + 1] : G.cc[(size_t)tj + 1];
        const int64_t i = G.table_index(0, ti, tj);
        for (size_t x = 0; x + 1 < axis.cuts.size(); ++x) {
          const int64_t lo = std::max(c0, axis.cuts[x]), hi = std::min(c1, axis.cuts[x + 1]);
          if (r1 > r0 && hi > lo)
            job((const char *)tiles[i] + (lo - c0) * es, ld[i] * es, m.at + (size_t)(r0 * pitch + axis.place(lo) * es), pitch, r1 - r0, (hi - lo) * es);
        }
      }
    for (size_t x = 0; zeros && x + 1 < axis.cuts.size(); ++x) {
      const int64_t end = axis.at[x] + axis.cuts[x + 1] - axis.cuts[x], next = x + 1 < axis.at.size() ? axis.at[x + 1] : axis.total;
      job(nullptr, 0, m.at + (size_t)(end * es), pitch, have_rows, (next - end) * es);
    }
    job(nullptr, 0, m.at + (size_t)(have_rows * pitch), pitch, rows - have_rows, axis.total * es);
    made.push_back({tiles, ld, &G, m});
    return m;
  }
  // scales of replica 0, one behind another
  size_t scales(const std::vector<int64_t> &cuts, const float *const *s) {
    const size_t at = size;
    size += (size_t)(cuts.back() * 4 + 4095) / 4096 * 4096;
    for (size_t i = 0; i + 1 < cuts.size(); ++i) job(s[i], 0, at + (size_t)cuts[i] * 4, 0, 1, (cuts[i + 1] - cuts[i]) * 4);
    return at;
  }
  double us() const { return (back.empty() ? 4.0 : 8.0) + bytes / 4.0e6; }
  bool possible() const;
};
constexpr double kTail = 5;                                    // us, see choose_layer
constexpr size_t kLayerCopies = (size_t)1 << 30;               // of a product
bool LayerCopies::possible() const { return fits && size <= kLayerCopies && blocks <= kLayerBlocks && back_blocks <= kLayerBlocks; }


// The macro-tile, and into how many runs K is cut, with the shortest estimate in us, from measured steps (128 bytes of K): for every shape a step's time with
// few workgroups and what it grows by until all CUs have one, and a tile's ends.  Where rows are not aligned to 16 bytes a step takes a quarter more (integers a
// third: 8191^3 direct 625 us, on copies 497; aligned 423; gated 40 and 45 %), what is left of a segment 5 us whatever the shape.  Both sides of what it decides:
//   gated, 8 bits, 2501 x 512 x 1777     two on a CU 14.3, 256 x 128 19.2          4096 x 4096 x 8192    265 and 237
//   gated, bf16, 256 x 2048 x 2048       two on a CU 18.6, 128 x 128 24.6          1024 x 4096 x 4096    73 and 58
//   8 bits, 2048^3                       128 x 128 13.4, 256 x 256 27.8            4096 x 4096 x 8192    136 and 117
//   gated, bf16, 128 x 8192 x 4096       K in four runs 37, whole 64               1 x 8192 x 28672 in 8 bits: 43 and 36 (B is in a cache), whole
// `fixed`: the runs are given, and a macro-tile is looked for.
LayerChoice choose_layer(const LayerWork &W, int cus, int64_t fixed = 0) {
  const bool gated = layer_gated(W.kind);
  double cells = 0, k_steps = 0, k_tails = 0, b_once = 0;
  int64_t most = 0;
  for (const LayerGroup &g : W.groups) {
    most = std::max(most, g.m);
    double steps = 0, tails = 0, bytes = 0;
    for (size_t x = g.seg; x < g.seg + g.n_segs; ++x) {
      const LayerSeg &s = W.segs[x];
      const bool odd = (((uintptr_t)s.a | (uintptr_t)s.b | (uintptr_t)s.b2 | s.a_pitch | s.b_pitch | s.b2_pitch) & 15) != 0;
      steps += s.steps * (!odd ? 1.0 : gated ? (layer_i8(W.kind) ? 1.45 : 1.4) : layer_i8(W.kind) ? 1.35 : 1.25);
      tails += s.tail > 0;
      bytes += s.steps + (s.tail > 0);
    }
    const double area = (double)g.m * (double)g.n;
    cells += area;
    k_steps += area * steps;
    k_tails += area * tails;
    b_once += area / (double)W.rows * bytes * (gated ? 256.0 : 128.0);
  }
  const double steps = cells > 0 ? std::max(1.0, k_steps / cells) : 1, tails = cells > 0 ? k_tails / cells : 0;
  LayerChoice best;
  best.runs = fixed ? fixed : 1;
  best.steps = steps;
  best.tails = tails;
  double best_us = 0;
  for (int shape = 0; shape < LAYER_SHAPES; ++shape) {
    const int tm = kLayerTile[W.kind][shape].tm, tn = kLayerTile[W.kind][shape].tn;
    if (tm == 0 || (shape == LAYER_64 && most > 128) || (shape == LAYER_32 && most > 64)) continue;
    double tiles = 0, strips = 0;                              // strips: columns of B that rows of tiles read, in all
    for (const LayerGroup &g : W.groups) {
      tiles += (double)(((g.m + tm - 1) / tm) * ((g.n + tn - 1) / tn));
      strips += (double)((g.m + tm - 1) / tm) * (double)g.n;
    }
    if (tiles == 0) return best;
    if (tiles > (double)kLayerBlocks) continue;
    // (two workgroups on a CU where the stages leave room)
    const int places = shape == LAYER_TWO || (!gated && shape != LAYER_256) ? 2 * cus : cus;
    // B from memory; another row of tiles reads it from a cache (48 x 8192 x 28672 gated, integers: 85 us on tiles of 64 rows, 103 on those of 32)
    const double down = strips * (double)W.rows / std::max(cells, 1.0);
    if (shape == LAYER_128) best.tiles = tiles;
    const double memory = 2.0 + b_once * (0.8 + 0.2 * down) / 5.4e6;
    for (int64_t runs = fixed ? fixed : 1; runs <= (fixed ? fixed : 32); ++runs) {
      const double work = tiles * (double)runs, per = std::ceil(steps / (double)runs);
      if (!fixed && runs > 1 && (work > places || per < 3)) break;
      auto round = [&](double n) {
        if (n <= 0) return 0.0;
        const double full = n / cus, ends = kTail * tails / (double)runs;
        switch (shape) {
          case LAYER_256: return ends + per * (1.15 + 0.3 * full) + (W.kind == LAYER_I8_GATED ? 12.0 : 9.0);
          case LAYER_128: return ends + (gated ? per * ((layer_i8(W.kind) ? 0.62 : 0.5) + 0.3 * full) + 6.5 : per * (full > 1 ? 1.1 : 0.5 + 0.16 * full) + 5.0);
          case LAYER_TWO: return ends + per * (full > 1 ? (layer_i8(W.kind) ? 0.93 : 1.07) : 0.36 + 0.18 * full) + 4.5;
          case LAYER_64: return ends + (gated ? per * (0.42 + 0.2 * full) + 5.0 : per * (full > 1 ? 1.0 : 0.35 + 0.25 * full) + 4.0);
          default: return ends + (gated ? per * (0.38 + 0.15 * full) + 4.0 : per * (full > 1 ? 0.9 : 0.3 + 0.2 * full) + 3.5);
        }
      };
      const double whole = std::floor(work / places);
      double us = std::max(whole * round(places) + round(work - whole * places), memory);
      if (runs > 1) us += 4.5 + 2.0 * work * tm * tn * (gated ? 2 : 1) * 4 / 3e6;
      // (of equal estimates, as where memory bounds all of them, the smaller tile's)
      if (best_us == 0 || us < best_us || (us == best_us && shape != best.shape)) best_us = best.us = us, best.shape = shape, best.runs = runs, best.memory = memory;
    }
  }
  return best;
}

// Both gradients in one launch of macro-tiles of 128 x 128, each with its own runs of K (what a product is asked for with does not change its bits).  Both sides,
// gated backward: 2501 x 1999 x 1777 uneven 145 us in two launches, 126 in one; 2048^3 84 and 81; 1448 x 512 x 768 in row blocks 52 and 36; 4096^3 452 and 522.
double pair_us(const LayerChoice *c, int cus) {
  double n = 0, busy = 0, longest = 0, us = 0;
  for (int x = 0; x < 2; ++x) n += c[x].tiles * (double)c[x].runs;
  const double full = n / cus;
  for (int x = 0; x < 2; ++x) {
    const double per = std::ceil(c[x].steps / (double)c[x].runs), ends = kTail * c[x].tails / (double)c[x].runs, work = c[x].tiles * (double)c[x].runs;
    busy += work * (0.45 * per + 2.0 + 0.4 * ends) / cus;
    longest = std::max(longest, per * (full > 1 ? 0.8 : 0.5 + 0.16 * full) + 5.0 + ends);
    if (c[x].runs > 1) us += 4.5 + 2.0 * work * 128 * 128 * 4 / 3e6;
  }
  // (rounds are not full: a third of the longest tile; a launch less, with its start and its last tiles)
  const double rounds = full > 1 ? busy + 0.3 * (longest - 5.0) : longest;
  return us - 7.0 + std::max({rounds, longest, c[0].memory + c[1].memory});
}

// Tables of one product, appended to `h`; partial sums in slots of M's buffer, which have addresses from 0 on until place_parts.
int lay_out(const LayerWork &W, const LayerChoice &choice, std::vector<char> *h, LayerLayout *L, size_t *scratch) {
  *L = LayerLayout();
  L->kind = W.kind;
  L->act = W.act;
  const int shape = choice.shape, tm = kLayerTile[W.kind][shape].tm, tn = kLayerTile[W.kind][shape].tn;
  const bool gated = layer_gated(W.kind);
  const int wide = gated ? 2 * tn : tn;                        // columns of a slot
  const size_t slot_bytes = (size_t)tm * wide * 4;
  std::vector<LayerItem> items;
  std::vector<LayerJoin> joins;
  int64_t slots = 0;
  for (const LayerGroup &g : W.groups) {
    const int64_t rows = (g.m + tm - 1) / tm, cols = (g.n + tn - 1) / tn;
    int64_t whole = 0, k = 0;
    for (size_t s = g.seg; s < g.seg + g.n_segs; ++s) {
      whole += W.segs[s].steps;
      k += W.segs[s].steps * (int64_t)layer_step(W.kind) + W.segs[s].tail;
    }
    if (whole > 0x3fffffff || W.segs.size() > 0x3fffffff) return DMM_ELIMIT;
    int64_t runs = std::min<int64_t>(choice.runs, std::max<int64_t>(1, whole / 3));
    if (layer_i8(W.kind) && k > kLayerSum) runs = std::max<int64_t>(runs, (k + kLayerSum / 2 - 1) / (kLayerSum / 2));
    const int64_t per = std::max<int64_t>(1, (whole + runs - 1) / runs);
    runs = std::max<int64_t>(1, (whole + per - 1) / per);
    const int64_t first_slot = slots;
    size_t seg = g.seg, tail = g.seg;
    int64_t first = 0, done = 0;                               // steps into `seg`; steps of the segments whose tails have been given out
    for (int64_t run = 0; run < runs; ++run) {
      const int64_t n_steps = std::min(per, whole - run * per);
      while (seg < g.seg + g.n_segs && first >= W.segs[seg].steps) first -= W.segs[seg++].steps;
      // a segment's tail goes to the run that has its last whole step
      const size_t tail0 = tail;
      int64_t sum = n_steps * layer_step(W.kind);
      while (tail < g.seg + g.n_segs && (run == runs - 1 || done + W.segs[tail].steps <= (run + 1) * per)) {
        done += W.segs[tail].steps;
        sum += W.segs[tail++].tail;
      }
      if (layer_i8(W.kind) && sum > kLayerSum) return DMM_ELIMIT;
      // Blocks of 32 neighbours that share operands, eight tile rows by four tile columns, and the same columns of the eight rows below next, so that eight
      // blocks are 16 by 16 tiles.  All first ranges of K, then all second ones, ...
      int64_t tile = 0;
      for (int64_t r0 = 0; r0 < rows; r0 += 16) {
        const int64_t wide_block = 32 / std::min<int64_t>(8, rows - r0);
        for (int64_t c0 = 0; c0 < cols; c0 += wide_block)
          for (int64_t band = r0; band < std::min(r0 + 16, rows); band += 8)
            for (int64_t c = c0; c < std::min(c0 + wide_block, cols); ++c)
              for (int64_t r = band; r < std::min(band + 8, rows); ++r, ++tile) {
                LayerItem it;
                std::memset(&it, 0, sizeof it);
                it.m_off = (int32_t)(r * tm);
                it.n_off = (int32_t)(c * tn);
                it.m_ext = (int32_t)std::min<int64_t>(tm, g.m - r * tm);
                it.n_ext = (int32_t)std::min<int64_t>(tn, g.n - c * tn);
                it.c = g.c + (r * tm * g.ldc + c * tn) * W.c_es;
                it.ldc = g.ldc;
                it.c_es = W.c_es;
                if (g.g) it.g = g.g + (r * tm * g.ldg + c * tn) * 2;
                if (g.u) it.u = g.u + (r * tm * g.ldu + c * tn) * 2;
                it.ldg = g.ldg;
                it.ldu = g.ldu;
                if (g.sa) it.sa = g.sa + r * tm;
                if (g.sb) it.sb = g.sb + c * tn;
                if (g.sb2) it.sb2 = g.sb2 + c * tn;
                if (n_steps > 0) it.front = W.segs[seg];
                it.seg = (int32_t)seg;
                it.n_segs = (int32_t)(g.seg + g.n_segs - seg);
                it.first = (int32_t)first;
                it.steps = (int32_t)n_steps;
                it.tail_seg = (int32_t)tail0;
                it.n_tails = (int32_t)(tail - tail0);
                it.kind = W.kind;
                it.what = k == 0 ? LAYER_ZERO : LAYER_STORE;
                if (runs > 1) {
                  const int64_t slot = first_slot + tile * runs;
                  if (run == 0)
                    joins.push_back({it.c, it.ldc, it.g, it.u, it.ldg, it.ldu, it.sa, it.sb, it.sb2, (const char *)(uintptr_t)((size_t)slot * slot_bytes),
                                     (int32_t)runs, tm, wide, it.m_ext, it.n_ext, it.c_es});
                  it.c = (char *)(uintptr_t)((size_t)(slot + run) * slot_bytes);
                  it.what = LAYER_PARTS;
                  ++slots;
                }
                items.push_back(it);
              }
      }
      first += n_steps;
    }
  }
  if ((int64_t)items.size() > kLayerBlocks || (int64_t)joins.size() * ((tm * tn + 1023) / 1024) > kLayerBlocks) return DMM_ELIMIT;
  if (items.empty()) return DMM_OK;
  // Workgroup w runs on XCD w % 8.  Blocks go to the XCDs in turn, so that all of them are in one region of one group, where what one brings into the
  // last-level cache serves the others (8192 x 12288 x 49152 gated in column blocks, each with a replica of A of its own: 15.7 ms with a run of the
  // list for every XCD); what is left of the list, a run of it for each.
  std::vector<LayerItem> ordered(items.size());
  {
    const size_t even = items.size() / 256 * 256;
    for (size_t x = 0; x < even; ++x) ordered[x / 256 * 256 + x % 32 * 8 + x / 32 % 8] = items[x];
    size_t from = even;
    for (size_t xcd = 0; xcd < 8; ++xcd)
      for (size_t w = even + xcd; w < items.size(); w += 8) ordered[w] = items[from++];
  }
  *scratch = std::max(*scratch, (size_t)slots * slot_bytes);
  L->shape = shape;
  L->n_items = (int)ordered.size();
  L->n_joins = (int)joins.size();
  L->o_items = h->size();
  L->o_segs = L->o_items + ordered.size() * sizeof(LayerItem);
  L->o_joins = L->o_segs + W.segs.size() * sizeof(LayerSeg);
  h->resize(L->o_joins + joins.size() * sizeof(LayerJoin));
  std::memcpy(h->data() + L->o_items, ordered.data(), ordered.size() * sizeof(LayerItem));
  if (!W.segs.empty()) std::memcpy(h->data() + L->o_segs, W.segs.data(), W.segs.size() * sizeof(LayerSeg));
  if (!joins.empty()) std::memcpy(h->data() + L->o_joins, joins.data(), joins.size() * sizeof(LayerJoin));
  static_assert(sizeof(LayerItem) % 8 == 0 && sizeof(LayerSeg) % 8 == 0 && sizeof(LayerJoin) % 8 == 0, "tables lie one behind another");
  return DMM_OK;
}

// Partial sums and copies get their places in the buffer: the former at its front, the latter from `copies` on.
void place_parts(std::vector<char> *h, const LayerLayout &L, char *buf, char *copies, LayerDense dense) {
  auto move = [&](auto *&p, bool copied) {
    if (copied) p = (std::decay_t<decltype(p)>)(copies + (uintptr_t)p);
  };
  const bool left = dense != LAYER_IN_PLACE, right = dense == LAYER_BOTH, out = dense == LAYER_ROWS;
  auto move_segment = [&](LayerSeg &s) {
    move(s.a, left);
    move(s.b, right);
    move(s.b2, right);
  };
  LayerItem *items = (LayerItem *)(h->data() + L.o_items);
  for (int i = 0; i < L.n_items; ++i) {
    LayerItem &it = items[i];
    if (it.what == LAYER_PARTS) it.c = buf + (uintptr_t)it.c;
    else move(it.c, out);
    move(it.g, out && it.ldg);
    move(it.u, out && it.ldu);
    move_segment(it.front);
    move(it.sa, left);
    move(it.sb, right);
    move(it.sb2, right);
  }
  for (LayerSeg *s = (LayerSeg *)(h->data() + L.o_segs); s < (LayerSeg *)(h->data() + L.o_joins); ++s) move_segment(*s);
  LayerJoin *joins = (LayerJoin *)(h->data() + L.o_joins);
  for (int i = 0; i < L.n_joins; ++i) {
    joins[i].parts = buf + (uintptr_t)joins[i].parts;
    move(joins[i].c, out);
    move(joins[i].g, out && joins[i].ldg);
    move(joins[i].u, out && joins[i].ldu);
    move(joins[i].sa, left);
    move(joins[i].sb, right);
    move(joins[i].sb2, right);
  }
}

// The tables of two products, one behind the other in `h`, as those of one launch: that with the longer tiles first.
void merge_pair(std::vector<char> *h, LayerLayout *L, bool second_first) {
  std::vector<char> all;
  const int order[2] = {second_first ? 1 : 0, second_first ? 0 : 1};
  auto put = [&](size_t from, size_t to) { all.insert(all.end(), h->data() + from, h->data() + to); };
  const size_t n_segs = (L[order[0]].o_joins - L[order[0]].o_segs) / sizeof(LayerSeg);
  for (LayerItem *it = (LayerItem *)(h->data() + L[order[1]].o_items), *end = it + L[order[1]].n_items; it < end; ++it) {
    it->seg += (int32_t)n_segs;
    it->tail_seg += (int32_t)n_segs;
  }
  LayerLayout both = L[0];
  both.kind = LAYER_PAIR;
  both.shape = LAYER_128;
  both.n_items = L[0].n_items + L[1].n_items;
  both.n_joins = L[0].n_joins + L[1].n_joins;
  both.o_items = 0;
  for (int x : order) put(L[x].o_items, L[x].o_segs);
  both.o_segs = all.size();
  for (int x : order) put(L[x].o_segs, L[x].o_joins);
  both.o_joins = all.size();
  for (int x : order) put(L[x].o_joins, L[x].o_joins + (size_t)L[x].n_joins * sizeof(LayerJoin));
  h->swap(all);
  L[0] = both;
  L[1] = LayerLayout();
}

// The part of a call that all kinds have in common: the tables of the call before if they are of the same inputs (`key`), else new ones,
// made from what `make` tells of each product (on the operands, or on copies; the first `lefts` products can be on copies of the left operand alone); then `in_front`, the launches and, where `reduce` asks for it, the sum of
// C's replicas.  `part`: the last product has one of two results that are cut alike.  Its runs of K, and whether it is on copies, are those that both
// together are estimated to be best with (`make`'s last argument), so that its bits do not depend on the other's being asked for.
template <class Make, class Front>
int run_layer_on(dmm_plan_t *P, int which, const std::vector<char> &inputs, void *const *c_tiles, const int64_t *c_ld, bool reduce, hipStream_t stream, int products,
              int lefts, bool part, Make make, Front in_front) {
  int rc;
  const bool capturing = is_capturing(stream), known = P->dev && P->dev->layer[which].cached;
  if (!known && (rc = materialize(P))) return rc;
  if (capturing && !known) return DMM_EINVAL;                  // (a graph cannot wait for tables that are on their way)
  if ((rc = ensure_state(P)) || (rc = allow_layer_lds())) return rc;
  int device = 0, cus = 0;
  DMM_HIP(hipGetDevice(&device));
  if ((rc = device_cus(&cus))) return rc;
  LayerState &M = P->dev->layer[which];
  std::vector<char> key(inputs);
  key.insert(key.end(), (const char *)&device, (const char *)&device + sizeof device);
  if (M.cached && key == M.key) {
    if ((rc = M.table.order_behind_copy(stream))) return rc;
    if ((M.layout[0].n_joins || M.layout[1].n_joins || M.n_copies) && (rc = P->dev->uses.order(stream))) return rc;
  } else {
    if (capturing) return DMM_EINVAL;
    M.cached = false;
    LayerLayout layout[2];
    LayerChoice choice[2];
    RedLaunch red;
    std::vector<char> &h = P->dev->host;
    // each product on its operands as they lie, or on copies where that is estimated to be faster and there is room (by itself: what it is asked for with
    // does not change its bits)
    LayerWork work[2];
    LayerDense dense[2] = {LAYER_IN_PLACE, LAYER_IN_PLACE};
    LayerCopies copies;
    // what is laid out: on copies, or of a part
    auto settle = [&](int x) {
      const bool of_part = part && x == products - 1;
      if (dense[x] || of_part) work[x] = make(x, dense[x], &copies, false);
      if (of_part) choice[x] = choose_layer(work[x], cus, choice[x].runs);
    };
    for (int x = 0; x < products; ++x) {
      work[x] = make(x, LAYER_IN_PLACE, nullptr, true);
      choice[x] = choose_layer(work[x], cus);
      double best = choice[x].us;
      for (LayerDense d : {LAYER_BOTH, LAYER_LEFT, LAYER_ROWS}) {
        if (P->C.c != 1 || (d != LAYER_BOTH && x >= lefts)) continue;
        LayerCopies tried;
        const LayerWork then = make(x, d, &tried, true);
        const LayerChoice c = choose_layer(then, cus);
        if (c.us + tried.us() < best && tried.possible())
          best = c.us + tried.us(), dense[x] = d, choice[x] = c;
      }
    }
    for (int x = 0; x < products; ++x) settle(x);
    if ((rc = P->dev->uses.order(stream))) return rc;
    for (;;) {
      h.clear();
      size_t parts[2] = {0, 0};                                // partial sums of each product
      const bool pair = products == 2 && choice[0].tiles > 0 && choice[1].tiles > 0 && pair_us(choice, cus) < choice[0].us + choice[1].us;
      for (int x = 0; x < products; ++x) {
        LayerChoice as = choice[x];                            // (should there be no memory, what was chosen counts again)
        if (pair) as.shape = LAYER_128;
        if ((rc = lay_out(work[x], as, &h, &layout[x], &parts[x]))) return rc;
      }
      const size_t scratch = ((pair ? parts[0] + parts[1] : std::max(parts[0], parts[1])) + 4095) / 4096 * 4096;
      const size_t need = scratch + copies.size;
      if (need > M.cap) {
        if (M.buf) {
          if ((rc = P->dev->uses.wait())) return rc;
          DMM_HIP(hipStreamSynchronize(stream));
          scratch_pool().release(&M.buf, &M.cap);
        }
        rc = scratch_pool().acquire(need, &M.buf, &M.cap);
        if (rc == DMM_ENOMEM && copies.size) {
          (void)hipGetLastError();
          copies = LayerCopies();
          for (int x = 0; x < products; ++x) {
            if (!dense[x]) continue;
            dense[x] = LAYER_IN_PLACE;
            work[x] = make(x, LAYER_IN_PLACE, nullptr, true);
            choice[x] = choose_layer(work[x], cus);
            settle(x);
          }
          continue;
        }
        if (rc) return rc;
      }
      char *const at = copies.size ? M.buf + scratch : nullptr;
      for (int x = 0; x < products; ++x) place_parts(&h, layout[x], M.buf + (pair && x == 1 ? parts[0] : 0), at, dense[x]);
      if (pair && layout[0].n_items && layout[1].n_items) merge_pair(&h, layout, choice[1].steps / (double)choice[1].runs > choice[0].steps / (double)choice[0].runs);
      for (LayerCopy &j : copies.jobs) j.dst = at + (uintptr_t)j.dst;
      for (LayerCopy &j : copies.back) j.src = at + (uintptr_t)j.src;
      break;
    }
    M.n_copies = (int)copies.jobs.size();
    M.copy_blocks = (int)copies.blocks;
    M.n_back = (int)copies.back.size();
    M.back_blocks = (int)copies.back_blocks;
    M.o_copies = h.size();
    M.o_back = M.o_copies + copies.jobs.size() * sizeof(LayerCopy);
    for (const std::vector<LayerCopy> *v : {&copies.jobs, &copies.back}) h.insert(h.end(), (const char *)v->data(), (const char *)(v->data() + v->size()));
    static_assert(sizeof(LayerCopy) % 8 == 0, "tables lie one behind another");
    if (c_tiles && (rc = build_reduce(P, c_tiles, c_ld, 0, &h, h.size(), &red))) return rc;
    if ((rc = M.table.upload(h.data(), h.size(), stream, P->dev->uses))) return rc;
    red.dev_base = M.table.dev();
    M.layout[0] = layout[0];
    M.layout[1] = layout[1];
    M.red = red;
    M.key.swap(key);
    M.cached = true;
  }
  if ((rc = in_front())) return rc;
  const bool sum = reduce && M.red.n_items;
  if (!M.layout[0].n_items && !M.layout[1].n_items && !sum) return DMM_OK;
  hipEvent_t behind = nullptr;
  if ((rc = P->dev->uses.claim(stream, &behind))) return rc;
  const char *d = M.table.dev();
  bool marked = false;
  if (M.n_copies) {
    layer_copy_launch((const LayerCopy *)(d + M.o_copies), M.n_copies, M.copy_blocks, stream);
    DMM_HIP(hipGetLastError());
  }
  for (int x = 0; x < 2; ++x) {
    const LayerLayout &L = M.layout[x];
    if (!L.n_items) continue;
    const bool last = !sum && !M.n_back && (x == 1 || !M.layout[1].n_items);
    marked = layer_launch(last ? behind : nullptr, L.kind, L.shape, L.act, cus, (const LayerItem *)(d + L.o_items), L.n_items, (const LayerSeg *)(d + L.o_segs),
                          (const LayerJoin *)(d + L.o_joins), L.n_joins, stream);
    DMM_HIP(hipGetLastError());
  }
  if (M.n_back) {
    layer_copy_launch((const LayerCopy *)(d + M.o_back), M.n_back, M.back_blocks, stream);
    DMM_HIP(hipGetLastError());
  }
  if (sum && (rc = fire_reduce(P, M.red, stream, false, behind, &marked))) return rc;
  return marked ? DMM_OK : P->dev->uses.mark(stream);
}

template <class Make, class Front>
int run_layer(dmm_plan_t *P, int which, const std::vector<char> &inputs, void *const *c_tiles, const int64_t *c_ld, bool reduce, hipStream_t stream, int products,
              int lefts, bool part, Make make, Front in_front) {
  const int rc = run_layer_on(P, which, inputs, c_tiles, c_ld, reduce, stream, products, lefts, part, make, in_front);
  if (rc == DMM_ENOMEM) (void)hipGetLastError();               // (it would be the next call's)
  return rc;
}

struct LayerKey {
  std::vector<char> bytes;
  void put(const void *p, size_t n) { bytes.insert(bytes.end(), (const char *)p, (const char *)p + n); }
  void put(const dmm_tiles *t, int64_t n) {
    const char there = t != nullptr;
    put(&there, 1);
    if (!t) return;
    put(t->tiles, (size_t)n * sizeof(void *));
    put(t->ld, (size_t)n * sizeof(int64_t));
  }
  void put(const dmm_int_tiles *t, const Grid &G, bool by_cols) {
    const size_t n = (size_t)(G.c * G.tiles_per_rep());
    put(t->codes, n * sizeof(void *));
    put(t->code_ld, n * sizeof(int64_t));
    put(t->scales, (size_t)G.c * (size_t)(by_cols ? G.gc : G.gr) * sizeof(void *));
  }
};

// Corner of a region inside a tile.
char *corner(const Grid &G, const dmm_tiles *t, int64_t i, int32_t ti, int32_t tj, int64_t row, int64_t col, int es) {
  return (char *)t->tiles[i] + ((row - G.rc[(size_t)ti]) * t->ld[i] + col - G.cc[(size_t)tj]) * es;
}

// Groups of a plan's own product: the op list by output sub-tile, and zeros where no op writes.
template <class Segment, class Out>
void plan_groups(const dmm_plan_t *P, LayerWork *W, Segment segment, Out out) {
  for (const Group &g : P->groups) {
    LayerGroup r;
    std::memset(&r, 0, sizeof r);
    r.m = g.m1 - g.m0;
    r.n = g.n1 - g.n0;
    r.seg = W->segs.size();
    for (int64_t x = g.first; x < g.first + g.count; ++x) segment(g, P->tasks[(size_t)P->order[(size_t)x]]);
    r.n_segs = W->segs.size() - r.seg;
    out(g.c_rep, g.c_ti, g.c_tj, g.m0, g.n0, g.count ? &P->tasks[(size_t)P->order[(size_t)g.first]] : nullptr, &r);
    W->groups.push_back(r);
  }
  for (const dmm_work_item &w : P->items) {
    if (w.group >= 0) continue;
    LayerGroup r;
    std::memset(&r, 0, sizeof r);
    r.m = w.m_ext;
    r.n = w.n_ext;
    r.seg = W->segs.size();
    out(w.c_rep, w.c_ti, w.c_tj, w.m0, w.n0, nullptr, &r);
    W->groups.push_back(r);
  }
}

// The same on copies (C has one replica): C's tiles, all of K in one segment.
template <class Segment, class Out>
void tile_groups(const Grid &G, LayerWork *W, Segment segment, Out out) {
  for (int32_t ti = 0; ti < G.gr; ++ti)
    for (int32_t tj = 0; tj < G.gc; ++tj) {
      LayerGroup r;
      std::memset(&r, 0, sizeof r);
      r.m = G.rc[(size_t)ti + 1] - G.rc[(size_t)ti];
      r.n = G.cc[(size_t)tj + 1] - G.cc[(size_t)tj];
      if (r.m <= 0 || r.n <= 0) continue;
      r.seg = W->segs.size();
      segment(G.rc[(size_t)ti], G.cc[(size_t)tj]);
      r.n_segs = W->segs.size() - r.seg;
      out(0, ti, tj, G.rc[(size_t)ti], G.cc[(size_t)tj], &r);
      W->groups.push_back(r);
    }
}
int32_t interval_of(const std::vector<int64_t> &cuts, int64_t at) {   // the non-empty interval that holds `at`
  return (int32_t)(std::upper_bound(cuts.begin(), cuts.end(), at) - cuts.begin()) - 1;
}

// On a copy of the left operand alone, whose row cuts then play no part (few rows, cut into blocks that would each bring in all of the right operand): C's
// tiles, cut where B's columns are; a segment for every tile of B down them.  `whole`: C's cuts play no part either, its tiles are filled from scratch memory
// afterwards.  (8 x 8192 x 28672 in 8 bits, A in 8 row blocks, B in 8 column blocks, C in 4 x 2: 255 us in place, 134 with LAYER_LEFT, 46 with LAYER_ROWS.)
template <class Segment, class Out>
void left_groups(const dmm_plan_t *P, bool whole, LayerWork *W, Segment segment, Out out) {
  const Grid &B = P->B, &C = P->C;
  const std::vector<int64_t> nc = whole ? merged_cuts({&B.cc}) : merged_cuts({&B.cc, &C.cc}), mc = whole ? std::vector<int64_t>{0, C.rows} : merged_cuts({&C.rc});
  for (size_t y = 0; y + 1 < mc.size(); ++y)
    for (size_t x = 0; x + 1 < nc.size(); ++x) {
      const int32_t bj = interval_of(B.cc, nc[x]);
      LayerGroup r;
      std::memset(&r, 0, sizeof r);
      r.m = mc[y + 1] - mc[y];
      r.n = nc[x + 1] - nc[x];
      if (r.m <= 0 || r.n <= 0) continue;
      r.seg = W->segs.size();
      for (int32_t bi = 0; bi < B.gr; ++bi)
        if (B.rc[(size_t)bi + 1] > B.rc[(size_t)bi]) segment(bi, bj, mc[y], nc[x], r.n);
      r.n_segs = W->segs.size() - r.seg;
      out(bj, mc[y], nc[x], &r);
      W->groups.push_back(r);
    }
}
// A segment on copies: places of the operands' first element, whole steps of K.
LayerSeg dense_segment(size_t a, int64_t a_pitch, size_t b, int64_t b_pitch, size_t b2, int64_t b2_pitch, int64_t steps) {
  LayerSeg s;
  s.a = (const char *)(uintptr_t)a;
  s.b = (const char *)(uintptr_t)b;
  s.b2 = (const char *)(uintptr_t)b2;
  s.a_pitch = (uint32_t)a_pitch;
  s.b_pitch = (uint32_t)b_pitch;
  s.b2_pitch = (uint32_t)b2_pitch;
  s.steps = (int32_t)steps;
  s.tail = 0;
  s.pad = 0;
  return s;
}

// dA = dC B^T (summed over the pairs): A's tiles, cut where C's rows and B's rows are; both operands lie along n.
void input_gradient(const dmm_plan_t *P, const dmm_tiles *const *dc, const dmm_tiles *const *b, int pairs, const dmm_tiles *da, LayerWork *W) {
  const Grid &A = P->A, &B = P->B, &C = P->C;
  const std::vector<int64_t> mc = merged_cuts({&A.rc, &C.rc}), kc = merged_cuts({&A.cc, &B.rc}), nc = merged_cuts({&B.cc, &C.cc});
  for (size_t i = 0; i + 1 < mc.size(); ++i)
    for (size_t j = 0; j + 1 < kc.size(); ++j) {
      const int32_t ai = interval_of(A.rc, mc[i]), ci = interval_of(C.rc, mc[i]), aj = interval_of(A.cc, kc[j]), bi = interval_of(B.rc, kc[j]);
      LayerGroup r;
      std::memset(&r, 0, sizeof r);
      r.m = mc[i + 1] - mc[i];
      r.n = kc[j + 1] - kc[j];
      r.seg = W->segs.size();
      for (int p = 0; p < pairs; ++p)
        for (size_t x = 0; x + 1 < nc.size(); ++x) {
          const int32_t bj = interval_of(B.cc, nc[x]), cj = interval_of(C.cc, nc[x]);
          const int64_t ct = C.table_index(0, ci, cj), bt = B.table_index(0, bi, bj);
          LayerSeg s;
          s.a = corner(C, dc[p], ct, ci, cj, mc[i], nc[x], 2);
          s.b = corner(B, b[p], bt, bi, bj, kc[j], nc[x], 2);
          s.b2 = nullptr;
          s.a_pitch = (uint32_t)(dc[p]->ld[ct] * 2);
          s.b_pitch = (uint32_t)(b[p]->ld[bt] * 2);
          s.b2_pitch = 0;
          put_segment(W, s, nc[x + 1] - nc[x], 0);
        }
      r.n_segs = W->segs.size() - r.seg;
      const int64_t at = A.table_index(0, ai, aj);
      r.c = corner(A, da, at, ai, aj, mc[i], kc[j], W->c_es);
      r.ldc = da->ld[at];
      W->groups.push_back(r);
    }
}

// dB = A^T dC: B's tiles, cut where A's columns and C's columns are; both operands lie across m.
void weight_gradient(const dmm_plan_t *P, const dmm_tiles *a, const dmm_tiles *dc, const dmm_tiles *db, LayerWork *W) {
  const Grid &A = P->A, &B = P->B, &C = P->C;
  const std::vector<int64_t> mc = merged_cuts({&A.rc, &C.rc}), kc = merged_cuts({&A.cc, &B.rc}), nc = merged_cuts({&B.cc, &C.cc});
  for (size_t i = 0; i + 1 < kc.size(); ++i)
    for (size_t j = 0; j + 1 < nc.size(); ++j) {
      const int32_t aj = interval_of(A.cc, kc[i]), bi = interval_of(B.rc, kc[i]), bj = interval_of(B.cc, nc[j]), cj = interval_of(C.cc, nc[j]);
      LayerGroup r;
      std::memset(&r, 0, sizeof r);
      r.m = kc[i + 1] - kc[i];
      r.n = nc[j + 1] - nc[j];
      r.seg = W->segs.size();
      for (size_t x = 0; x + 1 < mc.size(); ++x) {
        const int32_t ai = interval_of(A.rc, mc[x]), ci = interval_of(C.rc, mc[x]);
        const int64_t at = A.table_index(0, ai, aj), ct = C.table_index(0, ci, cj);
        LayerSeg s;
        s.a = corner(A, a, at, ai, aj, mc[x], kc[i], 2);
        s.b = corner(C, dc, ct, ci, cj, mc[x], nc[j], 2);
        s.b2 = nullptr;
        s.a_pitch = (uint32_t)(a->ld[at] * 2);
        s.b_pitch = (uint32_t)(dc->ld[ct] * 2);
        s.b2_pitch = 0;
        const int64_t ga = rows_past_end(A.rc[ai + 1] - A.rc[ai], A.cc[aj + 1] - A.cc[aj], a->ld[at], mc[x + 1] - A.rc[ai], kc[i] - A.cc[aj], r.m);
        const int64_t gc = rows_past_end(C.rc[ci + 1] - C.rc[ci], C.cc[cj + 1] - C.cc[cj], dc->ld[ct], mc[x + 1] - C.rc[ci], nc[j] - C.cc[cj], r.n);
        put_segment(W, s, mc[x + 1] - mc[x], std::max(ga, gc));
      }
      r.n_segs = W->segs.size() - r.seg;
      const int64_t bt = B.table_index(0, bi, bj);
      r.c = corner(B, db, bt, bi, bj, kc[i], nc[j], W->c_es);
      r.ldc = db->ld[bt];
      W->groups.push_back(r);
    }
}

// The products behind both backward calls, from the operands or from copies of these: dA (`input`) or all dB, of `pairs` of dC and B.
LayerWork gradients(const dmm_plan_t *P, bool input, const dmm_tiles *a, const dmm_tiles *const *b, const dmm_tiles *const *dc, int pairs, const dmm_tiles *da,
                    const dmm_tiles *const *db, int es, LayerDense dense, LayerCopies *copies) {
  const Grid &A = P->A, &B = P->B, &C = P->C;
  LayerWork W;
  W.kind = input ? LAYER_NT : LAYER_TN;
  W.rows = input ? A.rows : A.cols;
  W.c_es = input ? 2 : es;
  if (dense == LAYER_IN_PLACE) {
    if (input) input_gradient(P, dc, b, pairs, da, &W);
    for (int p = 0; p < pairs && !input; ++p)
      if (db[p]) weight_gradient(P, a, dc[p], db[p], &W);
    return W;
  }
  // dC serves along n and across m; its columns are those of dB's tiles
  const LayerCopies::Axis cols(B.cc, 64), rows(B.rc, 64);
  const int64_t m = up_to(C.rows, 64), n = cols.total;
  LayerCopies::Matrix cc[2], cb[2];
  for (int p = 0; p < pairs; ++p)
    if (input || db[p]) cc[p] = copies->matrix(C, dc[p]->tiles, dc[p]->ld, 2, false, m, cols, true);
  if (dense != LAYER_BOTH) {
    const bool whole = dense == LAYER_ROWS;
    const LayerCopies::Matrix out = whole ? copies->results(A, da, 2) : LayerCopies::Matrix{0, 0};
    const std::vector<int64_t> mc = whole ? std::vector<int64_t>{0, A.rows} : merged_cuts({&A.rc}), kc = whole ? merged_cuts({&B.rc}) : merged_cuts({&A.cc, &B.rc});
    for (size_t y = 0; y + 1 < mc.size(); ++y)
      for (size_t x = 0; x + 1 < kc.size(); ++x) {
        const int32_t bi = interval_of(B.rc, kc[x]);
        LayerGroup r;
        std::memset(&r, 0, sizeof r);
        r.m = mc[y + 1] - mc[y];
        r.n = kc[x + 1] - kc[x];
        if (r.m <= 0 || r.n <= 0) continue;
        r.seg = W.segs.size();
        for (int p = 0; p < pairs; ++p)
          for (int32_t bj = 0; bj < B.gc; ++bj) {
            if (B.cc[(size_t)bj + 1] == B.cc[(size_t)bj]) continue;
            const int64_t i = B.table_index(0, bi, bj);
            LayerSeg s = dense_segment(cc[p].at + (size_t)(mc[y] * cc[p].pitch + cols.place(B.cc[(size_t)bj]) * 2), cc[p].pitch, 0, b[p]->ld[i] * 2, 0, 0, 0);
            s.b = corner(B, b[p], i, bi, bj, kc[x], B.cc[(size_t)bj], 2);
            put_segment(&W, s, B.cc[(size_t)bj + 1] - B.cc[(size_t)bj], 0);
          }
        r.n_segs = W.segs.size() - r.seg;
        if (whole) {
          r.c = (char *)(uintptr_t)(out.at + (size_t)kc[x] * 2);
          r.ldc = out.pitch / 2;
        } else {
          const int32_t ti = interval_of(A.rc, mc[y]), tj = interval_of(A.cc, kc[x]);
          const int64_t i = A.table_index(0, ti, tj);
          r.c = corner(A, da, i, ti, tj, mc[y], kc[x], 2);
          r.ldc = da->ld[i];
        }
        W.groups.push_back(r);
      }
    return W;
  }
  if (input) {
    for (int p = 0; p < pairs; ++p) cb[p] = copies->matrix(B, b[p]->tiles, b[p]->ld, 2, false, B.rows, cols, true);
    tile_groups(
        A, &W,
        [&](int64_t m0, int64_t k0) {
          for (int p = 0; p < pairs; ++p)
            W.segs.push_back(dense_segment(cc[p].at + (size_t)(m0 * cc[p].pitch), cc[p].pitch, cb[p].at + (size_t)(k0 * cb[p].pitch), cb[p].pitch, 0, 0, n / 64));
        },
        [&](int32_t, int32_t ti, int32_t tj, int64_t m0, int64_t k0, LayerGroup *r) {
          const int64_t i = A.table_index(0, ti, tj);
          r->c = corner(A, da, i, ti, tj, m0, k0, 2);
          r->ldc = da->ld[i];
        });
    return W;
  }
  const LayerCopies::Matrix ca = copies->matrix(A, a->tiles, a->ld, 2, false, m, rows, false);
  for (int p = 0; p < pairs; ++p) {
    if (!db[p]) continue;
    tile_groups(
        B, &W,
        [&](int64_t k0, int64_t n0) {
          W.segs.push_back(dense_segment(ca.at + (size_t)rows.place(k0) * 2, ca.pitch, cc[p].at + (size_t)cols.place(n0) * 2, cc[p].pitch, 0, 0, m / 64));
        },
        [&](int32_t, int32_t ti, int32_t tj, int64_t k0, int64_t n0, LayerGroup *r) {
          const int64_t i = B.table_index(0, ti, tj);
          r->c = corner(B, db[p], i, ti, tj, k0, n0, es);
          r->ldc = db[p]->ld[i];
        });
  }
  return W;
}

bool is_activation(int act) { return act == DMM_SILU || act == DMM_GELU || act == DMM_GELU_TANH; }

// C = A B, or the gated product of A with two right operands, in 8-bit integers.
int i8_product(dmm_plan_t *P, int which, int act, const dmm_int_tiles *a, const dmm_int_tiles *b, const dmm_int_tiles *b2, const dmm_tiles *c, int c_es,
               bool reduce, hipStream_t stream) {
  const Grid &A = P->A, &B = P->B, &C = P->C;
  int rc;
  if ((rc = check_i8(A, a, false)) || (rc = check_i8(B, b, true)) || (b2 && (rc = check_i8(B, b2, true))) || (rc = check_layer_tiles(C, c, c_es)) ||
      (rc = check_sizes(P)))
    return rc;
  LayerKey key;
  const int head[2] = {act, c_es};
  key.put(head, sizeof head);
  key.put(a, A, false);
  key.put(b, B, true);
  if (b2) key.put(b2, B, true);
  key.put(c, C.c * C.tiles_per_rep());
  auto make = [&](int, LayerDense dense, LayerCopies *copies, bool) {
    LayerWork W;
    W.kind = b2 ? LAYER_I8_GATED : LAYER_I8;
    W.act = act;
    W.c_es = c_es;
    W.rows = C.rows;
    auto result = [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, LayerGroup *r) {
      const int64_t i = C.table_index(rep, ti, tj);
      r->c = corner(C, c, i, ti, tj, m0, n0, c_es);
      r->ldc = c->ld[i];
    };
    if (dense == LAYER_LEFT || dense == LAYER_ROWS) {
      const LayerCopies::Axis along(B.rc, layer_step(W.kind));
      const LayerCopies::Matrix ca = copies->matrix(A, a->codes, a->code_ld, 1, false, A.rows, along, false);
      const size_t sa = copies->scales(A.rc, a->scales);
      const LayerCopies::Matrix cc = dense == LAYER_ROWS ? copies->results(C, c, c_es) : LayerCopies::Matrix{0, 0};
      left_groups(
          P, dense == LAYER_ROWS, &W,
          [&](int32_t bi, int32_t bj, int64_t m0, int64_t n0, int64_t) {
            const int64_t i = B.table_index(0, bi, bj), bc = n0 - B.cc[(size_t)bj];
            LayerSeg s;
            s.a = (const char *)(uintptr_t)(ca.at + (size_t)(m0 * ca.pitch + along.place(B.rc[(size_t)bi])));
            s.b = (const char *)b->codes[i] + bc * b->code_ld[i];
            s.b2 = b2 ? (const char *)b2->codes[i] + bc * b2->code_ld[i] : nullptr;
            s.a_pitch = (uint32_t)ca.pitch;
            s.b_pitch = (uint32_t)b->code_ld[i];
            s.b2_pitch = b2 ? (uint32_t)b2->code_ld[i] : 0;
            put_segment(&W, s, B.rc[(size_t)bi + 1] - B.rc[(size_t)bi], 0);
          },
          [&](int32_t bj, int64_t m0, int64_t n0, LayerGroup *r) {
            if (dense == LAYER_ROWS) r->c = (char *)(uintptr_t)(cc.at + (size_t)(n0 * c_es)), r->ldc = cc.pitch / c_es;
            else result(0, interval_of(C.rc, m0), interval_of(C.cc, n0), m0, n0, r);
            r->sa = (const float *)(uintptr_t)(sa + (size_t)m0 * 4);
            r->sb = b->scales[bj] + (n0 - B.cc[(size_t)bj]);
            r->sb2 = b2 ? b2->scales[bj] + (n0 - B.cc[(size_t)bj]) : nullptr;
          });
      return W;
    }
    if (dense == LAYER_BOTH) {
      const LayerCopies::Axis along({0, A.cols}, layer_step(W.kind));
      const int64_t k = along.total;
      const LayerCopies::Matrix ca = copies->matrix(A, a->codes, a->code_ld, 1, false, A.rows, along, true),
                                cb = copies->matrix(B, b->codes, b->code_ld, 1, true, B.cols, along, true);
      LayerCopies::Matrix cb2 = {0, 0};
      if (b2) cb2 = copies->matrix(B, b2->codes, b2->code_ld, 1, true, B.cols, along, true);
      const size_t sa = copies->scales(A.rc, a->scales), sb = copies->scales(B.cc, b->scales), sb2 = b2 ? copies->scales(B.cc, b2->scales) : 0;
      tile_groups(
          C, &W,
          [&](int64_t m0, int64_t n0) {
            W.segs.push_back(dense_segment(ca.at + (size_t)(m0 * ca.pitch), ca.pitch, cb.at + (size_t)(n0 * cb.pitch), cb.pitch, cb2.at + (size_t)(n0 * cb2.pitch),
                                           cb2.pitch, k / layer_step(W.kind)));
          },
          [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, LayerGroup *r) {
            result(rep, ti, tj, m0, n0, r);
            r->sa = (const float *)(uintptr_t)(sa + (size_t)m0 * 4);
            r->sb = (const float *)(uintptr_t)(sb + (size_t)n0 * 4);
            r->sb2 = (const float *)(uintptr_t)(sb2 + (size_t)n0 * 4);
          });
      return W;
    }
    plan_groups(
        P, &W,
        [&](const Group &g, const dmm_task &t) {
          const int64_t ai = A.table_index(t.a_rep, t.a_ti, t.a_tj), bi = B.table_index(t.b_rep, t.b_ti, t.b_tj);
          const int64_t ak = t.k0 - A.cc[(size_t)t.a_tj], bk = t.k0 - B.rc[(size_t)t.b_ti];
          const int64_t ar = g.m0 - A.rc[(size_t)t.a_ti], bc = g.n0 - B.cc[(size_t)t.b_tj];
          LayerSeg s;
          s.a = (const char *)a->codes[ai] + ar * a->code_ld[ai] + ak;
          s.b = (const char *)b->codes[bi] + bc * b->code_ld[bi] + bk;
          s.b2 = b2 ? (const char *)b2->codes[bi] + bc * b2->code_ld[bi] + bk : nullptr;
          s.a_pitch = (uint32_t)a->code_ld[ai];
          s.b_pitch = (uint32_t)b->code_ld[bi];
          s.b2_pitch = b2 ? (uint32_t)b2->code_ld[bi] : 0;
          put_segment(&W, s, t.k1 - t.k0, 0);
        },
        [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, const dmm_task *t, LayerGroup *r) {
          result(rep, ti, tj, m0, n0, r);
          if (!t) return;
          r->sa = a->scales[(int64_t)t->a_rep * A.gr + t->a_ti] + (m0 - A.rc[(size_t)t->a_ti]);
          const int64_t s = (int64_t)t->b_rep * B.gc + t->b_tj, at = n0 - B.cc[(size_t)t->b_tj];
          r->sb = b->scales[s] + at;
          r->sb2 = b2 ? b2->scales[s] + at : nullptr;
        });
    return W;
  };
  return run_layer(P, which, key.bytes, c->tiles, c->ld, reduce, stream, 1, 1, false, make, [] { return DMM_OK; });
}

// dU = dH act(G), dG = dH U act'(G), tile by tile.
int64_t slope_blocks(int64_t h, int64_t w) { return (h * ((w + 7) / 8) + SLOPE_CHUNKS - 1) / SLOPE_CHUNKS; }
int slope(const Grid &C, int act, const dmm_tiles *g, const dmm_tiles *u, const dmm_tiles *dh, const dmm_tiles *dg, const dmm_tiles *du, hipStream_t stream) {
  SlopeArgs args;
  std::memset(&args, 0, sizeof args);
  args.act = act;
  int64_t blocks = 0;
  auto flush = [&]() -> int {
    if (!args.n) return DMM_OK;
    slope_launch(args, (int)blocks, stream);
    args.n = 0;
    blocks = 0;
    DMM_HIP(hipGetLastError());
    return DMM_OK;
  };
  int rc;
  for (int32_t ti = 0; ti < C.gr; ++ti)
    for (int32_t tj = 0; tj < C.gc; ++tj) {
      const int64_t h = C.rc[(size_t)ti + 1] - C.rc[(size_t)ti], w = C.cc[(size_t)tj + 1] - C.cc[(size_t)tj];
      if (h <= 0 || w <= 0) continue;
      const int64_t i = C.table_index(0, ti, tj);
      SlopeTile t;
      std::memset(&t, 0, sizeof t);
      t.g = (const char *)g->tiles[i];
      t.u = (const char *)u->tiles[i];
      t.dh = (const char *)dh->tiles[i];
      t.dg = (char *)dg->tiles[i];
      t.du = (char *)du->tiles[i];
      t.pg = g->ld[i] * 2;
      t.pu = u->ld[i] * 2;
      t.ph = dh->ld[i] * 2;
      t.pdg = dg->ld[i] * 2;
      t.pdu = du->ld[i] * 2;
      t.h = (int32_t)h;
      t.w = (int32_t)w;
      const int64_t n = slope_blocks(h, w);
      if ((args.n == SLOPE_TILES || blocks + n > kLayerBlocks) && (rc = flush())) return rc;
      t.first_block = (int32_t)blocks;
      blocks += n;
      args.tile[args.n++] = t;
    }
  return flush();
}
// (before anything is launched: a call that is refused writes nothing)
int check_slope(const Grid &C) {
  for (int32_t ti = 0; ti < C.gr; ++ti)
    for (int32_t tj = 0; tj < C.gc; ++tj) {
      const int64_t h = C.rc[(size_t)ti + 1] - C.rc[(size_t)ti], w = C.cc[(size_t)tj + 1] - C.cc[(size_t)tj];
      if (slope_blocks(h, w) > kLayerBlocks) return DMM_ELIMIT;
    }
  return DMM_OK;
}

// ---- integers and values --------------------------------------------------------------------------------

// Runs `launch` over all tiles in blocks of `rows` by `cols`, as many tiles at a time as a launch's argument holds.
template <class F>
int over_i8_tiles(const Grid &G, int es, char *const *x, const int64_t *x_ld, const dmm_int_tiles *q, bool by_cols, int64_t rows, int64_t cols, F launch) {
  I8Args args;
  std::memset(&args, 0, sizeof args);
  int64_t blocks = 0;
  auto flush = [&]() -> int {
    if (!args.n) return DMM_OK;
    launch(args, (int)blocks);
    args.n = 0;
    blocks = 0;
    DMM_HIP(hipGetLastError());
    return DMM_OK;
  };
  int rc;
  for (int32_t rep = 0; rep < G.c; ++rep)
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t h = G.rc[(size_t)ti + 1] - G.rc[(size_t)ti], w = G.cc[(size_t)tj + 1] - G.cc[(size_t)tj];
        if (h <= 0 || w <= 0) continue;
        const int64_t i = G.table_index(rep, ti, tj);
        I8Tile t;
        std::memset(&t, 0, sizeof t);
        t.x = x[i];
        t.x_pitch = x_ld[i] * es;
        t.q = (char *)q->codes[i];
        t.q_pitch = q->code_ld[i];
        t.scale = q->scales[by_cols ? (int64_t)rep * G.gc + tj : (int64_t)rep * G.gr + ti];
        t.h = (int32_t)h;
        t.w = (int32_t)w;
        t.blocks_across = (int32_t)((w + cols - 1) / cols);
        const int64_t n = (h + rows - 1) / rows * t.blocks_across;
        if ((args.n == I8_TILES || blocks + n > kLayerBlocks) && (rc = flush())) return rc;
        t.first_block = (int32_t)blocks;
        blocks += n;
        args.tile[args.n++] = t;
      }
  return flush();
}
int check_i8_blocks(const Grid &G, int es) {
  for (int32_t ti = 0; ti < G.gr; ++ti)
    for (int32_t tj = 0; tj < G.gc; ++tj) {
      const int64_t h = G.rc[(size_t)ti + 1] - G.rc[(size_t)ti], w = G.cc[(size_t)tj + 1] - G.cc[(size_t)tj];
      if (h > kLayerRows || w > kLayerRows || (h + 127) / 128 * ((w + i8_block_cols(es == 4) - 1) / i8_block_cols(es == 4)) > kLayerBlocks) return DMM_ELIMIT;
    }
  return DMM_OK;
}

int over_scales(const Grid &G, const dmm_int_tiles *q, bool by_cols, int what, hipStream_t stream) {
  I8ScaleArgs args;
  std::memset(&args, 0, sizeof args);
  int64_t blocks = 0;
  const std::vector<int64_t> &cuts = by_cols ? G.cc : G.rc;
  const int32_t n = by_cols ? G.gc : G.gr;
  auto flush = [&]() -> int {
    if (!args.n) return DMM_OK;
    i8_scales_launch(args, (int)blocks, what, stream);
    args.n = 0;
    blocks = 0;
    DMM_HIP(hipGetLastError());
    return DMM_OK;
  };
  int rc;
  for (int32_t rep = 0; rep < G.c; ++rep)
    for (int32_t t = 0; t < n; ++t) {
      const int64_t len = cuts[(size_t)t + 1] - cuts[(size_t)t], need = (len + 255) / 256;
      if (len <= 0) continue;
      if ((args.n == I8_PIECES || blocks + need > kLayerBlocks) && (rc = flush())) return rc;
      args.piece[args.n++] = {q->scales[(int64_t)rep * n + t], (int32_t)len, (int32_t)blocks};
      blocks += need;
    }
  return flush();
}

// One form.  Along the rows, a workgroup takes a whole row where it meets few tiles and rows are many or short; along the columns, a block where
// there are no more rows than it has; otherwise the largest magnitudes are collected block by block first.
int i8_form(const Grid &G, int dtype, char *const *x, const int64_t *x_ld, const dmm_int_tiles *q, bool by_cols, hipStream_t stream) {
  const int es = dtype == DMM_F32 ? 4 : 2;
  const bool f32 = es == 4;
  int rc;
  if (!by_cols && G.gc <= I8_ROW_CUTS && G.cols <= kLayerRows) {
    I8RowArgs args;
    std::memset(&args, 0, sizeof args);
    for (int32_t tj = 0; tj < G.gc; ++tj) {
      const int64_t w = G.cc[(size_t)tj + 1] - G.cc[(size_t)tj];
      args.n += w > 0;
      args.vectors += (int32_t)((w + 7) / 8);
    }
    int64_t blocks = 0;
    auto flush = [&]() -> int {
      if (!blocks) return DMM_OK;
      // (few rows: a vector a thread; many: I8_ROW_KEPT, and more rows on a CU at a time)
      const int per = blocks < kLayerManyRows ? 1 : I8_ROW_KEPT;
      i8_whole_rows_launch(args, (int)blocks, (int)std::min<int64_t>(I8_ROW_THREADS, up_to(std::max(args.vectors / per, 1), 64)), f32, stream);
      args.groups = 0;
      blocks = 0;
      DMM_HIP(hipGetLastError());
      return DMM_OK;
    };
    const int64_t most = ((int64_t)1 << 32) / I8_ROW_THREADS - 1;   // (a launch has less than 2^32 threads)
    for (int32_t rep = 0; rep < G.c; ++rep)
      for (int32_t ti = 0; ti < G.gr; ++ti) {
        const int64_t all = G.rc[(size_t)ti + 1] - G.rc[(size_t)ti];
        for (int64_t at = 0; at < all;) {
          if ((args.groups == I8_ROW_GROUPS || (args.groups + 1) * args.n > I8_ROW_PIECES || blocks == most) && (rc = flush())) return rc;
          const int64_t h = std::min(all - at, most - blocks);
          I8RowPiece *piece = args.piece + args.groups * args.n;
          args.group[args.groups] = {q->scales[(int64_t)rep * G.gr + ti] + at, (int32_t)blocks, args.groups * args.n};
          int32_t first = 0;
          for (int32_t tj = 0; tj < G.gc; ++tj) {
            const int64_t w = G.cc[(size_t)tj + 1] - G.cc[(size_t)tj], i = G.table_index(rep, ti, tj);
            if (w <= 0) continue;
            *piece++ = {x[i] + at * x_ld[i] * es, (char *)q->codes[i] + at * q->code_ld[i], x_ld[i] * es, q->code_ld[i], (int32_t)w, first};
            first += (int32_t)((w + 7) / 8);
          }
          ++args.groups;
          blocks += h;
          at += h;
        }
      }
    return flush();
  }
  if (by_cols && merged_cuts({&G.rc}).size() == 2 && G.rows <= 128)
    return over_i8_tiles(G, es, x, x_ld, q, true, 128, i8_block_cols(f32), [&](const I8Args &args, int blocks) { i8_whole_cols_launch(args, blocks, f32, stream); });
  if ((rc = over_scales(G, q, by_cols, I8_CLEAR, stream))) return rc;
  if ((rc = over_i8_tiles(G, es, x, x_ld, q, by_cols, 128, i8_block_cols(f32),
                          [&](const I8Args &args, int blocks) { i8_amax_launch(args, blocks, f32, by_cols, stream); })))
    return rc;
  if ((rc = over_i8_tiles(G, es, x, x_ld, q, by_cols, 128, i8_block_cols(f32),
                          [&](const I8Args &args, int blocks) { i8_quantize_launch(args, blocks, f32, by_cols, stream); })))
    return rc;
  return over_scales(G, q, by_cols, I8_FINISH, stream);
}

}  // namespace
}  // namespace dmm

extern "C" {

int dmm_int_quantize(const dmm_matrix_desc *X, int dtype, const dmm_tiles *x, const dmm_int_tiles *rows, const dmm_int_tiles *cols, void *hip_stream) {
  using namespace dmm;
  if (!X || !x || !x->tiles || !x->ld || (!rows && !cols) || (dtype != DMM_BF16 && dtype != DMM_F32)) return DMM_EINVAL;
  TraceRange whole("dmm_int_quantize");
  try {
    Grid G;
    int rc;
    const int es = dtype == DMM_F32 ? 4 : 2;
    if ((rc = load_matrix(X, &G)) || (rc = check_lds(G, x->ld))) return rc;
    if (rows && (rc = check_i8(G, rows, false))) return rc;
    if (cols && (rc = check_i8(G, cols, true))) return rc;
    if ((rc = check_tiles(G, x->tiles, es)) || (rc = check_i8_blocks(G, es))) return rc;
    if (rows && (rc = i8_form(G, dtype, (char *const *)x->tiles, x->ld, rows, false, (hipStream_t)hip_stream))) return rc;
    return cols ? i8_form(G, dtype, (char *const *)x->tiles, x->ld, cols, true, (hipStream_t)hip_stream) : DMM_OK;
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_int_dequantize(const dmm_matrix_desc *X, const dmm_int_tiles *q, int along, int dtype, const dmm_tiles *x, void *hip_stream) {
  using namespace dmm;
  if (!X || !q || !x || !x->tiles || !x->ld) return DMM_EINVAL;
  if ((along != DMM_MX_ROWS && along != DMM_MX_COLS) || (dtype != DMM_BF16 && dtype != DMM_F32)) return DMM_EINVAL;
  TraceRange whole("dmm_int_dequantize");
  try {
    Grid G;
    int rc;
    const int es = dtype == DMM_F32 ? 4 : 2;
    const bool by_cols = along == DMM_MX_COLS;
    if ((rc = load_matrix(X, &G)) || (rc = check_lds(G, x->ld)) || (rc = check_i8(G, q, by_cols)) || (rc = check_tiles(G, x->tiles, es)) ||
        (rc = check_i8_blocks(G, es)))
      return rc;
    return over_i8_tiles(G, es, (char *const *)x->tiles, x->ld, q, by_cols, 128, i8_block_cols(es == 4),
                         [&](const I8Args &args, int blocks) { i8_values_launch(args, blocks, es == 4, by_cols, (hipStream_t)hip_stream); });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_int_execute(dmm_plan_t *P, const dmm_int_tiles *a, const dmm_int_tiles *b, const dmm_tiles *c, uint32_t flags, void *hip_stream) {
  using namespace dmm;
  if (!P || !a || !b || !c) return DMM_EINVAL;
  if (flags & ~(DMM_NO_REDUCE | DMM_C_BF16)) return DMM_EINVAL;
  if ((flags & DMM_C_BF16) && P->C.c != 1) return DMM_EINVAL;
  TraceRange whole("dmm_int_execute");
  try {
    return i8_product(P, LAYER_I8_EXECUTE, DMM_SILU, a, b, nullptr, c, (flags & DMM_C_BF16) ? 2 : 4, !(flags & DMM_NO_REDUCE), (hipStream_t)hip_stream);
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_int_gated_execute(dmm_plan_t *P, int activation, const dmm_int_tiles *a, const dmm_int_tiles *gate, const dmm_int_tiles *up, const dmm_tiles *h,
                         void *hip_stream) {
  using namespace dmm;
  if (!P || !a || !gate || !up || !h || !is_activation(activation) || P->C.c != 1) return DMM_EINVAL;
  TraceRange whole("dmm_int_gated_execute");
  try {
    return i8_product(P, LAYER_I8_GATED_EXECUTE, activation, a, gate, up, h, 2, false, (hipStream_t)hip_stream);
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_gated_execute(dmm_plan_t *P, int activation, const dmm_tiles *a, const dmm_tiles *gate, const dmm_tiles *up, const dmm_tiles *h, const dmm_tiles *g,
                      const dmm_tiles *u, void *hip_stream) {
  using namespace dmm;
  if (!P || !a || !gate || !up || !h || !is_activation(activation) || P->C.c != 1) return DMM_EINVAL;
  const Grid &A = P->A, &B = P->B, &C = P->C;
  int rc;
  if ((rc = check_layer_tiles(A, a, 2)) || (rc = check_layer_tiles(B, gate, 2)) || (rc = check_layer_tiles(B, up, 2)) || (rc = check_layer_tiles(C, h, 2)))
    return rc;
  if ((g && (rc = check_layer_tiles(C, g, 2))) || (u && (rc = check_layer_tiles(C, u, 2))) || (rc = check_sizes(P))) return rc;
  TraceRange whole("dmm_gated_execute");
  try {
    LayerKey key;
    key.put(&activation, sizeof activation);
    key.put(a, A.c * A.tiles_per_rep());
    key.put(gate, B.c * B.tiles_per_rep());
    key.put(up, B.c * B.tiles_per_rep());
    for (const dmm_tiles *t : {h, g, u}) key.put(t, C.tiles_per_rep());
    // the rows k0 to k1 of `n` columns of a tile of both weights, against what lies at `left`
    auto weights = [&](LayerWork *W, int64_t i, int32_t bi, int32_t bj, int64_t k0, int64_t k1, int64_t n0, int64_t n, const char *left, int64_t pitch) {
      LayerSeg s;
      s.a = left;
      s.b = corner(B, gate, i, bi, bj, k0, n0, 2);
      s.b2 = corner(B, up, i, bi, bj, k0, n0, 2);
      s.a_pitch = (uint32_t)pitch;
      s.b_pitch = (uint32_t)(gate->ld[i] * 2);
      s.b2_pitch = (uint32_t)(up->ld[i] * 2);
      int64_t guard = 0;
      for (const dmm_tiles *w : {gate, up})
        guard = std::max(guard, rows_past_end(B.rc[(size_t)bi + 1] - B.rc[(size_t)bi], B.cc[(size_t)bj + 1] - B.cc[(size_t)bj], w->ld[i], k1 - B.rc[(size_t)bi],
                                              n0 - B.cc[(size_t)bj], n));
      put_segment(W, s, k1 - k0, guard);
    };
    auto make = [&](int, LayerDense dense, LayerCopies *copies, bool) {
      LayerWork W;
      W.kind = LAYER_GATED;
      W.act = activation;
      W.c_es = 2;
      W.rows = C.rows;
      auto result = [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, LayerGroup *r) {
        const int64_t i = C.table_index(rep, ti, tj);
        r->c = corner(C, h, i, ti, tj, m0, n0, 2);
        r->ldc = h->ld[i];
        if (g) r->g = corner(C, g, i, ti, tj, m0, n0, 2), r->ldg = g->ld[i];
        if (u) r->u = corner(C, u, i, ti, tj, m0, n0, 2), r->ldu = u->ld[i];
      };
      if (dense == LAYER_LEFT || dense == LAYER_ROWS) {
        const bool whole = dense == LAYER_ROWS;
        const LayerCopies::Axis along(B.rc, 64);
        const LayerCopies::Matrix ca = copies->matrix(A, a->tiles, a->ld, 2, false, A.rows, along, false);
        LayerCopies::Matrix out[3] = {};
        const dmm_tiles *const results[3] = {h, g, u};
        for (int x = 0; x < 3 && whole; ++x)
          if (results[x]) out[x] = copies->results(C, results[x], 2);
        left_groups(
            P, whole, &W,
            [&](int32_t bi, int32_t bj, int64_t m0, int64_t n0, int64_t n) {
              weights(&W, B.table_index(0, bi, bj), bi, bj, B.rc[(size_t)bi], B.rc[(size_t)bi + 1], n0, n,
                      (const char *)(uintptr_t)(ca.at + (size_t)(m0 * ca.pitch + along.place(B.rc[(size_t)bi]) * 2)), ca.pitch);
            },
            [&](int32_t, int64_t m0, int64_t n0, LayerGroup *r) {
              if (!whole) return result(0, interval_of(C.rc, m0), interval_of(C.cc, n0), m0, n0, r);
              auto at = [&](int x) { return (char *)(uintptr_t)(out[x].at + (size_t)n0 * 2); };
              r->c = at(0), r->ldc = out[0].pitch / 2;
              if (g) r->g = at(1), r->ldg = out[1].pitch / 2;
              if (u) r->u = at(2), r->ldu = out[2].pitch / 2;
            });
        return W;
      }
      if (dense == LAYER_BOTH) {
        const LayerCopies::Axis along({0, A.cols}, 64), cols(C.cc, 64);
        const int64_t k = along.total;
        const LayerCopies::Matrix ca = copies->matrix(A, a->tiles, a->ld, 2, false, A.rows, along, true),
                                  cg = copies->matrix(B, gate->tiles, gate->ld, 2, false, k, cols, false),
                                  cu = copies->matrix(B, up->tiles, up->ld, 2, false, k, cols, false);
        tile_groups(
            C, &W,
            [&](int64_t m0, int64_t n0) {
              const size_t col = (size_t)cols.place(n0) * 2;
              W.segs.push_back(dense_segment(ca.at + (size_t)(m0 * ca.pitch), ca.pitch, cg.at + col, cg.pitch, cu.at + col, cu.pitch, k / 64));
            },
            result);
        return W;
      }
      plan_groups(
          P, &W,
          [&](const Group &gr, const dmm_task &t) {
            const int64_t ai = A.table_index(t.a_rep, t.a_ti, t.a_tj), bi = B.table_index(t.b_rep, t.b_ti, t.b_tj);
            weights(&W, bi, t.b_ti, t.b_tj, t.k0, t.k1, gr.n0, gr.n1 - gr.n0, corner(A, a, ai, t.a_ti, t.a_tj, gr.m0, t.k0, 2), a->ld[ai] * 2);
          },
          [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, const dmm_task *, LayerGroup *r) { result(rep, ti, tj, m0, n0, r); });
      return W;
    };
    return run_layer(P, LAYER_GATED_EXECUTE, key.bytes, nullptr, nullptr, false, (hipStream_t)hip_stream, 1, 1, false, make, [] { return DMM_OK; });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_gated_backward(dmm_plan_t *P, int activation, const dmm_tiles *a, const dmm_tiles *gate, const dmm_tiles *up, const dmm_tiles *g, const dmm_tiles *u,
                       const dmm_tiles *dh, const dmm_tiles *dg, const dmm_tiles *du, const dmm_tiles *da, const dmm_tiles *dgate, const dmm_tiles *dup,
                       uint32_t flags, void *hip_stream) {
  using namespace dmm;
  if (!P || !g || !u || !dh || !dg || !du || !is_activation(activation) || P->C.c != 1 || (flags & ~DMM_DB_F32)) return DMM_EINVAL;
  if ((da && (!gate || !up)) || ((dgate || dup) && !a)) return DMM_EINVAL;
  const Grid &A = P->A, &B = P->B, &C = P->C;
  const int es = (flags & DMM_DB_F32) ? 4 : 2;
  TraceRange whole("dmm_gated_backward");
  try {
    int rc;
    for (const dmm_tiles *t : {g, u, dh, dg, du})
      if ((rc = check_layer_tiles(C, t, 2))) return rc;
    if (da && ((rc = check_layer_tiles(B, gate, 2)) || (rc = check_layer_tiles(B, up, 2)) || (rc = check_layer_single(A, da, 2)))) return rc;
    if ((dgate || dup) && (rc = check_layer_tiles(A, a, 2))) return rc;
    if ((dgate && (rc = check_layer_single(B, dgate, es))) || (dup && (rc = check_layer_single(B, dup, es))) || (rc = check_sizes(P)) || (rc = check_slope(C)))
      return rc;
    LayerKey key;
    key.put(&flags, sizeof flags);
    key.put(dgate || dup ? a : nullptr, A.tiles_per_rep());
    for (const dmm_tiles *t : {da ? gate : nullptr, da ? up : nullptr, dgate, dup}) key.put(t, B.tiles_per_rep());
    for (const dmm_tiles *t : {dg, du}) key.put(t, C.tiles_per_rep());
    key.put(da, A.tiles_per_rep());
    const dmm_tiles *const bs[2] = {gate, up}, *const dcs[2] = {dg, du}, *const dbs[2] = {dgate, dup}, *const either[2] = {dgate ? dgate : dup, dup ? dup : dgate};
    const int first = da ? 0 : 1, last = dgate || dup ? 1 : 0;
    auto make = [&](int x, LayerDense dense, LayerCopies *copies, bool both) {
      return gradients(P, first + x == 0, a, bs, dcs, 2, da, both ? either : dbs, es, dense, copies);
    };
    hipStream_t stream = (hipStream_t)hip_stream;
    return run_layer(P, LAYER_GATED_BACKWARD, key.bytes, nullptr, nullptr, false, stream, std::max(0, last - first + 1), da != nullptr, (dgate != nullptr) != (dup != nullptr), make,
                     [&] { return slope(C, activation, g, u, dh, dg, du, stream); });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_execute_backward(dmm_plan_t *P, const dmm_tiles *a, const dmm_tiles *b, const dmm_tiles *dc, const dmm_tiles *da, const dmm_tiles *db, uint32_t flags,
                         void *hip_stream) {
  using namespace dmm;
  if (!P || !dc || (!da && !db) || (da && !b) || (db && !a) || (flags & ~DMM_DB_F32)) return DMM_EINVAL;
  const Grid &A = P->A, &B = P->B, &C = P->C;
  const int es = (flags & DMM_DB_F32) ? 4 : 2;
  TraceRange whole("dmm_execute_backward");
  try {
    int rc;
    if ((rc = check_layer_single(C, dc, 2))) return rc;
    if (da && ((rc = check_layer_single(B, b, 2)) || (rc = check_layer_single(A, da, 2)))) return rc;
    if (db && ((rc = check_layer_single(A, a, 2)) || (rc = check_layer_single(B, db, es)))) return rc;
    if ((rc = check_sizes(P))) return rc;
    LayerKey key;
    key.put(&flags, sizeof flags);
    key.put(db ? a : nullptr, A.tiles_per_rep());
    key.put(da, A.tiles_per_rep());
    key.put(da ? b : nullptr, B.tiles_per_rep());
    key.put(db, B.tiles_per_rep());
    key.put(dc, C.tiles_per_rep());
    const int first = da ? 0 : 1;
    auto make = [&](int x, LayerDense dense, LayerCopies *copies, bool) { return gradients(P, first + x == 0, a, &b, &dc, 1, da, &db, es, dense, copies); };
    return run_layer(P, LAYER_EXECUTE_BACKWARD, key.bytes, nullptr, nullptr, false, (hipStream_t)hip_stream, (da != nullptr) + (db != nullptr), da != nullptr, false, make,
                     [] { return DMM_OK; });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

}  // extern "C"
