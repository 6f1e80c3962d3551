// The entry points for 4-bit microscaled matrices (included by exec.hip): arguments checked on the host,
// tiles to be quantised handed to the kernels with the launch, products run from a plan's op list.
#pragma once

#include <cmath>

namespace dmm {
namespace {

constexpr int64_t kMxBlocks = (1 << 24) - 1;                   // workgroups of a launch: 2^32 threads are too many

// Pointers and pitches of one form of a matrix, checked: rows of codes hold whole chunks of 128 elements at multiples of 16
// bytes, rows of scales four bytes a chunk at multiples of 4.  `by_cols`: a tile's rows of codes are its columns.
int check_mx(const Grid &G, const dmm_mx_tiles *q, bool by_cols) {
  if (!q->codes || !q->code_ld || !q->scales || !q->scale_ld) return DMM_EINVAL;
  for (int32_t rep = 0; rep < G.c; ++rep)
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t h = G.rc[ti + 1] - G.rc[ti], w = G.cc[tj + 1] - G.cc[tj];
        if (h <= 0 || w <= 0) continue;
        const int64_t i = G.table_index(rep, ti, tj), chunks = ((by_cols ? h : w) + 127) / 128;
        if (!q->codes[i] || !q->scales[i] || ((uintptr_t)q->codes[i] & 15) || ((uintptr_t)q->scales[i] & 3)) return DMM_EINVAL;
        if (q->code_ld[i] < chunks * 64 || q->code_ld[i] % 16 || q->scale_ld[i] < chunks * 4 || q->scale_ld[i] % 4) return DMM_ELD;
        if (q->code_ld[i] >= (int64_t)1 << 24 || q->scale_ld[i] >= (int64_t)1 << 24) return DMM_ELD;
      }
  return DMM_OK;
}

// A matrix by itself: no ranks to deal its tiles to, so the process grid plays no part.
int load_matrix(const dmm_matrix_desc *d, Grid *g) {
  if (d->grid_rows < 1 || d->grid_cols < 1 || d->replication < 1) return DMM_EINVAL;
  const int64_t *cuts[2] = {d->row_cuts, d->col_cuts};
  const int32_t n[2] = {d->grid_rows, d->grid_cols};
  const int64_t dim[2] = {d->rows, d->cols};
  for (int x = 0; x < 2; ++x) {
    if (!cuts[x] || dim[x] < 0 || cuts[x][0] != 0 || cuts[x][n[x]] != dim[x]) return DMM_EINVAL;
    for (int32_t i = 0; i < n[x]; ++i)
      if (cuts[x][i + 1] < cuts[x][i]) return DMM_EINVAL;
    // (tiles are addressed with 32-bit rows and columns, filled up to whole blocks)
    for (int32_t i = 0; i < n[x]; ++i)
      if (cuts[x][i + 1] - cuts[x][i] > 0x7fffff00) return DMM_EINVAL;
  }
  g->rows = d->rows;
  g->cols = d->cols;
  g->gr = d->grid_rows;
  g->gc = d->grid_cols;
  g->rc.assign(d->row_cuts, d->row_cuts + d->grid_rows + 1);
  g->cc.assign(d->col_cuts, d->col_cuts + d->grid_cols + 1);
  g->c = d->replication;
  return DMM_OK;
}

int allow_mx_lds() {
  static std::mutex mu;
  static bool done[64] = {};
  int device = 0;
  DMM_HIP(hipGetDevice(&device));
  if (device < 0 || device >= 64) return DMM_EINVAL;
  std::lock_guard<std::mutex> g(mu);
  if (!done[device]) {
    DMM_HIP(mx_allow_lds());
    done[device] = true;
  }
  return DMM_OK;
}

// Runs `launch` over all tiles, as many at a time as a launch's argument holds.
template <class F>
int over_tiles(const Grid &G, int es, char *const *x, const int64_t *x_ld, const dmm_mx_tiles *rows, const dmm_mx_tiles *cols, F launch) {
  int64_t units = 0;
  for (int32_t ti = 0; ti < G.gr; ++ti)
    for (int32_t tj = 0; tj < G.gc; ++tj) units += G.c * (G.rc[ti + 1] - G.rc[ti]) * ((G.cc[tj + 1] - G.cc[tj] + 511) / 512);
  const int per = mx_rows_per_unit(units);
  const int along = (rows ? MX_ALONG_ROWS : 0) | (cols ? MX_ALONG_COLS : 0);
  // workgroups of a tile, and how many of them side by side
  auto blocks_of = [&](int64_t h, int64_t w, int32_t *across) -> int64_t {
    if (along == MX_ALONG_ROWS) {
      *across = (int32_t)((w + 511) / 512);
      return ((h + per - 1) / per * *across + 3) / 4;
    }
    // (with the rows too, down to the end of the last chunk)
    const int64_t cols = mx_block_cols(es == 4), wide = rows ? (w + 127) / 128 * 128 : w;
    *across = (int32_t)((wide + cols - 1) / cols);
    return (h + 127) / 128 * *across;
  };
  // (all tiles before the first launch: a call that is refused writes nothing)
  for (int32_t ti = 0; ti < G.gr; ++ti)
    for (int32_t tj = 0; tj < G.gc; ++tj) {
      int32_t across;
      if (blocks_of(G.rc[ti + 1] - G.rc[ti], G.cc[tj + 1] - G.cc[tj], &across) > kMxBlocks) return DMM_ELIMIT;
    }
  MxTileArgs args;
  std::memset(&args, 0, sizeof args);
  int64_t blocks = 0;
  auto flush = [&]() -> int {
    if (!args.n) return DMM_OK;
    launch(args, (int)blocks, along, per);
    args.n = 0;
    blocks = 0;
    DMM_HIP(hipGetLastError());
    return DMM_OK;
  };
  for (int32_t rep = 0; rep < G.c; ++rep)
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        const int64_t h = G.rc[ti + 1] - G.rc[ti], w = G.cc[tj + 1] - G.cc[tj];
        if (h <= 0 || w <= 0) continue;
        const int64_t i = G.table_index(rep, ti, tj);
        MxTile t;
        std::memset(&t, 0, sizeof t);
        t.x = x[i];
        t.x_pitch = x_ld[i] * es;
        if (rows) {
          t.row_codes = (char *)rows->codes[i];
          t.row_pitch = rows->code_ld[i];
          t.row_scales = (unsigned char *)rows->scales[i];
          t.row_scale_pitch = rows->scale_ld[i];
        }
        if (cols) {
          t.col_codes = (char *)cols->codes[i];
          t.col_pitch = cols->code_ld[i];
          t.col_scales = (unsigned char *)cols->scales[i];
          t.col_scale_pitch = cols->scale_ld[i];
        }
        t.h = (int32_t)h;
        t.w = (int32_t)w;
        const int64_t n = blocks_of(h, w, &t.blocks_across);
        int rc;
        if ((args.n == MX_TILES || blocks + n > kMxBlocks) && (rc = flush())) return rc;
        t.first_block = (int32_t)blocks;
        blocks += n;
        args.tile[args.n++] = t;
      }
  return flush();
}

// ---- products -----------------------------------------------------------------------------------------

// Blocks of A and of B have to meet: every op starts at a whole chunk of both tiles.  (It then ends at one, or where
// both tiles end: the next op starts there.)
int check_chunks(const dmm_plan_t *P) {
  for (const dmm_task &t : P->tasks)
    if ((t.k0 - P->A.cc[(size_t)t.a_tj]) % DMM_MX_CHUNK || (t.k0 - P->B.rc[(size_t)t.b_ti]) % DMM_MX_CHUNK) return DMM_EINVAL;
  return DMM_OK;
}

// Which kernel runs a plan's product, and into how many ranges of K its tiles are cut.
struct MxChoice {
  int shape = MX_256;
  int64_t runs = 1;                    // of a tile of average length
};

// By an estimate in us.  What a step (256 of k) of a tile costs, measured as what more of K costs:
//   256 x 256  1.4 to 2.0 with all CUs at it (random codes more than normal data: power)
//   128 x 128  0.54 (64 tiles) to 0.66 (256); two on a CU 1.1 to 1.4
//   64 x 128   0.5 (112) and 0.55 (224) where a cache holds B, 0.8 and 0.95 where it comes from memory (two stages); two on a CU 1.1 to 1.25
//   32 x 128   0.35 and 0.5, from memory 0.55 and 0.75 (three stages); two on a CU 1.0 to 1.1
// and none is faster than memory: 570 MB of B take tiles of 32 113 us, of 64 130, of 128 131, of 256 149; 125 MB 27, 34, 30, 50.  Up to 32 rows the
// tile of 32 is the best everywhere.  From 33 to 64 it is that of 64, or that of 128 where almost every CU has one and B comes from memory: 64 x 4096 x 14336 16.7
// and 17.2, 64 x 4096 x 28000 20.9 and 18.8 (13.0 and 15.0 with B in the cache, which the choice does not know).  A tile cut along K costs its
// partial sums and a launch that adds them up.  Of equal estimates the smaller tile's.
MxChoice choose_mx(const dmm_plan_t *P, int cus) {
  int64_t most = 0;                    // rows of a group
  double cells = 0, k_steps = 0, b_bytes = 0, b_once = 0;
  struct Columns {
    int32_t rep;
    int64_t n0;
    double bytes;
  };
  std::vector<Columns> columns;        // of B, for every group that reads them
  for (size_t x = 0; x < P->groups.size(); ++x) {
    const Group &g = P->groups[x];
    most = std::max(most, g.m1 - g.m0);
    int64_t steps = 0;
    for (int64_t y = g.first; y < g.first + g.count; ++y) {
      const dmm_task &t = P->tasks[(size_t)P->order[(size_t)y]];
      steps += (t.k1 - t.k0 + 255) / 256;
    }
    const double area = (double)(g.m1 - g.m0) * (double)(g.n1 - g.n0), bytes = (double)(g.n1 - g.n0) * (double)steps * 136.0;
    cells += area;
    k_steps += area * (double)steps;
    b_bytes += bytes;
    columns.push_back({g.c_rep, g.n0, bytes});
  }
  std::sort(columns.begin(), columns.end(), [](const Columns &a, const Columns &b) { return a.rep != b.rep ? a.rep < b.rep : a.n0 < b.n0; });
  for (size_t x = 0; x < columns.size(); ++x)
    if (!x || columns[x].rep != columns[x - 1].rep || columns[x].n0 != columns[x - 1].n0) b_once += columns[x].bytes;
  const double steps = cells > 0 ? k_steps / cells : 0;
  const double cold = b_bytes > 0 ? b_once / b_bytes : 0;   // of what is read of B, the part that comes from memory
  MxChoice best;
  double best_us = 0;
  for (const int shape : {MX_SKINNY, MX_32, MX_64, MX_128, MX_256}) {
    const int tm = kMxShape[shape].tm, tn = kMxShape[shape].tn;
    if ((shape == MX_SKINNY && most > 32) || (shape == MX_32 && most > tm) || (shape == MX_64 && most > tm)) continue;
    double tiles = 0;
    for (const Group &g : P->groups) tiles += (double)(((g.m1 - g.m0 + tm - 1) / tm) * ((g.n1 - g.n0 + tn - 1) / tn));
    if (tiles == 0) return best;
    if (tiles > (double)kMxBlocks) continue;
    if (shape == MX_SKINNY) {
      // (every eighth pair of chunks is a wave's next; 16 rows of A are read with every 16 columns of B, and B again with 16 more rows.  Workgroups on
      // one CU share its first cache, which takes 0.8 to 1.3 us for eight steps of each: 128 x 47936 x 532 on 8 blocks of rows, 360 tiles, 62 us)
      const double us = 2.5 + std::max((most <= 2 ? 0.8 : 1.2) * std::ceil(steps / 8) * std::ceil(tiles / cus),
                                       b_bytes / (most <= 2 ? 4.6e6 : 3.0e6) + (double)((most - 1) / 16) * b_bytes / 8e6);
      if (best_us == 0 || us < best_us) best_us = us, best.shape = shape, best.runs = 1;
      continue;
    }
    const int places = shape == MX_256 ? cus : 2 * cus;
    const double memory = 2.0 + b_once / (shape == MX_32 ? 5.0e6 : 4.4e6);
    for (int64_t runs = 1; runs <= 32; ++runs) {
      const double work = tiles * (double)runs, per = std::ceil(steps / (double)runs);
      if (runs > 1 && (work > places || per < 3)) break;
      // rounds of all places, and one of the rest
      auto round = [&](double n) {
        if (n <= 0) return 0.0;
        const double full = n / cus;
        switch (shape) {
          case MX_256: return per * (1.2 + 0.55 * full) + 8.0;
          case MX_128: return per * (full > 1 ? 1.13 : 0.5 + 0.16 * full) + 4.5;
          case MX_64: return per * (full > 1 ? 1.15 : 0.33 + (0.25 + 0.37 * cold) * full) + 3.5;
          default: return per * (full > 1 ? 1.05 : 0.3 + (0.22 + 0.28 * cold) * full) + 3.5;
        }
      };
      const double whole = std::floor(work / places);
      double us = std::max(whole * round(places) + round(work - whole * places), memory);
      if (runs > 1) us += 4.5 + 2.0 * work * tm * tn * 4 / 3e6;
      if (best_us == 0 || us < best_us) best_us = us, best.shape = shape, best.runs = runs;
    }
  }
  return best;
}

int build_mx(dmm_plan_t *P, const dmm_mx_tiles *a, const dmm_mx_tiles *b, void *const *c_tiles, const int64_t *c_ld, int c_es, int cus,
             hipStream_t stream, MxLayout *L) {
  const Grid &A = P->A, &B = P->B, &C = P->C;
  std::vector<NtSeg> segs;
  std::vector<int32_t> group_seg, group_steps;                // a group's first segment; its K steps
  for (const Group &g : P->groups) {
    group_seg.push_back((int32_t)segs.size());
    int64_t steps = 0;
    for (int64_t x = g.first; x < g.first + g.count; ++x) {
      const dmm_task &t = P->tasks[(size_t)P->order[(size_t)x]];
      const int64_t ai = A.table_index(t.a_rep, t.a_ti, t.a_tj), bi = B.table_index(t.b_rep, t.b_ti, t.b_tj);
      const int64_t ak = t.k0 - A.cc[(size_t)t.a_tj], bk = t.k0 - B.rc[(size_t)t.b_ti];
      const int64_t ar = g.m0 - A.rc[(size_t)t.a_ti], bc = g.n0 - B.cc[(size_t)t.b_tj];
      NtSeg s;
      s.a = (const char *)a->codes[ai] + ar * a->code_ld[ai] + ak / 2;
      s.b = (const char *)b->codes[bi] + bc * b->code_ld[bi] + bk / 2;
      s.a_scale = (const char *)a->scales[ai] + ar * a->scale_ld[ai] + ak / 32;
      s.b_scale = (const char *)b->scales[bi] + bc * b->scale_ld[bi] + bk / 32;
      s.a_pitch = (uint32_t)a->code_ld[ai];
      s.b_pitch = (uint32_t)b->code_ld[bi];
      s.a_scale_pitch = (uint32_t)a->scale_ld[ai];
      s.b_scale_pitch = (uint32_t)b->scale_ld[bi];
      s.chunks = (int32_t)((t.k1 - t.k0 + 127) / 128);
      s.pad = 0;
      steps += (s.chunks + 1) / 2;
      segs.push_back(s);
    }
    if (steps > 0x3fffffff || segs.size() > 0x3fffffff) return DMM_ELIMIT;
    group_steps.push_back((int32_t)steps);
  }
  group_seg.push_back((int32_t)segs.size());

  const MxChoice choice = choose_mx(P, cus);
  const int shape = choice.shape;
  const int tm = kMxShape[shape].tm, tn = kMxShape[shape].tn;
  auto corner = [&](int32_t rep, int32_t ti, int32_t tj, int64_t m0, int64_t n0, MxItem *it) {
    const int64_t i = C.table_index(rep, ti, tj);
    it->ldc = c_ld[i];
    it->c = (char *)c_tiles[i] + ((m0 - C.rc[(size_t)ti]) * c_ld[i] + n0 - C.cc[(size_t)tj]) * c_es;
    it->c_es = c_es;
    it->pad = 0;
    return c_tiles[i] != nullptr;
  };
  std::vector<MxItem> items;
  std::vector<MxJoin> joins;
  int64_t slots = 0;
  for (size_t x = 0; x < P->groups.size(); ++x) {
    const Group &g = P->groups[x];
    const int64_t rows = (g.m1 - g.m0 + tm - 1) / tm, cols = (g.n1 - g.n0 + tn - 1) / tn;
    int64_t runs = std::min<int64_t>(choice.runs, std::max(1, group_steps[x] / 3));
    const int32_t per = (int32_t)((group_steps[x] + runs - 1) / runs);
    runs = (group_steps[x] + per - 1) / per;
    // bands of eight tile rows, column by column: neighbours in the list share operands.  All first ranges of K, then all second ones, ...
    const int64_t first_slot = slots;
    int32_t seg = group_seg[x], first = 0;
    for (int64_t run = 0; run < runs; ++run) {
      const int32_t n_steps = std::min<int32_t>(per, group_steps[x] - (int32_t)run * per);
      int64_t tile = 0;
      for (int64_t r0 = 0; r0 < rows; r0 += 8)
        for (int64_t c = 0; c < cols; ++c)
          for (int64_t r = r0; r < std::min(r0 + 8, rows); ++r, ++tile) {
            MxItem it;
            if (!corner(g.c_rep, g.c_ti, g.c_tj, g.m0 + r * tm, g.n0 + c * tn, &it)) return DMM_EINVAL;
            it.m_off = (int32_t)(r * tm);
            it.n_off = (int32_t)(c * tn);
            it.m_ext = (int32_t)std::min<int64_t>(tm, g.m1 - g.m0 - r * tm);
            it.n_ext = (int32_t)std::min<int64_t>(tn, g.n1 - g.n0 - c * tn);
            it.front = seg < group_seg[x + 1] ? segs[(size_t)seg] : NtSeg{};
            it.seg = seg;
            it.n_segs = group_seg[x + 1] - seg;
            it.first = first;
            it.steps = n_steps;
            if (runs > 1) {
              const int64_t slot = first_slot + tile * runs;
              if (run == 0) joins.push_back({it.c, it.ldc, (const float *)(uintptr_t)slot, (int32_t)runs, tm, tn, it.m_ext, it.n_ext, c_es});
              it.c = (char *)(uintptr_t)(slot + run);
              it.ldc = tn;
              it.c_es = 4;
              it.pad = 1;
              ++slots;
            }
            items.push_back(it);
          }
      first += n_steps;
      while (seg < group_seg[x + 1] && first >= (segs[(size_t)seg].chunks + 1) / 2) first -= (segs[(size_t)seg++].chunks + 1) / 2;
    }
  }
  // regions of C that no op writes: zeros
  for (const dmm_work_item &w : P->items) {
    if (w.group >= 0) continue;
    for (int32_t r = 0; r < w.m_ext; r += tm)
      for (int32_t c = 0; c < w.n_ext; c += tn) {
        MxItem it;
        std::memset(&it, 0, sizeof it);
        if (!corner(w.c_rep, w.c_ti, w.c_tj, w.m0 + r, w.n0 + c, &it)) return DMM_EINVAL;
        it.m_ext = std::min(tm, w.m_ext - r);
        it.n_ext = std::min(tn, w.n_ext - c);
        items.push_back(it);
      }
  }
  if (items.empty()) {
    L->n_items = 0;
    return DMM_OK;
  }
  if ((int64_t)items.size() > kMxBlocks) return DMM_ELIMIT;
  // workgroup w runs on XCD w % 8: every XCD gets a run of the list
  std::vector<MxItem> ordered(items.size());
  {
    const size_t n = items.size();
    size_t from = 0;
    for (size_t xcd = 0; xcd < 8; ++xcd)
      for (size_t w = xcd; w < n; w += 8) ordered[w] = items[from++];
  }
  int rc;
  MxState &M = P->dev->mx;
  if (slots) {
    const size_t slot = (size_t)tm * tn * 4, need = (size_t)slots * slot;
    if ((rc = P->dev->uses.order(stream))) return rc;
    if (need > M.cap) {
      if (M.buf) {
        if ((rc = P->dev->uses.wait())) return rc;
        DMM_HIP(hipStreamSynchronize(stream));
        scratch_pool().release(&M.buf, &M.cap);
      }
      if ((rc = scratch_pool().acquire(need, &M.buf, &M.cap))) return rc;
    }
    for (MxItem &it : ordered)
      if (it.pad) it.c = M.buf + (uintptr_t)it.c * slot;
    for (MxJoin &j : joins) j.parts = (const float *)(M.buf + (uintptr_t)j.parts * slot);
  }
  L->shape = shape;
  L->n_items = (int)ordered.size();
  L->n_joins = (int)joins.size();
  L->o_segs = ordered.size() * sizeof(MxItem);
  L->o_joins = L->o_segs + segs.size() * sizeof(NtSeg);
  std::vector<char> &h = P->dev->host;
  h.resize(L->o_joins + joins.size() * sizeof(MxJoin));
  std::memcpy(h.data(), ordered.data(), ordered.size() * sizeof(MxItem));
  if (!segs.empty()) std::memcpy(h.data() + L->o_segs, segs.data(), segs.size() * sizeof(NtSeg));
  if (!joins.empty()) std::memcpy(h.data() + L->o_joins, joins.data(), joins.size() * sizeof(MxJoin));
  static_assert(sizeof(MxItem) % 8 == 0 && sizeof(NtSeg) % 8 == 0 && sizeof(MxJoin) % 8 == 0, "tables lie one behind another");
  // those of the sum of C's replicas, also for a call without it: the next one with these arguments may be captured
  if ((rc = build_reduce(P, c_tiles, c_ld, 0, &h, h.size(), &L->red))) return rc;
  if ((rc = M.table.upload(h.data(), h.size(), stream, P->dev->uses))) return rc;
  L->red.dev_base = M.table.dev();
  return DMM_OK;
}

}  // namespace
}  // namespace dmm

extern "C" {

int dmm_mx_quantize(const dmm_matrix_desc *X, int dtype, const void *const *x_tiles, const int64_t *x_ld, const dmm_mx_tiles *rows,
                    const dmm_mx_tiles *cols, void *hip_stream) {
  using namespace dmm;
  if (!X || !x_tiles || !x_ld || (!rows && !cols)) return DMM_EINVAL;
  if (dtype != DMM_BF16 && dtype != DMM_F32) return DMM_EINVAL;
  TraceRange whole("dmm_mx_quantize");
  try {
    Grid G;
    int rc;
    if ((rc = load_matrix(X, &G)) || (rc = check_lds(G, x_ld))) return rc;
    if (rows && (rc = check_mx(G, rows, false))) return rc;
    if (cols && (rc = check_mx(G, cols, true))) return rc;
    if ((rc = check_tiles(G, x_tiles, dtype == DMM_F32 ? 4 : 2))) return rc;
    return over_tiles(G, dtype == DMM_F32 ? 4 : 2, (char *const *)x_tiles, x_ld, rows, cols, [&](const MxTileArgs &args, int blocks, int along, int per) {
      mx_quantize_launch(args, blocks, dtype == DMM_F32, along, per, (hipStream_t)hip_stream);
    });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_mx_dequantize(const dmm_matrix_desc *X, const dmm_mx_tiles *q, int along, int dtype, void *const *x_tiles, const int64_t *x_ld,
                      void *hip_stream) {
  using namespace dmm;
  if (!X || !q || !x_tiles || !x_ld) return DMM_EINVAL;
  if ((along != DMM_MX_ROWS && along != DMM_MX_COLS) || (dtype != DMM_BF16 && dtype != DMM_F32)) return DMM_EINVAL;
  TraceRange whole("dmm_mx_dequantize");
  try {
    Grid G;
    int rc;
    if ((rc = load_matrix(X, &G)) || (rc = check_lds(G, x_ld)) || (rc = check_mx(G, q, along == DMM_MX_COLS))) return rc;
    if ((rc = check_tiles(G, x_tiles, dtype == DMM_F32 ? 4 : 2))) return rc;
    return over_tiles(G, dtype == DMM_F32 ? 4 : 2, (char *const *)x_tiles, x_ld, along == DMM_MX_ROWS ? q : nullptr, along == DMM_MX_COLS ? q : nullptr,
                      [&](const MxTileArgs &args, int blocks, int by, int per) {
                        mx_values_launch(args, blocks, dtype == DMM_F32, by, per, (hipStream_t)hip_stream);
                      });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_mx_execute(dmm_plan_t *P, const dmm_mx_tiles *a, const dmm_mx_tiles *b, void *const *c_tiles, const int64_t *c_ld, uint32_t flags,
                   void *hip_stream) {
  using namespace dmm;
  if (!P || !a || !b || !c_tiles || !c_ld) return DMM_EINVAL;
  if (flags & ~(DMM_NO_REDUCE | DMM_C_BF16)) return DMM_EINVAL;
  if ((flags & DMM_C_BF16) && P->C.c != 1) return DMM_EINVAL;
  const int c_es = (flags & DMM_C_BF16) ? 2 : 4;
  int rc;
  if ((rc = check_mx(P->A, a, false)) || (rc = check_mx(P->B, b, true)) || (rc = check_lds(P->C, c_ld)) ||
      (rc = check_tiles(P->C, c_tiles, c_es)))
    return rc;
  for (int64_t i = 0; i < P->C.c * P->C.tiles_per_rep(); ++i)
    if (c_ld[i] >= ((int64_t)1 << 24) / c_es) return DMM_ELD;
  hipStream_t stream = (hipStream_t)hip_stream;
  TraceRange whole("dmm_mx_execute");
  try {
    const bool capturing = is_capturing(stream), known = P->dev && P->dev->mx.cached;
    if (!known && ((rc = materialize(P)) || (rc = check_chunks(P)))) return rc;
    if (capturing && !known) return DMM_EINVAL;                // (a graph cannot wait for tables that are on their way)
    if ((rc = ensure_state(P)) || (rc = allow_mx_lds())) return rc;
    int device = 0, cus = 0;
    DMM_HIP(hipGetDevice(&device));
    if ((rc = device_cus(&cus))) return rc;
    MxState &M = P->dev->mx;
    // a call with the tables of the call before it launches from what that left on the device
    std::vector<char> &key = P->dev->key_scratch;
    key.clear();
    auto put = [&key](const void *p, size_t bytes) { key.insert(key.end(), (const char *)p, (const char *)p + bytes); };
    const int64_t head[2] = {c_es, device};
    put(head, sizeof head);
    const size_t na = (size_t)(P->A.c * P->A.tiles_per_rep()), nb = (size_t)(P->B.c * P->B.tiles_per_rep()), nc = (size_t)(P->C.c * P->C.tiles_per_rep());
    const dmm_mx_tiles *operand[2] = {a, b};
    for (int x = 0; x < 2; ++x) {
      const size_t n = x ? nb : na;
      put(operand[x]->codes, n * sizeof(void *));
      put(operand[x]->code_ld, n * sizeof(int64_t));
      put(operand[x]->scales, n * sizeof(void *));
      put(operand[x]->scale_ld, n * sizeof(int64_t));
    }
    put(c_tiles, nc * sizeof(void *));
    put(c_ld, nc * sizeof(int64_t));
    if (M.cached && key == M.key) {
      if ((rc = M.table.order_behind_copy(stream))) return rc;
      if (M.layout.n_joins && (rc = P->dev->uses.order(stream))) return rc;
    } else {
      if (capturing) return DMM_EINVAL;
      M.cached = false;
      MxLayout L;
      if ((rc = build_mx(P, a, b, c_tiles, c_ld, c_es, cus, stream, &L))) return rc;
      M.key = key;
      M.layout = L;
      M.cached = true;
    }
    const MxLayout &L = M.layout;
    if (L.n_items == 0) return DMM_OK;
    const bool sum = L.red.n_items && !(flags & DMM_NO_REDUCE);
    hipEvent_t behind = nullptr;
    if ((rc = P->dev->uses.claim(stream, &behind))) return rc;
    const char *d = M.table.dev();
    bool marked = mx_launch(sum ? nullptr : behind, L.shape, (const MxItem *)d, L.n_items, (const NtSeg *)(d + L.o_segs),
                            (const MxJoin *)(d + L.o_joins), L.n_joins, cus, stream);
    DMM_HIP(hipGetLastError());
    if (sum && (rc = fire_reduce(P, L.red, stream, false, behind, &marked))) return rc;
    return marked ? DMM_OK : P->dev->uses.mark(stream);
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

}  // extern "C"
