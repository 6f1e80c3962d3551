// dmm_orthogonalize (included by exec.hip): the layout of its workspace and the launches.
#pragma once

#include <cmath>

namespace dmm {
namespace {

static_assert(ORTHO_STEPS == DMM_ORTHOGONALIZE_STEPS, "coefficients travel with the launch");
constexpr int kOrthoSums = 1024;       // workgroups that add up the squares of a matrix, about
constexpr int64_t kOrthoBlocks = (1 << 24) - 1;   // workgroups of a launch: 2^32 threads are too many
constexpr int kOrthoCus = 256;          // how products are cut along K, and so the workspace, does not depend on the device

// How a symmetric (X X^T, S S) or plain (P X) product of m x n outputs and K steps is cut.
struct OrthoCut {
  int edge, tiles_m, tiles_n, tiles, runs, per;
  int whole;                           // tiles of all matrices that are not cut along K
  size_t parts;                        // bytes of partial sums
};
// Tiles that fill the device evenly are not cut; the others (all of them, where they are few) are cut along K if an
// estimate finds that faster.
OrthoCut ortho_cut(int64_t m, int64_t n, bool symmetric, int64_t steps, int64_t count) {
  OrthoCut best;
  double best_us = 0.0;
  for (int edge = 64; edge <= 256; edge *= 2) {
    OrthoCut c;
    c.edge = edge;
    c.tiles_m = (int)((m + edge - 1) / edge);
    c.tiles_n = (int)((n + edge - 1) / edge);
    c.tiles = symmetric ? c.tiles_m * (c.tiles_m + 1) / 2 : c.tiles_m * c.tiles_n;
    const int places = kOrthoCus * (edge == 256 ? 1 : edge == 128 ? 2 : 3);
    const int64_t tiles = c.tiles * count, rest = tiles % places;
    // us: a step of tiles of 256, of two of 128 on a CU, of one (the more there are the longer L2 takes, and the less power is
    // left for each), of one to three of 64 (of the CU that has most); and a tile's ends.  Tiles of 64 do 0.6 of the work of 128 in the time where the device is
    // full, and have less of it where it is not: X X^T of 513 x 700 8 us instead of 12, 16 of 300 x 700 17 instead of 28, but P X of
    // 2048 x 2048 55 instead of 49.
    auto round = [&](int64_t n_tiles, int64_t n_steps, bool cut) {
      if (n_tiles == 0) return 0.0;
      const double full = (double)n_tiles / kOrthoCus;
      if (edge == 64) return (0.03 + 0.19 * std::ceil(full)) * (double)n_steps + (cut ? 5.0 : 6.5);
      const double step = edge == 256 ? 1.45 + 0.9 * full : full > 1.0 ? 1.35 : 0.4 + 0.2 * full;
      return step * (double)n_steps + (edge == 256 ? 14.0 : cut ? 6.0 : 11.0);
    };
    const double whole_us = (tiles / places) * round(places, steps, false);
    for (int64_t runs = 1; runs <= 32; ++runs) {
      const int64_t per = (steps + runs - 1) / runs;
      if (runs > 1 && (rest == 0 || rest * runs > places || per < 4 || (steps + per - 1) / per != runs)) continue;
      const double bytes = runs > 1 ? 2.0 * rest * runs * edge * edge * 4 : 0.0;
      const double us = whole_us + round(rest * runs, per, runs > 1) + (runs > 1 ? 5.0 + bytes / 3e6 : 0.0);
      if (best_us == 0.0 || us < best_us) {
        best_us = us;
        best = c;
        best.runs = (int)runs;
        best.per = (int)per;
        best.whole = (int)(runs > 1 ? tiles - rest : tiles);
        best.parts = (size_t)(bytes / 2);
      }
    }
  }
  return best;
}

struct OrthoLayout {
  int64_t s, l, sp, lp;                // fewer rows, more columns; filled up to multiples of 32
  bool flip;                           // the matrix has more rows than columns: its transpose is worked on
  // byte offsets in a matrix' buffers: two generations of X by rows and by columns, S, P
  int64_t wide[2], tall[2], S, P, stride;
  int64_t tiles;                       // non-empty tiles of a matrix
  int64_t sums, o_sums, o_parts, total;
  OrthoCut cut_s, cut_p, cut_x;
  bool small;                          // a workgroup a matrix, no workspace
};

int ortho_layout(const Grid &G, int32_t count, OrthoLayout *L) {
  // (rows and columns are 32-bit numbers in the kernels, and so are workgroups)
  if (G.rows > 1 << 20 || G.cols > 1 << 20) return DMM_ELIMIT;
  auto up = [](int64_t x, int64_t m) { return (x + m - 1) / m * m; };
  L->flip = G.rows > G.cols;
  L->s = std::min(G.rows, G.cols);
  L->l = std::max(G.rows, G.cols);
  L->sp = up(L->s, 32);
  L->lp = up(L->l, 32);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at = up(at + bytes, 256);
    return o;
  };
  for (int i = 0; i < 2; ++i) {
    L->wide[i] = take(4 * L->s * L->lp);
    L->tall[i] = take(4 * L->l * L->sp);
  }
  L->S = take(4 * L->s * L->sp);
  L->P = take(4 * L->s * L->sp);
  L->stride = at;
  L->tiles = 0;
  for (int32_t i = 0; i < G.gr; ++i)
    for (int32_t j = 0; j < G.gc; ++j) L->tiles += G.rc[(size_t)i + 1] > G.rc[(size_t)i] && G.cc[(size_t)j + 1] > G.cc[(size_t)j];
  // one tile, and no more than registers and LDS of a CU hold
  L->small = G.gr == 1 && G.gc == 1 && L->l <= ORTHO_SMALL && L->s > 0 && count > 0;
  L->total = 0;
  if (L->small || L->s == 0 || count == 0) return DMM_OK;
  if (at > (int64_t)1 << 46 || (L->s + 127) / 128 * ((L->l + 127) / 128) > ((int64_t)1 << 21) / count) return DMM_ELIMIT;
  at *= count;
  L->sums = kOrthoSums + L->tiles;
  L->o_sums = take(count * L->sums * 8);
  L->cut_s = ortho_cut(L->s, L->s, true, L->lp / 32, count);
  L->cut_p = ortho_cut(L->s, L->s, true, L->sp / 32, count);
  L->cut_x = ortho_cut(L->s, L->l, false, L->sp / 32, count);
  L->o_parts = take((int64_t)std::max({L->cut_s.parts, L->cut_p.parts, L->cut_x.parts}));
  L->total = at;
  return DMM_OK;
}

// Whether every matrix on the way stays below 15 (2^12 times that has a place in fp16): bounds on the singular values, from 1 on.
bool ortho_in_range(const float *c, int32_t steps) {
  double top = 1.0;
  for (int32_t i = 0; i < steps; ++i, c += 3) {
    if (!std::isfinite(c[0]) || !std::isfinite(c[1]) || !std::isfinite(c[2])) return false;
    double next = 0.0, poly = 0.0;
    for (int x = 0; x <= 4096; ++x) {
      const double v = top * x / 4096, q = v * v, p = c[1] * q + c[2] * q * q;
      poly = std::max(poly, std::max(std::fabs(p), std::fabs(c[0] + p)));
      next = std::max(next, std::fabs(v * (c[0] + p)));
    }
    if (!(top * top <= 15.0) || !(poly <= 15.0) || !(next <= 15.0)) return false;
    top = next * 1.001;                // (between the points, and rounding on the way)
  }
  return true;
}

constexpr float kOrthoCoefficients[15] = {3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f,
                                          2.0315f, 3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f};

// Runs `launch` over the tiles of all matrices, as many at a time as a launch's argument holds; `blocks(h, w, &across)` workgroups a tile.
template <class B, class F>
int over_ortho_tiles(const Grid &G, int32_t count, OrthoTiles &args, int es, char *const *p, const int64_t *ld, B blocks_of, F launch) {
  int64_t blocks = 0;
  args.n = 0;
  auto flush = [&]() -> int {
    if (!args.n) return DMM_OK;
    launch((int)blocks);
    args.n = 0;
    blocks = 0;
    DMM_HIP(hipGetLastError());
    return DMM_OK;
  };
  for (int32_t x = 0; x < count; ++x) {
    int64_t before = 0;                // workgroups of this matrix' tiles in front
    for (int32_t ti = 0; ti < G.gr; ++ti)
      for (int32_t tj = 0; tj < G.gc; ++tj) {
        OrthoTile t;
        t.row0 = (int32_t)G.rc[(size_t)ti];
        t.col0 = (int32_t)G.cc[(size_t)tj];
        t.h = (int32_t)G.rc[(size_t)ti + 1] - t.row0;
        t.w = (int32_t)G.cc[(size_t)tj + 1] - t.col0;
        if (t.h <= 0 || t.w <= 0) continue;
        const int64_t i = x * G.tiles_per_rep() + (int64_t)ti * G.gc + tj;
        t.p = p[i];
        t.pitch = ld[i] * es;
        t.matrix = x;
        const int64_t n = blocks_of(t);
        if (n > kOrthoBlocks) return DMM_ELIMIT;
        int rc;
        if ((args.n == ORTHO_TILES || blocks + n > kOrthoBlocks) && (rc = flush())) return rc;
        t.first_block = (int32_t)blocks;
        t.pad = (int32_t)before;
        blocks += n;
        before += n;
        args.tile[args.n++] = t;
      }
  }
  return flush();
}

int allow_ortho_lds() {
  static std::mutex mu;
  static bool done[64] = {};
  int device = 0;
  DMM_HIP(hipGetDevice(&device));
  if (device < 0 || device >= 64) return DMM_EINVAL;
  std::lock_guard<std::mutex> g(mu);
  if (!done[device]) {
    DMM_HIP(ortho_allow_lds());
    done[device] = true;
  }
  return DMM_OK;
}

// ld >= width and a buffer, aligned to its elements, for every tile of `count` matrices
int check_matrices(const Grid &G, int32_t count, const void *const *tiles, const int64_t *ld, int es) {
  for (int32_t x = 0; x < count; ++x) {
    const int64_t first = x * G.tiles_per_rep();
    int rc;
    if ((rc = check_lds(G, ld + first)) || (rc = check_tiles(G, tiles + first, es))) return rc;
    for (int64_t i = first; i < first + G.tiles_per_rep(); ++i)
      if (ld[i] > 0xffffffff) return DMM_ELD;
  }
  return DMM_OK;
}

}  // namespace
}  // namespace dmm

extern "C" {

int dmm_orthogonalize_workspace(const dmm_matrix_desc *X, int32_t count, int64_t *bytes) {
  using namespace dmm;
  if (!X || !bytes || count < 0) return DMM_EINVAL;
  try {
    Grid G;
    OrthoLayout L;
    int rc;
    if ((rc = load_matrix(X, &G))) return rc;
    if (G.c != 1) return DMM_EREPL;
    if ((rc = ortho_layout(G, count, &L))) return rc;
    *bytes = L.total;
    return DMM_OK;
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

int dmm_orthogonalize(const dmm_matrix_desc *X, int32_t count, int x_dtype, const void *const *x_tiles, const int64_t *x_ld, int y_dtype,
                      void *const *y_tiles, const int64_t *y_ld, const float *coefficients, int32_t steps, void *workspace,
                      int64_t workspace_bytes, void *hip_stream) {
  using namespace dmm;
  if (!X || count < 0 || !x_tiles || !x_ld || !y_tiles || !y_ld || steps < 1 || steps > ORTHO_STEPS) return DMM_EINVAL;
  if ((x_dtype != DMM_BF16 && x_dtype != DMM_F32) || (y_dtype != DMM_BF16 && y_dtype != DMM_F32)) return DMM_EINVAL;
  if (!coefficients) {
    if (steps > 5) return DMM_EINVAL;
    coefficients = kOrthoCoefficients;
  }
  if (!ortho_in_range(coefficients, steps)) return DMM_EINVAL;
  TraceRange whole("dmm_orthogonalize");
  try {
    Grid G;
    OrthoLayout L;
    int rc;
    if ((rc = load_matrix(X, &G))) return rc;
    if (G.c != 1) return DMM_EREPL;
    const int x_es = x_dtype == DMM_F32 ? 4 : 2, y_es = y_dtype == DMM_F32 ? 4 : 2;
    if ((rc = check_matrices(G, count, x_tiles, x_ld, x_es)) || (rc = check_matrices(G, count, y_tiles, y_ld, y_es))) return rc;
    if ((rc = ortho_layout(G, count, &L))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (L.small) {
      if ((rc = allow_ortho_lds())) return rc;
      OrthoSmall args;
      std::memset(&args, 0, sizeof args);
      args.rows = (int32_t)G.rows;
      args.cols = (int32_t)G.cols;
      args.steps = steps;
      args.x_f32 = x_dtype == DMM_F32;
      args.y_f32 = y_dtype == DMM_F32;
      std::memcpy(args.coefficients, coefficients, (size_t)steps * 3 * sizeof(float));
      bool even = count >= 2 && count <= 1 << 22;
      for (int32_t i = 2; i < count && even; ++i)
        even = (const char *)x_tiles[i] - (const char *)x_tiles[i - 1] == (const char *)x_tiles[1] - (const char *)x_tiles[0] &&
               (char *)y_tiles[i] - (char *)y_tiles[i - 1] == (char *)y_tiles[1] - (char *)y_tiles[0];
      for (int32_t i = 1; i < count && even; ++i) even = x_ld[i] == x_ld[0] && y_ld[i] == y_ld[0];
      args.even = even;
      for (int32_t first = 0; first < count;) {
        const int n = even ? count : std::min(count - first, ORTHO_MATRICES);
        for (int i = 0; i < (even ? 2 : n); ++i)
          args.matrix[i] = {(const char *)x_tiles[first + i], (char *)y_tiles[first + i], (uint32_t)x_ld[first + i], (uint32_t)y_ld[first + i]};
        ortho_small_launch(args, n, stream);
        DMM_HIP(hipGetLastError());
        first += n;
      }
      return DMM_OK;
    }
    if (L.total == 0) return DMM_OK;
    if (!workspace || ((uintptr_t)workspace & 255)) return DMM_EINVAL;
    if (workspace_bytes < L.total) return DMM_ELIMIT;
    if ((rc = allow_ortho_lds())) return rc;
    char *const ws = (char *)workspace;

    // ---- G / |G| as pairs ------------------------------------------------------------------
    OrthoTiles args;
    std::memset(&args, 0, sizeof args);
    args.f32 = x_dtype == DMM_F32;
    args.rows = (int32_t)G.rows;
    args.cols = (int32_t)G.cols;
    args.row_pitch = (int32_t)(L.flip ? L.sp : L.lp);
    args.col_pitch = (int32_t)(L.flip ? L.lp : L.sp);
    args.stride = L.stride;
    args.ws = ws;
    args.by_rows = L.flip ? L.tall[0] : L.wide[0];
    args.by_cols = L.flip ? L.wide[0] : L.tall[0];
    args.sums = (double *)(ws + L.o_sums);
    const int64_t share = std::max<int64_t>(1, kOrthoSums / L.tiles);
    int64_t sums = 0;
    for (int32_t i = 0; i < G.gr; ++i)
      for (int32_t j = 0; j < G.gc; ++j)
        sums += std::min<int64_t>(share, ((G.rc[(size_t)i + 1] - G.rc[(size_t)i] + 63) / 64) * ((G.cc[(size_t)j + 1] - G.cc[(size_t)j] + 63) / 64));
    args.sums_of_launch = (int32_t)sums;
    rc = over_ortho_tiles(G, count, args, x_es, (char *const *)x_tiles, x_ld, [&](OrthoTile &t) {
      t.across = (int32_t)std::min<int64_t>(share, (int64_t)((t.h + 63) / 64) * ((t.w + 63) / 64));
      return (int64_t)t.across;
    }, [&](int blocks) { ortho_norm_launch(args, blocks, stream); });
    if (rc) return rc;
    // (a matrix' last tiles also clear what fills its rows and columns up; workgroups begin at multiples of 8)
    auto blocks64 = [&](OrthoTile &t) {
      const int w = t.col0 + t.w == args.cols ? args.row_pitch - t.col0 : t.w, h = t.row0 + t.h == args.rows ? args.col_pitch - t.row0 : t.h;
      t.across = (w + (t.col0 & 7) + 63) / 64;
      return (int64_t)t.across * ((h + (t.row0 & 7) + 63) / 64);
    };
    if ((rc = over_ortho_tiles(G, count, args, x_es, (char *const *)x_tiles, x_ld, blocks64, [&](int blocks) { ortho_split_launch(args, blocks, stream); })))
      return rc;

    // ---- the steps -----------------------------------------------------------------------------
    OrthoProduct g;
    std::memset(&g, 0, sizeof g);
    g.ws = ws;
    g.stride = L.stride;
    g.count = count;
    g.parts = (float *)(ws + L.o_parts);
    auto product = [&](const OrthoCut &c, bool symmetric, int64_t m, int64_t n, int64_t kp) -> int {
      g.symmetric = symmetric;
      g.m = (int32_t)m;
      g.n = (int32_t)n;
      g.steps = (int32_t)(kp / 32);
      g.k_pitch_a = g.k_pitch_b = (uint32_t)(kp * 4);
      g.tiles_m = c.tiles_m;
      g.tiles_n = c.tiles_n;
      g.tiles = c.tiles;
      g.runs = c.runs;
      g.per = c.per;
      g.whole = c.whole;
      ortho_product_launch(g, c.edge, stream);
      DMM_HIP(hipGetLastError());
      return DMM_OK;
    };
    const float unit = 1.f / 4096.f;   // a product of two scaled matrices, scaled once
    // a X and b S X + ... nearly cancel in the strong directions: a X is added in the epilogue.  As a I in P it would be added up with
    // the rest in the matrix instructions, which round the sums so far twice for 16 values of K, at the size that they have on the way: a fp32
    // result is 1.3e-5 off then instead of 4.1e-6 (1021 x 4090, a few strong directions; plain fp32 6.2e-6), and of a bf16 one twice as many
    // elements are not the nearest (8192 x 8192: 1.2 % instead of 0.54 %; plain fp32 0.77 %).  Reading X once more takes 1 % there, 3 % at 2048.
    for (int32_t i = 0; i < steps; ++i) {
      const int now = i & 1;
      const float *c = coefficients + 3 * i;
      // S = X X^T
      g.a = g.b = L.wide[now];
      g.old = g.y = -1;
      g.out = g.turned = L.S;
      g.out_pitch = g.turned_pitch = (uint32_t)L.sp;
      g.alpha = 0.f;
      g.beta = unit;
      if ((rc = product(L.cut_s, true, L.s, L.s, L.lp))) return rc;
      // P = b S + c S S
      g.a = g.b = g.old = L.S;
      g.out = g.turned = L.P;
      g.alpha = c[1];
      g.beta = c[2] * unit;
      if ((rc = product(L.cut_p, true, L.s, L.s, L.sp))) return rc;
      // X <- a X + P X
      g.a = L.P;
      g.b = L.tall[now];
      g.old = L.wide[now];
      g.alpha = c[0];
      g.out = L.wide[now ^ 1];
      g.out_pitch = (uint32_t)L.lp;
      g.turned = L.tall[now ^ 1];
      g.turned_pitch = (uint32_t)L.sp;
      g.beta = unit;
      if (i + 1 == steps) {            // the result takes the place of the generation that it is not made from
        g.y = L.wide[now ^ 1];
        g.y_turned = L.flip;
      }
      if ((rc = product(L.cut_x, false, L.s, L.l, L.sp))) return rc;
    }
    args.f32 = y_dtype == DMM_F32;
    args.by_rows = g.y;
    return over_ortho_tiles(G, count, args, y_es, (char *const *)y_tiles, y_ld, [&](OrthoTile &t) {
      t.across = (t.w + 63) / 64;
      return (int64_t)t.across * ((t.h + 63) / 64);
    }, [&](int blocks) { ortho_store_launch(args, blocks, stream); });
  } catch (const std::bad_alloc &) {
    return DMM_ENOMEM;
  }
}

}  // extern "C"
