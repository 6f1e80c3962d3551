"""GPU tests of the layers around a product: 8-bit integers, the gated block, gradients of bf16 products, each against plain
arithmetic in 64 bits.

How far a result may be off, u = 2^-24 (half a step of fp32), h = 2^-8 (half a step of bf16):
  sums of bf16 products    4 K u |a_i| |b_j| (K products that fp32 holds exactly, added in an order and with the internal rounding that the matrix
                           instructions choose)
  scaled integers          3 u of the value: the integer to fp32, two products
  act, its slope           8 u for the function itself, 4 u |argument| for the argument of its exponential and 2 u for the products around it,
                           relative to act, and for the slope (where terms cancel) to 2: no slope is larger in magnitude
"""
import numpy as np
import pytest

from tests.layer_tiles import ACTS, Int8, Tiles, act, descs, normal, stream, uneven
import workloads

torch = pytest.importorskip("torch")
binding = pytest.importorskip("paper_2510_08874_amd.binding")
pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
LAYOUTS = ("whole", "blocks", "column", "uneven", "row_col")
TINY = 2.0 ** -126                                             # (results below the normal range of fp32 and bf16)


def sum_error(a, b):
    """Of a @ b, elements of a and b as given."""
    return 4 * a.shape[1] * U * torch.linalg.vector_norm(a, dim=1, keepdim=True) * torch.linalg.vector_norm(b, dim=0, keepdim=True)


def argument(g, name):
    """That of the exponential."""
    return g.abs() if name == "silu" else g * g / 2 if name == "gelu" else 1.6 * (g + 0.044715 * g ** 3).abs()


def close(got, want, limit, what):
    assert bool(torch.isfinite(want).all())
    off = (got - want).abs()
    bad = ~(off <= limit)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()}, limit {limit[bad][0].item()}"


# ---- integers -------------------------------------------------------------------------------------------

def quantized(X, axis):
    """Codes and scales by definition, in 64 bits."""
    X = X.double()
    top = X.abs().amax(axis, keepdim=True)
    q = torch.round(X * 127 / torch.where(top > 0, top, 1.0))  # (127 x fits 53 bits, and so does every half-way value of the quotient)
    return q, (top / 127).float().squeeze(axis)


GRIDS = [(1, 1, None), (1, 7, None), (3, 130, None), (5, 1000, (2, 3)), (129, 257, (3, 4)), (64, 16384, None), (33, 20001, (1, 2)), (257, 96, (4, 1)), (700, 513, (2, 40)),
         (200, 4100, (3, 3)), (1500, 700, (1, 5)), (1030, 41001, (1, 3)), (40, 70001, None), (200, 300, (30, 2)), (90, 500, (5, 31))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("along", ["rows", "cols"])
@pytest.mark.parametrize("rows,cols,grid", GRIDS, ids=str)
def test_integers_and_values(rows, cols, grid, along, dtype):
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    d = workloads.desc(rows, cols, [0, rows], [0, cols], 1, 1) if grid is None else workloads.desc(rows, cols, uneven(rows, grid[0]), uneven(cols, grid[1]), 1, 1)
    X = normal(rows, cols, rows + cols, dtype=torch.float32)
    X *= torch.exp2(torch.linspace(-100, 100, rows if along == "rows" else cols, device="cuda").round()).reshape((-1, 1) if along == "rows" else (1, -1))
    if rows > 2 and cols > 2:                                  # half-way values, a row and a column of zeros, the smallest numbers
        X[1, :] = X[1, :].sign() * torch.arange(cols, device="cuda").remainder(255).add(1).float() * 0.5
        X[:, 2] = 0
        X[2, :] = 0
        X[0, 0] = 2.0 ** -133
    X = X.to(t)
    axis = 1 if along == "rows" else 0
    want, scales = quantized(X, axis)
    for more, offset in ((0, 0), (5, 3)):
        x = Tiles(d, t, X, more, offset)
        form = Int8(d, along, more=more, offset=offset)
        values = Tiles(d, t, None, more, offset)
        binding.dmm_int_quantize(binding.matrix_desc(d), ACT_TYPES[dtype], x.table(), **{along: form.table()}, stream=stream())
        binding.dmm_int_dequantize(binding.matrix_desc(d), form.table(), binding.DMM_MX_ROWS if along == "rows" else binding.DMM_MX_COLS, ACT_TYPES[dtype],
                                  values.table(), stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(form.q.whole(), want)
        assert torch.equal(form.scales(), scales)
        v = (want.float() * (scales.unsqueeze(1) if along == "rows" else scales)).to(t)
        assert torch.equal(values.whole(), v.double())
        form.q.check_guards()
        values.check_guards()


ACT_TYPES = {"bf16": binding.DMM_BF16, "f32": binding.DMM_F32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_rows_without_a_scale_stand_for_nan(bad, dtype):
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows, cols = 40, 300
    X = normal(rows, cols, 3, dtype=t)
    X[7, 250] = bad
    for along, grid in (("rows", [0, cols]), ("rows", sorted({i * cols // 40 for i in range(41)})), ("cols", [0, 100, cols])):
        d = workloads.desc(rows, cols, [0, 11, rows], grid, 1, 1)
        form, values = Int8(d, along), Tiles(d, t)
        binding.dmm_int_quantize(binding.matrix_desc(d), ACT_TYPES[dtype], Tiles(d, t, X).table(), **{along: form.table()}, stream=stream())
        binding.dmm_int_dequantize(binding.matrix_desc(d), form.table(), binding.DMM_MX_ROWS if along == "rows" else binding.DMM_MX_COLS, ACT_TYPES[dtype],
                                  values.table(), stream=stream())
        nan = torch.isnan(values.whole())
        want = torch.zeros_like(nan)
        if along == "rows":
            want[7] = True
        else:
            want[:, 250] = True
        assert torch.equal(nan, want)
        assert bool((form.q.whole()[want] == 0).all()) and int(torch.isnan(form.scales()).sum()) == 1


def integers(rows, cols, seed):
    return torch.from_numpy(np.random.default_rng(seed).integers(-127, 128, (rows, cols), dtype=np.int8)).to("cuda")


def scales_of(n, seed, spread=8):
    return torch.from_numpy(np.exp2(np.random.default_rng(seed).uniform(-spread, spread, n)).astype(np.float32)).to("cuda")


SIZES = [(1, 1, 1), (1, 127, 3), (2, 128, 130), (17, 129, 128), (33, 300, 257), (64, 1000, 64), (100, 640, 129), (130, 257, 131), (257, 1025, 300), (5, 9000, 70), (300, 5000, 500), (40, 3001, 6001), (9, 2000, 12001)]


@pytest.mark.parametrize("layout,c_dtype", [(x, t) for x in LAYOUTS for t in ("f32", "bf16")] + [("replicated", "f32")])
@pytest.mark.parametrize("m,k,n", SIZES, ids=str)
def test_products_of_integers(m, k, n, layout, c_dtype):
    (da, db, dc), ranks = descs(layout, m, k, n)
    qa, qb, sa, sb = integers(m, k, m + n), integers(k, n, k), scales_of(m, 1), scales_of(n, 2)
    t = torch.float32 if c_dtype == "f32" else torch.bfloat16
    plan = binding.Plan(da, db, dc, ranks)
    for more, offset in ((0, 0), (7, 1)):
        a, b = Int8(da, "rows", qa, sa, more, offset), Int8(db, "cols", qb, sb, more, offset)
        c = Tiles(dc, t, None, more, offset)
        plan.execute_int(a.table(), b.table(), c.table(), binding.DMM_C_BF16 if c_dtype == "bf16" else 0, stream())
        torch.cuda.synchronize()
        scale = sa.double().unsqueeze(1) * sb.double()
        want = (qa.double() @ qb.double()) * scale
        if layout == "replicated":
            half = k // 2
            parts = [(qa[:, :half].double() @ qb[:half].double()) * scale, (qa[:, half:].double() @ qb[half:].double()) * scale]
            close(c.whole(1), parts[1], 3.01 * U * parts[1].abs(), "second replica")
            close(c.whole(0), want, 4.01 * U * (parts[0].abs() + parts[1].abs()), "sum")
        else:
            close(c.whole(), want, (3.01 * U + (H if c_dtype == "bf16" else 0)) * want.abs(), "product")
        c.check_guards()


def test_sums_of_any_length():
    """More products than an int32 sum holds, all of one sign and all codes at the end of their range."""
    m, n, k = 3, 5, 400003
    (da, db, dc), ranks = descs("whole", m, k, n)
    qa, qb = torch.full((m, k), -128, dtype=torch.int8, device="cuda"), torch.full((k, n), -128, dtype=torch.int8, device="cuda")
    qb[:, 1] = 127
    qb[:, 2] = integers(k, 1, 3)[:, 0]
    one = torch.ones(max(m, n), device="cuda")
    c = Tiles(dc, torch.float32)
    binding.Plan(da, db, dc, ranks).execute_int(Int8(da, "rows", qa, one[:m]).table(), Int8(db, "cols", qb, one[:n]).table(), c.table(), 0, stream())
    want = qa.double() @ qb.double()
    close(c.whole(), want, 3.01 * U * want.abs(), "long sums")


def test_scales_far_apart():
    """No product on the way leaves the range of fp32 where the result does not."""
    m, k, n = 40, 200, 33
    (da, db, dc), ranks = descs("whole", m, k, n)
    qa, qb = integers(m, k, 1), integers(k, n, 2)
    sa = torch.full((m,), 2.0 ** 120, device="cuda")
    sb = torch.full((n,), 2.0 ** -140, device="cuda")
    sa[3], sb[4] = 0, 0
    c = Tiles(dc, torch.float32)
    binding.Plan(da, db, dc, ranks).execute_int(Int8(da, "rows", qa, sa).table(), Int8(db, "cols", qb, sb).table(), c.table(), 0, stream())
    want = (qa.double() @ qb.double()) * (sa.double().unsqueeze(1) * sb.double())
    close(c.whole(), want, 3.01 * U * want.abs(), "scales")


# ---- the gated block ------------------------------------------------------------------------------------

GATED_SIZES = [(1, 1, 1), (1, 64, 3), (2, 65, 129), (17, 129, 128), (33, 200, 257), (64, 500, 64), (100, 320, 129), (130, 257, 131), (257, 513, 300), (5, 4500, 70), (300, 2500, 500), (40, 3001, 6001), (9, 2000, 12001)]


def gated_error(g, u, eg, eu, name):
    """H = act(G) U from sums that are off by eg and eu: no slope is larger than 1.13."""
    a, _ = act(g, name)
    return 1.13 * eg * (u.abs() + eu) + a.abs() * eu + (a * u).abs() * (10 + 4 * argument(g, name)) * U


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("m,k,n", GATED_SIZES, ids=str)
def test_gated_block(m, k, n, layout, name):
    (da, db, dc), ranks = descs(layout, m, k, n)
    A, Wg, Wu = normal(m, k, m), normal(k, n, n, 2 * k ** -0.5), normal(k, n, n + 1, k ** -0.5)
    plan = binding.Plan(da, db, dc, ranks)
    g, u = A.double() @ Wg.double(), A.double() @ Wu.double()
    eg, eu = sum_error(A.double(), Wg.double()), sum_error(A.double(), Wu.double())
    want = act(g, name)[0] * u
    for more, offset, keep in ((0, 0, True), (3, 1, False)):
        a, wg, wu = Tiles(da, torch.bfloat16, A, more, offset), Tiles(db, torch.bfloat16, Wg, more, offset), Tiles(db, torch.bfloat16, Wu, more + 8, offset)
        h, kg, ku = (Tiles(dc, torch.bfloat16, None, more + x, offset) for x in range(3))
        plan.gated(ACTS[name], a.table(), wg.table(), wu.table(), h.table(), kg.table() if keep else None, ku.table() if keep else None, stream())
        torch.cuda.synchronize()
        close(h.whole(), want, H * want.abs() + (1 + H) * gated_error(g, u, eg, eu, name) + TINY, "H")
        if keep:
            close(kg.whole(), g, H * g.abs() + (1 + H) * eg, "G")
            close(ku.whole(), u, H * u.abs() + (1 + H) * eu, "U")
        for t in (h, kg, ku):
            t.check_guards()


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("m,k,n", SIZES, ids=str)
def test_gated_block_of_integers(m, k, n, layout, name):
    (da, db, dc), ranks = descs(layout, m, k, n)
    qa, qg, qu = integers(m, k, m), integers(k, n, n), integers(k, n, n + 1)
    sa, sg, su = scales_of(m, 1, 1) * (k ** -0.5 / 40), scales_of(n, 2, 1) / 40, scales_of(n, 3, 1) / 40
    g, u = ((qa.double() @ q.double()) * (sa.double().unsqueeze(1) * s.double()) for q, s in ((qg, sg), (qu, su)))
    want = act(g, name)[0] * u
    plan = binding.Plan(da, db, dc, ranks)
    for more, offset in ((0, 0), (7, 1)):
        a, wg, wu = Int8(da, "rows", qa, sa, more, offset), Int8(db, "cols", qg, sg, more, offset), Int8(db, "cols", qu, su, more + 2, offset)
        h = Tiles(dc, torch.bfloat16, None, more, offset)
        plan.gated_int(ACTS[name], a.table(), wg.table(), wu.table(), h.table(), stream())
        torch.cuda.synchronize()
        close(h.whole(), want, H * want.abs() + (1 + H) * gated_error(g, u, 3.01 * U * g.abs(), 3.01 * U * u.abs(), name) + TINY, "H")
        h.check_guards()


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("db_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("m,k,n", GATED_SIZES, ids=str)
def test_gated_backward(m, k, n, layout, db_dtype, name):
    (da, db, dc), ranks = descs(layout, m, k, n)
    A, Wg, Wu = normal(m, k, m), normal(k, n, n, k ** -0.5), normal(k, n, n + 1, k ** -0.5)
    G, V, D = normal(m, n, 5, 2.0), normal(m, n, 6), normal(m, n, 7, 1e-3)
    t = torch.float32 if db_dtype == "f32" else torch.bfloat16
    out = 0 if db_dtype == "f32" else H
    plan = binding.Plan(da, db, dc, ranks)
    for more, offset in ((0, 0), (3, 1)):
        a, wg, wu = Tiles(da, torch.bfloat16, A, more, offset), Tiles(db, torch.bfloat16, Wg, more, offset), Tiles(db, torch.bfloat16, Wu, more, offset)
        g, u, dh = (Tiles(dc, torch.bfloat16, x, more, offset) for x in (G, V, D))
        dg, du = (Tiles(dc, torch.bfloat16, None, more + x, offset) for x in (1, 2))
        ga, gg, gu = Tiles(da, torch.bfloat16, None, more, offset, 1), Tiles(db, t, None, more, offset, 1), Tiles(db, t, None, more, offset, 1)
        plan.gated_backward(ACTS[name], *(x.table() for x in (a, wg, wu, g, u, dh, dg, du, ga, gg, gu)), binding.DMM_DB_F32 if db_dtype == "f32" else 0, stream())
        torch.cuda.synchronize()
        value, slope = act(G.double(), name)
        arg = argument(G.double(), name)
        want = D.double() * value
        close(du.whole(), want, H * want.abs() + (1 + H) * want.abs() * (10 + 4 * arg) * U + TINY, "dU")
        want = D.double() * V.double() * slope
        close(dg.whole(), want, H * want.abs() + (1 + H) * (D.double() * V.double()).abs() * 2 * (10 + 4 * arg) * U + TINY, "dG")
        # the products are of what is stored
        x, w = torch.cat((dg.whole(), du.whole()), 1), torch.cat((Wg, Wu), 1).double().t()
        want = x @ w
        close(ga.whole(), want, H * want.abs() + (1 + H) * sum_error(x, w) + TINY, "dA")
        for got, y in ((gg, dg), (gu, du)):
            want = A.double().t() @ y.whole()
            close(got.whole(), want, out * want.abs() + (1 + out) * sum_error(A.double().t(), y.whole()) + TINY, "a weight's gradient")
        for y in (dg, du, ga, gg, gu):
            y.check_guards()


@pytest.mark.parametrize("db_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [*LAYOUTS, "replicated"])
@pytest.mark.parametrize("m,k,n", GATED_SIZES, ids=str)
def test_gradients_of_a_product(m, k, n, layout, db_dtype):
    (da, db, dc), ranks = descs(layout, m, k, n)
    A, B, D = normal(m, k, m), normal(k, n, n, k ** -0.5), normal(m, n, 7, 1e-3)
    t = torch.float32 if db_dtype == "f32" else torch.bfloat16
    out = 0 if db_dtype == "f32" else H
    flags = binding.DMM_DB_F32 if db_dtype == "f32" else 0
    plan = binding.Plan(da, db, dc, ranks)
    for more, offset in ((0, 0), (3, 1)):
        a, b, c = (Tiles(d, torch.bfloat16, x, more, offset, 1) for d, x in ((da, A), (db, B), (dc, D)))
        ga, gb = Tiles(da, torch.bfloat16, None, more, offset, 1), Tiles(db, t, None, more, offset, 1)
        plan.execute_backward(a.table(), b.table(), c.table(), ga.table(), gb.table(), flags, stream())
        torch.cuda.synchronize()
        want = D.double() @ B.double().t()
        close(ga.whole(), want, H * want.abs() + (1 + H) * sum_error(D.double(), B.double().t()) + TINY, "dA")
        want = A.double().t() @ D.double()
        close(gb.whole(), want, out * want.abs() + (1 + out) * sum_error(A.double().t(), D.double()) + TINY, "dB")
        ga.check_guards()
        gb.check_guards()
    # each by itself
    ga2, gb2 = Tiles(da, torch.bfloat16, None, 3, 1, 1), Tiles(db, t, None, 3, 1, 1)
    plan.execute_backward(None, b.table(), c.table(), ga2.table(), None, flags, stream())
    plan.execute_backward(a.table(), None, c.table(), None, gb2.table(), flags, stream())
    torch.cuda.synchronize()
    assert torch.equal(ga2.whole(), ga.whole()) and torch.equal(gb2.whole(), gb.whole())
