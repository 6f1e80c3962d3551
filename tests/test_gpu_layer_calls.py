"""GPU tests of calls around each other for the layers around a product: captures, streams, threads, tiles in each other's place, operands that lie far
apart, and whole layers made of these calls.  Limits as in test_gpu_layer.py."""
import threading

import numpy as np
import pytest

import workloads
from tests.layer_tiles import ACTS, Int8, Tiles, act, descs, normal, stream
from tests.test_gpu_layer import H, TINY, U, close, gated_error, integers, quantized, scales_of, sum_error

torch = pytest.importorskip("torch")
binding = pytest.importorskip("paper_2510_08874_amd.binding")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# whole tiles; cut along K; on copies; on copies of few rows alone, results on their way through scratch memory
SIZES = [("blocks", 512, 512, 768), ("whole", 40, 8192, 300), ("uneven", 1301, 1103, 907), ("row_col", 9, 2000, 12001)]


class Calls:
    """Every product around a layer on the same sizes: what is called, and the tiles that it writes."""

    def __init__(self, layout, m, k, n, seed=0):
        self.descs, ranks = descs(layout, m, k, n)
        da, db, dc = self.descs
        self.plan = binding.Plan(da, db, dc, ranks)
        qa, qg, qu = integers(m, k, seed + 1), integers(k, n, seed + 2), integers(k, n, seed + 3)
        sa, sg, su = scales_of(m, 1, 1) * (k ** -0.5 / 40), scales_of(n, 2, 1) / 40, scales_of(n, 3, 1) / 40
        self.ints = Int8(da, "rows", qa, sa), Int8(db, "cols", qg, sg), Int8(db, "cols", qu, su)
        self.bf = [Tiles(d, BF16, normal(d["rows"], d["cols"], seed + 4 + i, s)) for i, (d, s) in enumerate(((da, 1), (db, k ** -0.5), (db, k ** -0.5)))]
        self.dc = [Tiles(dc, BF16, normal(m, n, seed + 7 + i)) for i in range(3)]
        self.out = {"int": [Tiles(dc, torch.float32)], "int_gated": [Tiles(dc, BF16)], "gated": [Tiles(dc, BF16) for _ in range(3)],
                    "backward": [Tiles(dc, BF16), Tiles(dc, BF16), Tiles(da, BF16, replicas=1), Tiles(db, BF16, replicas=1), Tiles(db, torch.bfloat16, replicas=1)],
                    "gradients": [Tiles(da, BF16, replicas=1), Tiles(db, torch.float32, replicas=1)]}
        a, g, u = (x.table() for x in self.bf)
        ints, dcs = [x.table() for x in self.ints], [x.table() for x in self.dc]
        o = {name: [t.table() for t in ts] for name, ts in self.out.items()}
        p = self.plan
        single = [Tiles(d, BF16, normal(d["rows"], d["cols"], seed + 4 + i), replicas=1) for i, d in enumerate((da, db))]
        sa, sb = (x.table() for x in single)
        self.run = {"int": lambda s: p.execute_int(*ints[:2], o["int"][0], 0, s), "int_gated": lambda s: p.gated_int(binding.DMM_SILU, *ints, o["int_gated"][0], s),
                    "gated": lambda s: p.gated(binding.DMM_GELU, a, g, u, *o["gated"], stream=s),
                    "backward": lambda s: p.gated_backward(binding.DMM_GELU, a, g, u, *dcs, *o["backward"], stream=s),
                    "gradients": lambda s: p.execute_backward(sa, sb, dcs[0], *o["gradients"], flags=binding.DMM_DB_F32, stream=s)}

    def values(self, name):
        torch.cuda.synchronize()
        return [v.clone() for t in self.out[name] for v in t.views if v is not None]

    def clear(self, name):
        for t in self.out[name]:
            for v in t.views:
                if v is not None:
                    v.fill_(float("nan"))
        torch.cuda.synchronize()


NAMES = ("int", "int_gated", "gated", "backward", "gradients")


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("mode", ["global", "relaxed"])
@pytest.mark.parametrize("layout,m,k,n", SIZES, ids=str)
def test_captures(layout, m, k, n, mode):
    """All calls of a plan in one graph, on another stream than the calls before: every replay gives what they gave, with eager calls on
    the same tables and with other plans' between."""
    c, other = Calls(layout, m, k, n), Calls(layout, m, k, n, 50)
    first, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    want = {}
    for name in NAMES:
        c.run[name](first.cuda_stream)
        other.run[name](first.cuda_stream)
        want[name] = c.values(name)
        assert not any(bool(torch.isnan(v).any()) for v in want[name])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode=mode):
        for name in NAMES:
            c.run[name](side.cuda_stream)
    for turn in range(3):
        for name in NAMES:
            c.clear(name)
        with torch.cuda.stream(side):
            graph.replay()
        for name in NAMES:
            assert same(c.values(name), want[name]), (turn, name)
            other.run[name](side.cuda_stream)
            c.clear(name)
            c.run[name](side.cuda_stream)
            assert same(c.values(name), want[name]), (turn, name)
    del graph


def test_two_graphs_of_a_plan():
    """Replayed in turn on one stream: they share the plan's tables and scratch memory."""
    c = Calls("whole", 40, 8192, 300)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for name in NAMES:
        c.run[name](side.cuda_stream)
    want = {name: c.values(name) for name in NAMES}
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g, names in zip(graphs, (NAMES[:3], NAMES[2:])):
        with torch.cuda.graph(g, stream=side, capture_error_mode="relaxed"):
            for name in names:
                c.run[name](side.cuda_stream)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for name in NAMES:
            c.clear(name)
        with torch.cuda.stream(side):
            for x in order:
                graphs[x].replay()
        assert all(same(c.values(name), want[name]) for name in NAMES), order
    del graphs


@pytest.mark.parametrize("layout,m,k,n", SIZES, ids=str)
def test_integers_are_captured_without_a_call_before(layout, m, k, n):
    (da, _, _), _ = descs(layout, m, k, n)
    x = Tiles(da, BF16, normal(m, k, 3))
    forms = Int8(da, "rows"), Int8(da, "cols")
    values = Tiles(da, BF16)
    tables, d = [f.table() for f in forms], binding.matrix_desc(da)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.dmm_int_quantize(d, binding.DMM_BF16, x.table(), *tables, stream=side.cuda_stream)
        binding.dmm_int_dequantize(d, tables[1], binding.DMM_MX_COLS, binding.DMM_BF16, values.table(), stream=side.cuda_stream)
    for seed in (4, 5, 6):
        X = normal(m, k, seed)
        for (r0, r1, c0, c1), v in zip(x.bounds, x.views):
            if v is not None:
                v.copy_(X[r0:r1, c0:c1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for f, axis in zip(forms, (1, 0)):
            q, s = quantized(X, axis)
            assert torch.equal(f.q.whole(), q) and torch.equal(f.scales(), s)
        assert torch.equal(values.whole(), (q.float() * s).to(BF16).double())
    del graph


def test_a_first_call_is_not_captured():
    """Refused, and the capture goes on; so are other operands than those of the call before."""
    c = Calls("blocks", 64, 128, 64)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="relaxed"):
        for name in NAMES:
            with pytest.raises(binding.DmmError) as e:
                c.run[name](side.cuda_stream)
            assert e.value.kind == "EINVAL"
        x += 1
    graph.replay()
    torch.cuda.synchronize()
    assert float(x.sum()) == 4
    del graph


@pytest.mark.parametrize("layout,m,k,n", SIZES, ids=str)
def test_streams_and_changing_operands(layout, m, k, n):
    """A plan's calls in turn on two streams, on two sets of tiles: partial sums, copies and tables of one call are not overwritten under another."""
    c = Calls(layout, m, k, n)
    second = [Tiles(c.descs[2], BF16), Int8(c.descs[0], "rows", integers(m, k, 77), scales_of(m, 5, 1) / 500)]
    tables = c.ints[1].table(), c.ints[2].table(), second[0].table(), second[1].table()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for name in NAMES:
        c.run[name](stream())
    want = {name: c.values(name) for name in NAMES}
    c.plan.gated_int(binding.DMM_GELU, tables[3], tables[0], tables[1], tables[2], stream())
    torch.cuda.synchronize()
    want2 = second[0].whole()
    for name in NAMES:
        c.clear(name)
    for turn in range(6):
        s = streams[turn % 2].cuda_stream
        for name in NAMES:
            c.run[name](s)
        c.plan.gated_int(binding.DMM_GELU, tables[3], tables[0], tables[1], tables[2], streams[(turn + 1) % 2].cuda_stream)
    torch.cuda.synchronize()
    assert all(same(c.values(name), want[name]) for name in NAMES)
    assert torch.equal(second[0].whole(), want2)


def test_threads_with_plans_of_their_own():
    calls = [Calls(*SIZES[x % 3], seed=20 * x) for x in range(4)]
    want = []
    for c in calls:
        for name in NAMES:
            c.run[name](stream())
        want.append({name: c.values(name) for name in NAMES})
        for name in NAMES:
            c.clear(name)
    wrong = []

    def work(c, want):
        s = torch.cuda.Stream()
        try:
            for _ in range(20):
                for name in NAMES:
                    c.run[name](s.cuda_stream)
            s.synchronize()
        except Exception as e:                                # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(calls, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    for c, w in zip(calls, want):
        assert all(same(c.values(name), w[name]) for name in NAMES)


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("layout,m,k,n", [*SIZES, ("uneven", 61, 50, 77)], ids=str)
def test_gradients_in_place_of_what_was_kept(layout, m, k, n, name):
    """dG and dU into the tiles of G and U: what separate tiles get, bit for bit, rows of any length."""
    c = Calls(layout, m, k, n)
    a, g, u = (x.table() for x in c.bf)
    out, kept = c.out["backward"], c.dc
    c.plan.gated_backward(ACTS[name], a, g, u, *(t.table() for t in kept), *(t.table() for t in out), stream=stream())
    want = c.values("backward")
    c.clear("backward")
    G, V, D = (t.table() for t in kept)
    c.plan.gated_backward(ACTS[name], a, g, u, G, V, D, G, V, *(t.table() for t in out[2:]), stream=stream())
    torch.cuda.synchronize()
    got = [v for t in (kept[0], kept[1], *out[2:]) for v in t.views if v is not None]
    assert same(got, want)


@pytest.mark.parametrize("m,k,n", [(0, 5, 7), (5, 0, 7), (5, 7, 0), (0, 0, 0)], ids=str)
def test_empty_sides(m, k, n):
    """No rows, no columns: nothing is written; no inner side: zeros."""
    (da, db, dc), ranks = descs("whole", m, k, n)
    plan = binding.Plan(da, db, dc, ranks)
    one = torch.ones(8, device="cuda")
    ints = Int8(da, "rows", torch.zeros(m, k, dtype=torch.int8, device="cuda"), one[:m]), Int8(db, "cols", torch.zeros(k, n, dtype=torch.int8, device="cuda"), one[:n])
    a, w, c, h = Tiles(da, BF16, torch.ones(m, k)), Tiles(db, BF16, torch.ones(k, n)), Tiles(dc, torch.float32), [Tiles(dc, BF16) for _ in range(5)]
    plan.execute_int(ints[0].table(), ints[1].table(), c.table(), 0, stream())
    plan.gated_int(binding.DMM_SILU, ints[0].table(), ints[1].table(), ints[1].table(), h[0].table(), stream())
    plan.gated(binding.DMM_SILU, a.table(), w.table(), w.table(), *(x.table() for x in h[1:4]), stream=stream())
    torch.cuda.synchronize()
    for t in (c, *h[:4]):
        assert bool((t.whole() == 0).all())
    ga, gw = Tiles(da, BF16), Tiles(db, torch.float32)
    d = Tiles(dc, BF16, torch.ones(m, n))
    plan.execute_backward(a.table(), w.table(), d.table(), ga.table(), gw.table(), binding.DMM_DB_F32, stream())
    torch.cuda.synchronize()
    assert bool((ga.whole() == n).all()) and bool((gw.whole() == m).all())


@pytest.mark.parametrize("layout,m,k,n", [("whole", 70, 200, 90), ("uneven", 300, 257, 260), ("uneven", 1301, 1103, 907), ("row_col", 9, 2000, 12001)], ids=str)
def test_infinities_and_nan_stay_in_their_rows_and_columns(layout, m, k, n):
    """Of the operands, whatever is filled up with zeros next to them."""
    (da, db, dc), ranks = descs(layout, m, k, n)
    plan = binding.Plan(da, db, dc, ranks)
    A, W, V, D = normal(m, k, 1), normal(k, n, 2), normal(k, n, 3), normal(m, n, 4)
    A[3, k - 1] = float("nan")
    A[5, 0] = float("inf")
    W[k - 1, n - 1] = float("nan")
    V[0, 7] = float("inf")
    D[m - 1, n - 2] = float("nan")
    h = Tiles(dc, BF16)
    plan.gated(binding.DMM_GELU, Tiles(da, BF16, A).table(), Tiles(db, BF16, W).table(), Tiles(db, BF16, V).table(), h.table(), stream=stream())
    ga, gw = Tiles(da, BF16, replicas=1), Tiles(db, torch.float32, replicas=1)
    plan.execute_backward(*(Tiles(d, BF16, x, replicas=1).table() for d, x in ((da, A), (db, W), (dc, D))), ga.table(), gw.table(), binding.DMM_DB_F32, stream())
    torch.cuda.synchronize()
    g, u = A.double() @ W.double(), A.double() @ V.double()
    touched = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    touched[[3, 5]] = True
    touched[:, [7, n - 1]] = True
    assert bool(torch.isfinite(h.whole()[~touched]).all()) and bool(torch.isnan(h.whole()[3]).all()) and bool(torch.isnan(h.whole()[:, n - 1]).all())
    assert torch.equal(torch.isfinite(ga.whole()), torch.isfinite(D.double() @ W.double().t()))
    assert torch.equal(torch.isfinite(gw.whole()), torch.isfinite(A.double().t() @ D.double()))
    # integers: a row or column whose scale is NaN
    qa, qb, sa, sb = integers(m, k, 5), integers(k, n, 6), scales_of(m, 7), scales_of(n, 8)
    sa[2], sb[n - 1] = float("nan"), float("nan")
    c = Tiles(dc, torch.float32)
    plan.execute_int(Int8(da, "rows", qa, sa).table(), Int8(db, "cols", qb, sb).table(), c.table(), 0, stream())
    torch.cuda.synchronize()
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[2] = True
    want[:, n - 1] = True
    assert torch.equal(torch.isnan(c.whole()), want)


def test_operands_past_32_bit_offsets():
    """More than 2^32 bytes of integers in one tile, more than 2^32 elements past a corner."""
    m, k, n = 70001, 65500, 17
    (da, db, dc), ranks = descs("whole", m, k, n)
    plan = binding.Plan(da, db, dc, ranks)
    qa = torch.empty(m, k, dtype=torch.int8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    for r in range(0, m, 10000):
        qa[r:r + 10000] = torch.randint(-127, 128, qa[r:r + 10000].shape, generator=gen, device="cuda").to(torch.int8)
    qb = integers(k, n, 4)
    one = torch.ones(m, device="cuda")
    c = Tiles(dc, torch.float32)
    plan.execute_int(binding.int_tiles([qa], [k], [one]), Int8(db, "cols", qb, one[:n]).table(), c.table(), 0, stream())
    torch.cuda.synchronize()
    rows = [0, 1, 255, 256, 32768, 65535, 65536, 65600, m - 257, m - 1]
    want = qa[rows].double() @ qb.double()
    close(c.whole()[rows], want, 3.01 * U * want.abs(), "product")
    # and through the quantisation of as many bf16 values, back and forth
    d = binding.matrix_desc(da)
    x = qa.to(BF16)                                           # (every row has 127 or -127: the integers come back)
    out, s = torch.empty_like(qa), torch.empty(m, device="cuda")
    form = binding.int_tiles([out], [k], [s])
    binding.dmm_int_quantize(d, binding.DMM_BF16, binding.tiles([x], [k]), rows=form, stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(out[rows], qa[rows]) and bool((s == 1).all())
    x.zero_()
    binding.dmm_int_dequantize(d, form, binding.DMM_MX_ROWS, binding.DMM_BF16, binding.tiles([x], [k]), stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(x[rows], qa[rows].to(BF16))


def test_replicas_are_quantised_from_their_own_tiles():
    d = workloads.block_desc(100, 300, 2, 2, replication=3)
    x = Tiles(d, BF16)
    want = []
    for rep in range(3):
        X = normal(100, 300, rep)
        want.append(X)
        for (r0, r1, c0, c1), v in list(zip(x.bounds, x.views))[4 * rep:4 * rep + 4]:
            v.copy_(X[r0:r1, c0:c1])
    rows, cols = Int8(d, "rows"), Int8(d, "cols")
    binding.dmm_int_quantize(binding.matrix_desc(d), binding.DMM_BF16, x.table(), rows=rows.table(), cols=cols.table(), stream=stream())
    torch.cuda.synchronize()
    for rep in range(3):
        for form, axis in ((rows, 1), (cols, 0)):
            q, s = quantized(want[rep], axis)
            assert torch.equal(form.q.whole(rep), q) and torch.equal(form.scales(rep), s)


# ---- layers -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("m,k,n", [(96, 128, 192), (131, 77, 203), (1, 64, 96)], ids=str)
def test_a_training_step_of_the_feed_forward_layer(m, k, n, name):
    """Gated block, down projection, their backward calls, as a trainer makes them, against the layer's gradients by differences in 64 bits:
    d loss / d t along a direction of each operand, for loss = sum of Y times a fixed R."""
    block = workloads.block_desc
    dx, dw, dh, dd, dy = block(m, k, 2, 2), block(k, n, 2, 2), block(m, n, 2, 2), block(n, k, 2, 2), block(m, k, 2, 2)
    up, down = binding.Plan(dx, dw, dh, 4), binding.Plan(dh, dd, dy, 4)
    X, Wg, Wu, Wd, R = normal(m, k, 1), normal(k, n, 2, k ** -0.5), normal(k, n, 3, k ** -0.5), normal(n, k, 4, n ** -0.5), normal(m, k, 5)
    x, wg, wu, wd, r = (Tiles(d, BF16, v) for d, v in ((dx, X), (dw, Wg), (dw, Wu), (dd, Wd), (dy, R)))
    h, g, u, dhh = (Tiles(dh, BF16) for _ in range(4))
    y, gx = Tiles(dy, BF16), Tiles(dx, BF16)
    gwd, gwg, gwu = Tiles(dd, torch.float32), Tiles(dw, torch.float32), Tiles(dw, torch.float32)
    s = stream()
    up.gated(ACTS[name], *(t.table() for t in (x, wg, wu, h, g, u)), stream=s)
    down.execute(binding.DMM_BF16, h.views, h.ld, wd.views, wd.ld, y.views, y.ld, binding.DMM_C_BF16, s)
    down.execute_backward(h.table(), wd.table(), r.table(), dhh.table(), gwd.table(), binding.DMM_DB_F32, s)
    gt, ut = g.table(), u.table()
    up.gated_backward(ACTS[name], x.table(), wg.table(), wu.table(), gt, ut, dhh.table(), gt, ut, gx.table(), gwg.table(), gwu.table(), binding.DMM_DB_F32, s)
    torch.cuda.synchronize()

    def layer(X, Wg, Wu, Wd):
        return ((act(X @ Wg, name)[0] * (X @ Wu)) @ Wd * R.double()).sum()

    at = [t.double() for t in (X, Wg, Wu, Wd)]
    want = (act(at[0] @ at[1], name)[0] * (at[0] @ at[2])) @ at[3]
    # H, G, U, dH, dG, dU are rounded to bf16 on the way: h of each, independent of each other
    assert float(torch.linalg.vector_norm(y.whole() - want) / torch.linalg.vector_norm(want)) <= 2 * H
    for i, grad in ((0, gx), (1, gwg), (2, gwu), (3, gwd)):
        size = torch.linalg.vector_norm(grad.whole())
        v = grad.whole() / size                               # the direction in which the loss grows: its derivative there is the gradient's norm
        e = 1e-4
        plus, minus = list(at), list(at)
        plus[i], minus[i] = at[i] + e * v, at[i] - e * v
        slope = (layer(*plus) - layer(*minus)) / (2 * e)
        # at most six roundings of h between the operands and a gradient, and the direction's own error
        assert abs(float(slope / size) - 1) <= 8 * H, (i, float(slope), float(size))


@pytest.mark.parametrize("m", [1, 3, 40, 200])
def test_a_serving_step_in_8_bits(m):
    """Tokens quantised, gated block from integers, its result quantised, down projection: step by step what the formulas give on what went in."""
    k, n = 320, 448
    block = workloads.block_desc
    dx, dw, dh, dd, dy = block(m, k, 1, 1), block(k, n, 1, 2), block(m, n, 1, 2), block(n, k, 2, 1), block(m, k, 1, 1)
    up, down = binding.Plan(dx, dw, dh, 2), binding.Plan(dh, dd, dy, 2)
    X, Wg, Wu, Wd = normal(m, k, 1), normal(k, n, 2, k ** -0.5), normal(k, n, 3, k ** -0.5), normal(n, k, 4, n ** -0.5)
    s = stream()
    forms = []
    for d, W in ((dw, Wg), (dw, Wu), (dd, Wd)):
        f = Int8(d, "cols")
        binding.dmm_int_quantize(binding.matrix_desc(d), binding.DMM_BF16, Tiles(d, BF16, W).table(), cols=f.table(), stream=s)
        forms.append(f)
    fx, fh, h, y = Int8(dx, "rows"), Int8(dh, "rows"), Tiles(dh, BF16), Tiles(dy, BF16)
    binding.dmm_int_quantize(binding.matrix_desc(dx), binding.DMM_BF16, Tiles(dx, BF16, X).table(), rows=fx.table(), stream=s)
    up.gated_int(binding.DMM_SILU, fx.table(), forms[0].table(), forms[1].table(), h.table(), s)
    binding.dmm_int_quantize(binding.matrix_desc(dh), binding.DMM_BF16, h.table(), rows=fh.table(), stream=s)
    down.execute_int(fh.table(), forms[2].table(), y.table(), binding.DMM_C_BF16, s)
    torch.cuda.synchronize()
    (qx, sx), (qg, sg), (qu, su), (qd, sd) = quantized(X, 1), quantized(Wg, 0), quantized(Wu, 0), quantized(Wd, 0)
    g, u = ((qx @ q) * (sx.double().unsqueeze(1) * t.double()) for q, t in ((qg, sg), (qu, su)))
    want = act(g, "silu")[0] * u
    close(h.whole(), want, H * want.abs() + (1 + H) * gated_error(g, u, 3.01 * U * g.abs(), 3.01 * U * u.abs(), "silu") + TINY, "H")
    qh, sh = quantized(h.whole(), 1)
    assert torch.equal(fh.q.whole(), qh) and torch.equal(fh.scales(), sh)
    want = (qh @ qd) * (sh.double().unsqueeze(1) * sd.double())
    close(y.whole(), want, (3.01 * U + H) * want.abs(), "Y")
    # the layer by itself: integers instead of values cost each operand at most half a step of its row
    exact = (act(X.double() @ Wg.double(), "silu")[0] * (X.double() @ Wu.double())) @ Wd.double()
    assert float(torch.linalg.vector_norm(y.whole() - exact) / torch.linalg.vector_norm(exact)) < 0.05
