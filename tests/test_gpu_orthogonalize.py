"""GPU tests of ``dmm_orthogonalize`` against the oracle: shapes, tile grids, types, many matrices at a time,
what must stay untouched, values that are no finite numbers, streams and graphs."""
import numpy as np
import pytest

import workloads
from oracle import orthogonalize as oracle

torch = pytest.importorskip("torch")
binding = pytest.importorskip("paper_2510_08874_amd.binding")
pytestmark = pytest.mark.gpu

DT = {"bf16": (torch.bfloat16, 1), "f32": (torch.float32, 2)}


def whole(h, w):
    return workloads.desc(h, w, [0, h], [0, w], 1, 1)


def bounds(d):
    return [(r0, r1, c0, c1) for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]) for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:])]


def tiles(mats, d, dtype, ld_more=0, offset=0):
    out, ld = [], []
    for M in mats:
        for r0, r1, c0, c1 in bounds(d):
            h, w = r1 - r0, c1 - c0
            ld.append(w + ld_more)
            if not h or not w:
                out.append(None)
                continue
            buf = torch.full((h * (w + ld_more) + offset,), 7.0, dtype=dtype, device="cuda")
            t = buf[offset:].view(h, w + ld_more)
            t[:, :w] = M[r0:r1, c0:c1].to(dtype)
            out.append(t)
    return out, ld


def gather(ts, d, count):
    per, out = len(bounds(d)), []
    for x in range(count):
        M = np.zeros((d["rows"], d["cols"]))
        for t, (r0, r1, c0, c1) in zip(ts[x * per:(x + 1) * per], bounds(d)):
            if t is not None:
                M[r0:r1, c0:c1] = t[:, :c1 - c0].double().cpu().numpy()
                assert (t[:, c1 - c0:] == 7.0).all(), "written behind a row's end"
        out.append(M)
    return out


def run(mats, d, x_dtype="f32", y_dtype="f32", coefficients=None, steps=5, ld_more=0, offset=0, in_place=False):
    x, x_ld = tiles(mats, d, DT[x_dtype][0], ld_more, offset)
    y, y_ld = (x, x_ld) if in_place else tiles([torch.zeros(d["rows"], d["cols"], device="cuda")] * len(mats), d, DT[y_dtype][0], ld_more, offset)
    desc = binding.matrix_desc(d)
    size = binding.dmm_orthogonalize_workspace(desc, len(mats))
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")    # (NaN as fp16, in every place)
    binding.dmm_orthogonalize(desc, len(mats), DT[x_dtype][1], binding.tile_table(x, x_ld), DT[y_dtype][1], binding.tile_table(y, y_ld), ws, size,
                              coefficients=coefficients, steps=steps, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (ws[size:] == 0xFF).all(), "written behind the workspace"
    given = [M.to(DT[x_dtype][0]).double().cpu().numpy() for M in mats]
    return gather(y, d, len(mats)), given


def check(got, given, y_dtype="f32", coefficients=oracle.DEFAULT):
    for Y, G in zip(got, given):
        want = oracle.orthogonalize(G, coefficients)
        far = oracle.limit(G, coefficients)
        if y_dtype == "bf16":
            far += 2.0 ** -8 * (np.linalg.norm(want) + far)
        assert np.linalg.norm(Y - want) <= far, (np.linalg.norm(Y - want), far)


def random(count, rows, cols, seed, kind="plain"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn(count, rows, cols, generator=g, device="cuda")
    if kind == "strong":                                     # a few strong directions over a floor of noise
        r = max(1, min(rows, cols) // 16)
        X = 0.03 * X + torch.matmul(torch.randn(count, rows, r, generator=g, device="cuda"), torch.randn(count, r, cols, generator=g, device="cuda"))
    return list(X * 1e-3)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 40), (40, 1), (2, 3), (31, 33), (32, 32), (33, 31), (64, 130), (127, 128), (128, 128), (129, 257),
                                       (300, 1000), (700, 256), (513, 520)], ids=str)
@pytest.mark.parametrize("kind", ["plain", "strong"])
def test_one_matrix(rows, cols, kind):
    got, given = run(random(1, rows, cols, rows * 7 + cols, kind), whole(rows, cols))
    check(got, given)


@pytest.mark.parametrize("x_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("y_dtype", ["bf16", "f32"])
def test_types_and_rows_that_are_longer(x_dtype, y_dtype):
    for rows, cols in ((70, 101), (101, 70)):
        got, given = run(random(2, rows, cols, 5), whole(rows, cols), x_dtype, y_dtype, ld_more=3, offset=1)
        check(got, given, y_dtype)


@pytest.mark.parametrize("count,rows,cols", [(3, 20, 30), (70, 17, 40), (64, 300, 700), (5, 200, 129)], ids=str)
def test_many_matrices(count, rows, cols):
    """Each by itself: very different sizes of their elements, more of them than a launch takes tiles of; large macro-tiles."""
    mats = [M * 10.0 ** (i % 9 - 4) for i, M in enumerate(random(count, rows, cols, count))]
    got, given = run(mats, whole(rows, cols))
    check(got[:4] + got[-2:], given[:4] + given[-2:])
    one, _ = run(mats[2:3], whole(rows, cols))
    assert np.linalg.norm(one[0] - got[2]) <= 2 * oracle.limit(given[2])


def test_tile_grids():
    """Uneven tiles, empty ones among them; more tiles than one launch takes."""
    d = workloads.desc(150, 210, [0, 0, 1, 64, 100, 150], [0, 70, 70, 199, 210, 210], 5, 5)
    got, given = run(random(2, 150, 210, 8, "strong"), d)
    check(got, given)
    d = workloads.desc(330, 250, list(range(0, 331, 30)), list(range(0, 251, 25)), 11, 10)
    got, given = run(random(1, 330, 250, 9), d, "bf16", "bf16")
    check(got, given, "bf16")


def test_diagonal_matrices_element_by_element():
    """The result is known in closed form: the polynomials of the normalised diagonal, zeros elsewhere."""
    v = np.concatenate([np.logspace(-6, 0, 50), -np.logspace(-2, 0, 20), [0.0]])
    for rows, cols in ((71, 90), (90, 71)):
        G = torch.zeros(rows, cols, device="cuda")
        G[range(71), range(71)] = torch.from_numpy(v).float().cuda() * 1e20
        got, given = run([G], whole(rows, cols))
        x = given[0][range(71), range(71)]
        x = x / np.sqrt((x * x).sum())
        far = np.full(71, 2.0 ** -22) * np.abs(x) + 2.0 ** -37
        for a, b, c in oracle.DEFAULT:
            # every value of the step is held or multiplied to 2^-21 of itself; fp16's smallest step, 2^-25 of 1 / 4096, below that
            size = np.abs(a * x) + np.abs(b * x ** 3) + np.abs(c * x ** 5)
            far = far * np.abs(a + 3 * b * x ** 2 + 5 * c * x ** 4) * 1.01 + 8 * 2.0 ** -21 * size + 2.0 ** -35
            x = a * x + b * x ** 3 + c * x ** 5
        err = np.abs(got[0][range(71), range(71)] - x)
        assert (err <= far).all(), (err / far).max()
        got[0][range(71), range(71)] = 0
        assert not got[0].any()


@pytest.mark.parametrize("coefficients", [((1.5, -0.5, 0.0),) * 7, ((2.0, -1.5, 0.5),), ((8.0, -20.0, 13.0), (1.875, -1.25, 0.375))], ids=str)
def test_other_coefficients(coefficients):
    got, given = run(random(1, 90, 150, 3), whole(90, 150), coefficients=coefficients)
    check(got, given, coefficients=coefficients)


def test_fewer_steps_and_in_place():
    mats = random(2, 60, 45, 12)
    for steps in (1, 2, 3):
        got, given = run(mats, whole(60, 45), steps=steps)
        check(got, given, coefficients=oracle.DEFAULT[:steps])
    got, given = run(mats, whole(60, 45), "bf16", "bf16", in_place=True)
    check(got, given, "bf16")


def test_values_that_are_no_numbers_stay_in_their_matrix():
    mats = random(5, 50, 77, 2)
    mats[0][3, 4], mats[1][49, 76], mats[2][:] = float("nan"), float("inf"), 0.0
    mats[3] *= 1e36                                          # squares beyond fp32
    mats[4] *= 1e-36
    got, given = run(mats, whole(50, 77))
    assert np.isnan(got[0]).all() and np.isnan(got[1]).all() and not got[2].any()
    check(got[3:], given[3:])
    got, _ = run([torch.full((9, 5), float("-inf"), device="cuda")], whole(9, 5), "bf16", "bf16")
    assert np.isnan(got[0]).all()


def test_nothing_to_do():
    for d, count in ((whole(0, 5), 1), (whole(5, 0), 2), (whole(5, 5), 0)):
        desc = binding.matrix_desc(d)
        assert binding.dmm_orthogonalize_workspace(desc, count) == 0
        binding.dmm_orthogonalize(desc, count, 1, binding.tile_table([None] * count, [5] * count), 1, binding.tile_table([None] * count, [5] * count), 0, 0)


def test_streams_and_a_captured_graph():
    """Two streams with workspaces of their own at the same time; a graph replayed with eager work in between; the same bits every time."""
    d, n = whole(260, 300), 2
    desc = binding.matrix_desc(d)
    size = binding.dmm_orthogonalize_workspace(desc, 1)
    G = [M.bfloat16() for M in random(n, 260, 300, 40, "strong")]
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(n)]
    Y = [torch.zeros(260, 300, device="cuda") for _ in range(n)]
    streams = [torch.cuda.Stream() for _ in range(n)]
    torch.cuda.synchronize()

    def call(i, stream):
        binding.dmm_orthogonalize(desc, 1, 1, binding.tile_table([G[i]], [300]), 2, binding.tile_table([Y[i]], [300]), ws[i], size, stream=stream)

    for i in range(n):
        call(i, streams[i].cuda_stream)
    torch.cuda.synchronize()
    check([y.double().cpu().numpy() for y in Y], [g.double().cpu().numpy() for g in G])
    want = [y.clone() for y in Y]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0], capture_error_mode="relaxed"):
        call(0, streams[0].cuda_stream)
    for _ in range(3):
        Y[0].zero_()
        ws[0].fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        call(1, streams[1].cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(y, w) for y, w in zip(Y, want))
        Y[1].zero_()
        torch.cuda.synchronize()
    del graph


def exact(G):
    X = G.double()
    X = X / torch.linalg.vector_norm(X)
    X = X.t().contiguous() if G.shape[0] > G.shape[1] else X
    for a, b, c in oracle.DEFAULT:
        S = X @ X.t().contiguous()
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.t() if G.shape[0] > G.shape[1] else X


@pytest.mark.parametrize("rows,cols", [(1021, 2043), (700, 513), (120, 90), (129, 3000), (2048, 2048), (4200, 4300)], ids=str)
def test_fp32_results_are_as_exact_as_fp32_arithmetic(rows, cols):
    """Strong directions nearly cancel on the way: whatever rounds at the size of the cancelling parts shows in the others.  The same
    steps in plain fp32 round as often at that size: no more than half as much again is lost."""
    X = random(1, rows, cols, 21, "strong")
    d = workloads.desc(rows, cols, [0, rows // 3, rows], [0, 1, cols], 2, 2)
    got, _ = run(X, d)
    want = exact(X[0]).cpu().numpy()
    Y = X[0] / X[0].double().norm().float()
    Y = Y.t().contiguous() if rows > cols else Y
    for a, b, c in oracle.DEFAULT:
        S = Y @ Y.t().contiguous()
        Y = a * Y + (b * S + c * (S @ S)) @ Y
    Y = (Y.t() if rows > cols else Y).double().cpu().numpy()
    assert np.linalg.norm(got[0] - want) <= 1.5 * np.linalg.norm(Y - want)


@pytest.mark.parametrize("even", [True, False])
def test_many_small_matrices(even):
    """More than a launch's argument names, evenly spaced in memory and not; the same matrix twice."""
    count, rows, cols = 301, 30, 41
    mats = random(count, rows, cols, 17)
    at = np.arange(count) * rows * cols if even else np.cumsum(np.random.default_rng(3).integers(rows * cols, rows * cols + 50, count))
    buf = torch.zeros(int(at[-1]) + rows * cols, device="cuda")
    out = torch.zeros_like(buf)
    view = lambda b, i: b[int(at[i]):int(at[i]) + rows * cols].view(rows, cols)
    for i, M in enumerate(mats):
        view(buf, i).copy_(M)
    x = [view(buf, i) for i in range(count)]
    if not even:
        x[7] = x[8]
    desc = binding.matrix_desc(whole(rows, cols))
    binding.dmm_orthogonalize(desc, count, 2, binding.tile_table(x, [cols] * count), 2, binding.tile_table([view(out, i) for i in range(count)], [cols] * count),
                              None, 0, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for i in (0, 1, 7, 143, 144, 145, 299, 300):
        G = x[i].double().cpu().numpy()
        assert np.linalg.norm(view(out, i).double().cpu().numpy() - oracle.orthogonalize(G)) <= oracle.limit(G)
    if not even:
        assert torch.equal(view(out, 7), view(out, 8))


def test_calls_from_several_threads():
    """Each with its own stream and buffers, on one shape of each kind; the same bits as one call alone."""
    import threading
    made = []
    for rows, cols in ((90, 100), (200, 333)):
        mats = random(3, rows, cols, rows)
        d = binding.matrix_desc(whole(rows, cols))
        size = binding.dmm_orthogonalize_workspace(d, 3)
        want, _ = run(mats, whole(rows, cols))
        made.append((mats, d, size, rows, cols, want))
    jobs, errors = [], []
    for i in range(6):
        mats, d, size, rows, cols, want = made[i % 2]
        out = [torch.zeros(rows, cols, device="cuda") for _ in mats]
        jobs.append((d, binding.tile_table(mats, [cols] * 3), binding.tile_table(out, [cols] * 3), torch.empty(size + 256, dtype=torch.uint8, device="cuda"), size,
                     torch.cuda.Stream(), out, want))
    torch.cuda.synchronize()

    def work(d, x, y, ws, size, stream, out, want):
        try:
            for _ in range(10):
                binding.dmm_orthogonalize(d, 3, 2, x, 2, y, ws if size else None, size, stream=stream.cuda_stream)
        except Exception as e:                                # (told by the test, not by the thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for j in jobs:
        for got, want in zip(j[6], j[7]):
            assert np.array_equal(got.double().cpu().numpy(), want)
