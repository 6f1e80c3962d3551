"""GPU tests of ``dmm_orthogonalize`` on rows of very different size, of small matrices in tile grids against the path
that takes them in one tile, and of results in bf16 against exact ones rounded."""
import numpy as np
import pytest

import workloads
from oracle import orthogonalize as oracle

torch = pytest.importorskip("torch")


def falling(rows, cols, decades, seed):
    """Rows whose sizes fall evenly over so many decades, in fp32."""
    X = np.random.default_rng(seed).standard_normal((rows, cols)) * (10.0 ** -np.linspace(0, decades, rows))[:, None]
    return X.astype(np.float32)


def row_errors(Y, exact):
    return np.sqrt(((np.asarray(Y, dtype=np.float64) - exact) ** 2).sum(axis=1))


def row_limits(G, exact):
    """What rounding to pairs and what sums in fp32 do to every row, each by itself; four times, since which way a rounding goes is
    another thing every time: with columns in other orders and values scaled before they become pairs, computed on the CPU, both
    together came to at most 2.2 times the sum."""
    return 4 * (row_errors(oracle.held(G, oracle.pair), exact) + row_errors(oracle.in_fp32(G), exact))


ROWS = [(256, 1024, d) for d in (0, 3, 6, 8)] + [(60, 90, 6), (128, 128, 8), (200, 300, 7)]


@pytest.mark.gpu
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows,cols,decades", ROWS, ids=str)
def test_rows_of_very_different_size(rows, cols, decades, turned):
    from tests.test_gpu_orthogonalize import run, whole
    G = falling(rows, cols, decades, rows + decades)
    M = torch.from_numpy(G.T.copy() if turned else G).cuda()
    got, _ = run([M], whole(*M.shape))
    exact = oracle.orthogonalize(G)
    err, far = row_errors(got[0].T if turned else got[0], exact), row_limits(G, exact)
    assert (err <= far).all(), (err / far).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,row_cuts,col_cuts", [
    (128, 128, [0, 64, 128], [0, 64, 128]), (100, 77, [0, 1, 50, 100], [0, 76, 77]), (77, 100, [0, 77], [0, 33, 33, 100]), (1, 50, [0, 1], [0, 7, 50]),
    (30, 1, [0, 29, 30], [0, 1]),
], ids=str)
def test_small_matrices_in_tile_grids(rows, cols, row_cuts, col_cuts, dtype):
    """The path of launches gives what the one-workgroup path gives, up to what both may be off."""
    from tests.test_gpu_orthogonalize import check, random, run, whole
    mats = random(2, rows, cols, rows + cols, "strong")
    one, given = run(mats, whole(rows, cols), dtype, dtype)
    grid, _ = run(mats, workloads.desc(rows, cols, row_cuts, col_cuts, len(row_cuts) - 1, len(col_cuts) - 1), dtype, dtype)
    check(one, given, dtype)
    check(grid, given, dtype)
    for x, y, G in zip(one, grid, given):
        # (bf16: two roundings of nearly the same value, a step of 2^-7 of it at most)
        far = 2 * oracle.limit(G)
        assert np.linalg.norm(x - y) <= far + (2.0 ** -7 * (np.linalg.norm(x) + far) if dtype == "bf16" else 0.0)
        exact = oracle.orthogonalize(G)
        if dtype == "f32" and min(rows, cols) > 64:
            assert (row_errors(x, exact) <= row_limits(G, exact)).all() and (row_errors(y, exact) <= row_limits(G, exact)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("count,rows,cols", [(1, 1024, 2048), (8, 700, 600), (24, 300, 500), (1, 2048, 2048), (32, 128, 128)], ids=str)
def test_bf16_results_are_as_near_as_those_of_fp32_arithmetic(count, rows, cols):
    """How many elements fall on the other side of a border of the last rounding goes with the error in front of it: no more than
    where the same steps are made in fp32, whose error a result in fp32 does not reach."""
    from tests.test_gpu_orthogonalize import exact, random, tiles, whole
    from paper_2510_08874_amd import binding
    mats = [M.bfloat16() for M in random(count, rows, cols, rows + cols, "strong")]
    d = whole(rows, cols)
    y, ld = tiles([torch.zeros(rows, cols, device="cuda")] * count, d, torch.bfloat16)
    desc = binding.matrix_desc(d)
    size = binding.dmm_orthogonalize_workspace(desc, count)
    ws = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    binding.dmm_orthogonalize(desc, count, 1, binding.tile_table(mats, [cols] * count), 1, binding.tile_table(y, ld), ws if size else None, size,
                              stream=torch.cuda.current_stream().cuda_stream)
    own = plain = 0
    for M, Y in zip(mats, y):
        want = exact(M).float().bfloat16()
        X = M.float() / M.double().norm().float()
        X = X.t().contiguous() if rows > cols else X
        for a, b, c in oracle.DEFAULT:
            S = X @ X.t().contiguous()
            X = a * X + (b * S + c * (S @ S)) @ X
        own += int((Y != want).sum())
        plain += int(((X.t() if rows > cols else X).bfloat16() != want).sum())
    assert 0 < own <= plain, (own, plain)


@pytest.mark.parametrize("rows,cols,decades", ROWS, ids=str)
def test_the_limits_tell_pairs_from_fp16(rows, cols, decades):
    """On the CPU: matrices held as single fp16 numbers are far outside."""
    G = falling(rows, cols, decades, rows + decades)
    exact = oracle.orthogonalize(G)
    far = row_limits(G, exact)
    single = oracle.held(G, lambda x: (x * 4096).astype(np.float16).astype(np.float64) / 4096)
    assert (row_errors(single, exact) > far).mean() > 0.5
    worst = (row_errors(oracle.held(G, oracle.pair), exact) / np.linalg.norm(exact, axis=1)).max()
    assert worst <= (1e-5 if decades <= 3 else 1e-1)
