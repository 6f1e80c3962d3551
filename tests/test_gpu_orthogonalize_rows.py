"""GPU tests of ``dmm_orthogonalize`` on rows of very different size, and of small matrices in tile grids against the path
that takes them in one tile."""
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
