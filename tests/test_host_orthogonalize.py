"""What ``dmm_orthogonalize`` refuses (made-up device addresses: nothing is launched), and its oracle
against singular values."""
import ctypes

import numpy as np
import pytest

import workloads
from oracle import orthogonalize as oracle
from paper_2510_08874_amd import binding

BASE = 1 << 40


def whole(h, w, replication=1):
    return workloads.desc(h, w, [0, h], [0, w], 1, 1, replication=replication)


def call(d=whole(40, 300), count=1, xt=1, x=BASE, x_ld=300, yt=2, y=BASE + (1 << 20), y_ld=300, ws=BASE + (1 << 30), size=None, coefficients=None, steps=5):
    desc = binding.matrix_desc(d)
    if size is None:
        size = binding.dmm_orthogonalize_workspace(binding.matrix_desc(whole(40, 300)), max(count, 0))
    binding.dmm_orthogonalize(desc, count, xt, binding.tile_table([x] * max(count, 1), [x_ld] * max(count, 1)), yt,
                              binding.tile_table([y] * max(count, 1), [y_ld] * max(count, 1)), ws, size, coefficients, steps)


@pytest.mark.parametrize("kind,kw", [
    ("EINVAL", dict(count=-1)), ("EINVAL", dict(xt=0)), ("EINVAL", dict(yt=3)), ("EINVAL", dict(x=0)), ("EINVAL", dict(y=0)),
    ("EINVAL", dict(x=BASE + 1)), ("EINVAL", dict(y=BASE + 2)), ("ELD", dict(x_ld=299)), ("ELD", dict(y_ld=299)), ("EINVAL", dict(steps=0)), ("EINVAL", dict(coefficients=[(1.0, 0.0, 0.0)] * 33)),
    ("EINVAL", dict(steps=6)), ("EINVAL", dict(coefficients=[])), ("EINVAL", dict(ws=0)), ("EINVAL", dict(ws=BASE + 128)), ("ELIMIT", dict(size=1000)),
    ("EREPL", dict(d=whole(40, 300, 2))), ("ELIMIT", dict(d=whole(1 << 21, 30))), ("EINVAL", dict(d=dict(whole(40, 300), col_cuts=(0, 301)))),
    ("EINVAL", dict(coefficients=[(16.0, 0.0, 0.0)])), ("EINVAL", dict(coefficients=[(1.0, 20.0, 0.0)])), ("EINVAL", dict(coefficients=[(4.0, 0.0, 0.0)] * 2)),
    ("EINVAL", dict(coefficients=[(float("nan"), 0.0, 0.0)])), ("EINVAL", dict(coefficients=[(1.0, float("inf"), 0.0)])),
], ids=str)
def test_arguments_that_are_refused(kind, kw):
    with pytest.raises(binding.DmmError) as e:
        call(**kw)
    assert e.value.kind == kind, e.value


def test_null_arguments():
    L, d, n = binding.lib(), binding.matrix_desc(whole(4, 4)), ctypes.c_int64()
    assert L.dmm_orthogonalize_workspace(None, 1, ctypes.byref(n)) == binding.DMM_EINVAL
    assert L.dmm_orthogonalize_workspace(ctypes.byref(d), 1, None) == binding.DMM_EINVAL
    assert L.dmm_orthogonalize(None, 1, 1, None, None, 1, None, None, None, 5, None, 0, None) == binding.DMM_EINVAL
    assert L.dmm_orthogonalize(ctypes.byref(d), 1, 1, None, None, 1, None, None, None, 5, None, 0, None) == binding.DMM_EINVAL


def test_workspace_grows_with_the_matrix_and_their_number():
    one = binding.dmm_orthogonalize_workspace(binding.matrix_desc(whole(1024, 4096)), 1)
    assert one >= 2 * 2 * 4 * 1024 * 4096 and binding.dmm_orthogonalize_workspace(binding.matrix_desc(whole(4096, 1024)), 1) == one
    assert binding.dmm_orthogonalize_workspace(binding.matrix_desc(whole(200, 200)), 8) > 7 * 2 * 2 * 4 * 200 * 200
    # one workgroup a matrix: none
    assert binding.dmm_orthogonalize_workspace(binding.matrix_desc(whole(128, 100)), 8) == 0
    assert binding.dmm_orthogonalize_workspace(binding.matrix_desc(workloads.desc(128, 100, [0, 64, 128], [0, 100], 2, 1)), 1) > 0


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 9), (9, 5), (40, 40)])
def test_oracle_acts_on_singular_values(rows, cols):
    rng = np.random.default_rng(rows + cols)
    G = rng.standard_normal((rows, cols))
    U, s, V = np.linalg.svd(G, full_matrices=False)
    s = s / np.sqrt((s * s).sum())
    for a, b, c in oracle.DEFAULT:
        s = a * s + b * s ** 3 + c * s ** 5
    Y = oracle.orthogonalize(G)
    assert np.abs(Y - (U * s) @ V).max() < 1e-12
    # the bound is one for fp32 arithmetic too, and tells a result in bf16 from it
    X = (G / np.linalg.norm(G)).astype(np.float32)
    X = X.T if rows > cols else X
    for a, b, c in oracle.DEFAULT:
        S = X @ X.T
        X = np.float32(a) * X + (np.float32(b) * S + np.float32(c) * (S @ S)) @ X
    X = X.T if rows > cols else X
    assert np.linalg.norm(X - Y) <= oracle.limit(G) < 2.0 ** -9 * np.linalg.norm(Y) * 2
