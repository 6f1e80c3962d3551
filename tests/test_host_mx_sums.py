"""The bounds for sums of 4-bit products tell fp32 from fewer bits: mistakes planted in sums made here, at the sizes that the
library cuts along K."""
import numpy as np
import pytest

from oracle import mx as oracle
from tests.test_gpu_mx_sums import CUT


def short(x, dtype):
    """Doubles rounded to bf16 or fp16."""
    if dtype == "fp16":
        return (x / 64).astype(np.float16).astype(np.float64) * 64
    bits = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return (((bits + 0x7FFF + (bits >> 16 & 1)) >> 16 << 16).astype(np.uint32)).view(np.float32).astype(np.float64)


def ranges(A, B, runs):
    cut = [-(-A.shape[1] * i // runs) // 256 * 256 for i in range(runs)] + [A.shape[1]]
    return [A[:, x:y] @ B[x:y] for x, y in zip(cut, cut[1:])]


@pytest.mark.parametrize("m,k,n", CUT, ids=str)
def test_random_terms(m, k, n):
    rng, n, m = np.random.default_rng(k + n), min(n, 128), min(m, 128)
    A = oracle.values(*oracle.quantize(rng.standard_normal((m, k))), k)
    B = oracle.values(*oracle.quantize(rng.standard_normal((n, k))), k).T
    exact, far = A @ B, oracle.sum_limit(A, B)
    steps = np.zeros((m, n), np.float32)
    for c in range(0, k, 64):
        steps = (steps + A[:, c:c + 64] @ B[c:c + 64]).astype(np.float32)
    assert np.linalg.norm(steps - exact) <= far
    for runs in (2, 4, 16):
        parts = ranges(A, B, runs)
        assert np.linalg.norm(sum(p.astype(np.float32).astype(np.float64) for p in parts) - exact) <= far
        for dtype in ("bf16", "fp16"):
            assert np.linalg.norm(sum(short(p, dtype) for p in parts) - exact) > far
    assert np.linalg.norm(short(exact, "bf16") - exact) > far


@pytest.mark.parametrize("m,k,n", CUT, ids=str)
def test_exact_sums(m, k, n):
    """Positive codes of one scale: every sum is a multiple of a quarter below 2^22, exact in fp32 and not in less."""
    rng, n, m = np.random.default_rng(k), min(n, 64), min(m, 64)
    A, B = oracle.VALUES[rng.integers(1, 8, (m, k))], oracle.VALUES[rng.integers(1, 8, (k, n))]
    exact = A @ B
    assert exact.max() < 2 ** 22 and np.array_equal(exact, exact.astype(np.float32)) and np.array_equal(exact * 4, np.rint(exact * 4))
    for runs in (2, 4, 16):
        parts = ranges(A, B, runs)
        assert np.array_equal(sum(parts), exact)
        for dtype in ("bf16", "fp16"):
            assert not np.array_equal(sum(short(p, dtype) for p in parts), exact)
