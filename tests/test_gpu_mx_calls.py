"""GPU tests of calls of `dmm_mx_execute` around each other: captures of replicated products."""
import numpy as np
import pytest

import workloads
from tests.test_gpu_mx import gather, limit, operand, tiles_of

torch = pytest.importorskip("torch")
binding = pytest.importorskip("paper_2510_08874_amd.binding")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["global", "relaxed"])
def test_a_replicated_product_is_captured(mode):
    """After a call that did not sum, and after a sum of other tiles on the same plan: every replay, with eager work between,
    gives what the eager call gives, in both replicas."""
    m, k, n = 300, 1024, 260
    d = [workloads.block_desc(r, c, 2, 2, replication=2) for r, c in ((m, k), (k, n), (m, n))]
    plan = binding.Plan(*d, 8)
    (a, A), (b, B) = operand(d[0], 1, 51), operand(d[1], 2, 52)
    fill = torch.full((m, n), float("nan"), device="cuda")
    c, ld = tiles_of(fill, d[2], torch.float32)
    other, other_ld = tiles_of(torch.ones(m, n, device="cuda"), d[2], torch.float32)
    ta, tb, tc = a.table(), b.table(), binding.tile_table(c, ld)
    first, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    plan.execute_mx(ta, tb, tc, binding.DMM_NO_REDUCE, first.cuda_stream)
    plan.reduce_replicas(other, other_ld, 1, first.cuda_stream)
    torch.cuda.synchronize()
    assert (gather(other, d[2], 1) == 2).all() and (gather(other, d[2], 0) == 1).all()
    part = gather(c, d[2], 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode=mode):
        plan.execute_mx(ta, tb, tc, 0, side.cuda_stream)
    plan.execute_mx(ta, tb, tc, 0, side.cuda_stream)
    torch.cuda.synchronize()
    want = [t.clone() for t in c]
    assert (np.abs(gather(c, d[2], 0) - A @ B) <= limit(A, B, "f32", k)).all() and np.array_equal(gather(c, d[2], 1), part)
    for _ in range(3):
        for t in c:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(c, want))
        plan.execute_mx(ta, tb, tc, binding.DMM_NO_REDUCE, side.cuda_stream)
        plan.reduce_replicas(other, other_ld, 0, side.cuda_stream)
        torch.cuda.synchronize()
        assert np.array_equal(gather(c, d[2], 1), part)
    del graph
