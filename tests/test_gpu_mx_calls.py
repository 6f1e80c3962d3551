"""GPU tests of calls of `dmm_mx_execute` around each other: captures of replicated products, few rows."""
import numpy as np
import pytest

import workloads
from oracle import mx as oracle
from tests.test_gpu_mx import DT, check_product, gather, limit, made, operand, tiles_of, whole

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


@pytest.mark.parametrize("c_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(3, 2100, 9001), (31, 1157, 8897), (32, 700, 12865)], ids=str)
def test_tiles_of_32_rows_are_stored_from_the_registers(m, k, n, c_dtype):
    """Uncut: whole tiles and such that end inside of 32 columns (one column, the last bf16 by itself), rows at any address; in
    row blocks, where every one of them has a tile of its own, too."""
    (a, A), (b, B) = made(m, k, 1, m + n), made(k, n, 2, k + n)
    flags, stream = binding.DMM_C_BF16 if c_dtype == "bf16" else 0, torch.cuda.current_stream().cuda_stream
    for offset, ld in ((0, n), (1, n + 2)):
        buf = torch.full((m * ld + offset,), 7.0, dtype=DT[c_dtype][0], device="cuda")
        c = buf[offset:].view(m, ld)
        binding.Plan(whole(m, k), whole(k, n), whole(m, n), 1).execute_mx(a.table(), b.table(), binding.tile_table([c], [ld]), flags, stream)
        check_product(c[:, :n], A, B, c_dtype)
        assert (c[:, n:] == 7.0).all() and (buf[:offset] == 7.0).all()
    cut = [0, m // 2, m]
    d = workloads.desc(m, k, cut, [0, k], 2, 1), whole(k, n), workloads.desc(m, n, cut, [0, n], 2, 1)
    rows = [(a.codes[0][r0:r1], a.scales[0][r0:r1]) for r0, r1 in zip(cut, cut[1:])]
    ta = binding.mx_tiles([x[0] for x in rows], [x[0].shape[1] for x in rows], [x[1] for x in rows], [x[1].shape[1] for x in rows])
    out, want = torch.full((m, n), 7.0, dtype=DT[c_dtype][0], device="cuda"), c[:, :n]
    binding.Plan(*d, 2).execute_mx(ta, b.table(), binding.tile_table([out[:m // 2], out[m // 2:]], [n, n]), flags, stream)
    assert torch.equal(out, want)


def test_values_of_scales_beyond_those_that_quantisation_makes():
    """Bytes 253 and 254: values past the largest number become infinite, with their sign; the others are exact."""
    codes = torch.arange(256, dtype=torch.int64).to(torch.uint8).repeat(2, 1).cuda()
    scales = torch.tensor([[253] * 16, [254] * 16], dtype=torch.uint8, device="cuda")
    want = oracle.values(oracle.unpack(codes.cpu().numpy()), scales.cpu().numpy(), 512)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    for dtype in ("bf16", "f32"):
        out = torch.zeros(2, 512, dtype=DT[dtype][0], device="cuda")
        binding.dmm_mx_dequantize(binding.matrix_desc(whole(2, 512)), binding.mx_tiles([codes], [256], [scales], [16]), 1, DT[dtype][1],
                                  binding.tile_table([out], [512]), torch.cuda.current_stream().cuda_stream)
        assert np.array_equal(out.double().cpu().numpy(), want) and np.isinf(want).any()
