"""GPU tests of the layers around a product at the edges of what their calls allow.  Limits as in test_gpu_layer.py."""
import pytest

import workloads
from tests.layer_tiles import ACTS, Tiles, act, descs, normal, stream
from tests.test_gpu_layer import H, TINY, U, argument, close, gated_error, sum_error

torch = pytest.importorskip("torch")
binding = pytest.importorskip("paper_2510_08874_amd.binding")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("m,blocks,k,n,last", [(8, 8, 4097, 8195, 3), (8, 1, 4098, 8194, 2), (8, 2, 4102, 8193, 1), (64, 8, 8193, 8195, 3)], ids=str)
def test_narrow_tiles_of_weights_behind_a_copy_of_the_rows(m, blocks, k, n, last, name):
    """The weights' last tile has one to three columns: rows that whole steps leave out are multiplied behind these, with the copy's columns there."""
    da, db, dc = workloads.block_desc(m, k, 8, 1), workloads.desc(k, n, [0, k], [0, n - last, n], 1, 2), workloads.block_desc(m, n, blocks, 1)
    plan = binding.Plan(da, db, dc, 8)
    A, Wg, Wu = normal(m, k, 1), normal(k, n, 2, 2 * k ** -0.5), normal(k, n, 3, k ** -0.5)
    g, u = A.double() @ Wg.double(), A.double() @ Wu.double()
    eg, eu = sum_error(A.double(), Wg.double()), sum_error(A.double(), Wu.double())
    want = act(g, name)[0] * u
    a, wg, wu = (Tiles(d, BF16, x) for d, x in ((da, A), (db, Wg), (db, Wu)))
    h, kg, ku = (Tiles(dc, BF16) for _ in range(3))
    plan.gated(ACTS[name], *(t.table() for t in (a, wg, wu, h, kg, ku)), stream=stream())
    torch.cuda.synchronize()
    close(kg.whole(), g, H * g.abs() + (1 + H) * eg, "G")
    close(ku.whole(), u, H * u.abs() + (1 + H) * eu, "U")
    close(h.whole(), want, H * want.abs() + (1 + H) * gated_error(g, u, eg, eu, name) + TINY, "H")
    for t in (h, kg, ku):
        t.check_guards()


@pytest.mark.parametrize("layout,m,k,n", [("whole", 4096, 1024, 1024), ("whole", 8192, 512, 768), ("whole", 8192, 1024, 3072), ("whole", 2048, 256, 512), ("whole", 1111, 300, 500),
                                          ("blocks", 3000, 256, 384), ("uneven", 1301, 1103, 907), ("uneven", 2500, 300, 400), ("row_col", 83, 520, 4096)], ids=str)
def test_gradients_do_not_depend_on_what_else_is_asked_for(layout, m, k, n):
    """Bit for bit, whatever macro-tiles and launches the others bring with them.  The sums are cut along K."""
    (da, db, dc), ranks = descs(layout, m, k, n)
    plan = binding.Plan(da, db, dc, ranks)
    a, wg, wu = (Tiles(d, BF16, normal(d["rows"], d["cols"], i, s)) for i, (d, s) in enumerate(((da, 1), (db, k ** -0.5), (db, k ** -0.5))))
    g, u, dh = (Tiles(dc, BF16, normal(m, n, 5 + i)) for i in range(3))
    dg, du = Tiles(dc, BF16), Tiles(dc, BF16)
    want = None
    for asked in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1)):
        out = [Tiles(da, BF16, replicas=1), Tiles(db, torch.float32, replicas=1), Tiles(db, torch.float32, replicas=1)]
        plan.gated_backward(binding.DMM_SILU, *(t.table() for t in (a, wg, wu, g, u, dh, dg, du)), *(t.table() if x else None for x, t in zip(asked, out)),
                            binding.DMM_DB_F32, stream())
        torch.cuda.synchronize()
        want = want or out
        for x, t, w, what in zip(asked, out, want, ("dA", "dWg", "dWu")):
            assert not x or torch.equal(t.whole(), w.whole()), (asked, what)
    for t, y in ((want[1], dg), (want[2], du)):
        close(t.whole(), a.whole().t() @ y.whole(), sum_error(a.whole().t(), y.whole()) + TINY, "a weight's gradient")


@pytest.mark.parametrize("name", list(ACTS))
def test_activations_of_every_number(name):
    """All finite bf16 numbers through the block (G = g, U = 1) and back (dH = 1): the function and its slope wherever these are.  Where the argument of the
    exponential is past 200 nothing is left of that in 64 bits of fp32's range, so that its error counts no further."""
    g = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(BF16)
    g = g[torch.isfinite(g)].reshape(-1, 1)
    m = len(g)
    (da, db, dc), ranks = descs("whole", m, 2, 1)
    plan = binding.Plan(da, db, dc, ranks)
    one = torch.ones(m, 1, dtype=BF16, device="cuda")
    x, w, v, d = Tiles(da, BF16, torch.cat((g, one), 1)), Tiles(db, BF16, torch.eye(2)[:, :1]), Tiles(db, BF16, torch.eye(2)[:, 1:]), Tiles(dc, BF16, one)
    h, kg, ku, dg, du = (Tiles(dc, BF16) for _ in range(5))
    plan.gated(ACTS[name], *(t.table() for t in (x, w, v, h, kg, ku)), stream=stream())
    plan.gated_backward(ACTS[name], None, None, None, *(t.table() for t in (kg, ku, d, dg, du)), stream=stream())
    torch.cuda.synchronize()
    G = g.double()
    value, slope = act(G, name)
    arg = argument(G, name).clamp(max=200)
    assert torch.equal(kg.whole(), G) and bool((ku.whole() == 1).all())
    limit = H * value.abs() + (1 + H) * value.abs() * (10 + 4 * arg) * U + TINY
    close(h.whole(), value, limit, "H")
    close(du.whole(), value, limit, "dU")
    close(dg.whole(), slope, H * slope.abs() + (1 + H) * 2 * (10 + 4 * arg) * U + TINY, "dG")
