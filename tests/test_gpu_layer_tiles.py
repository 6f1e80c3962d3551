"""``IntTileSet`` on the GPU: matrices to integers and back, and the products on them, by the tables it makes."""
import numpy as np
import pytest
import torch

from paper_2510_08874_amd import binding
from paper_2510_08874_amd.tiles import IntTileSet, TileSet, quantize
from tests.layer_tiles import ACTS, act, descs

pytestmark = pytest.mark.gpu


def scale_of(X, axis):
    return (np.abs(X).max(axis=axis, keepdims=True) / np.float32(127)).astype(np.float64)


def whole(form):
    """Codes and scales of replica 0, in 64 bits."""
    d, n = form.desc, (len(form.desc["row_cuts"]) - 1) * (len(form.desc["col_cuts"]) - 1)
    out, x = np.zeros((d["rows"], d["cols"])), 0
    for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]):
        for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:]):
            if form.codes[x] is not None:
                t = form.codes[x].cpu().numpy()
                out[r0:r1, c0:c1] = t[:, :c1 - c0] if form.along == "rows" else t[:, :r1 - r0].T
            x += 1
    s = np.concatenate([t.cpu().numpy() for t in form.scales[:len(form.scales) // d["replication"]] if t is not None]).astype(np.float64)
    return out, s[:, None] if form.along == "rows" else s[None, :]


@pytest.mark.parametrize("layout", ["whole", "uneven", "replicated"])
def test_there_and_back_and_products(layout):
    (da, db, dc), ranks = descs(layout, 173, 309, 221)
    rng = np.random.default_rng(11)
    A, B = (rng.standard_normal((d["rows"], d["cols"]), dtype=np.float32) for d in (da, db))
    a, b = TileSet(da, torch.float32), TileSet(db, torch.float32)
    a.scatter(A)
    b.scatter(B)
    rows, cols, b_rows = IntTileSet(da, "rows"), IntTileSet(db, "cols"), IntTileSet(db, "rows")
    quantize(a, rows=rows)
    quantize(b, rows=b_rows, cols=cols)
    # back: half a step, and the roundings of the scale and of the value, each 2^-24 of at most 127 scales
    for x, form, axis in ((A, rows, 1), (B, cols, 0), (B, b_rows, 1)):
        back = TileSet(form.desc, torch.float32, fill=float("nan"))
        form.write_values(back)
        assert (np.abs(back.gather().astype(np.float64) - x) <= scale_of(x, axis) * (0.5 + 2 * 127 * 2.0 ** -24)).all()
    # the product: the sum is exact, its conversion and two multiplications round (with replicas of C: a sum of two such, and its rounding)
    (qa, sa), (qb, sb) = whole(rows), whole(cols)
    plan = binding.Plan(da, db, dc, ranks)
    out = TileSet(dc, torch.float32, fill=float("nan"))
    stream = torch.cuda.current_stream().cuda_stream
    plan.execute_int(rows.table, cols.table, binding.tiles(out.tensors, out.ld), 0, stream)
    want, size = qa @ qb * sa * sb, np.abs(qa) @ np.abs(qb) * sa * sb
    assert (np.abs(out.gather() - want) <= (size if dc["replication"] > 1 else np.abs(want)) * 5 * 2.0 ** -24).all()
    plan.destroy()
    if dc["replication"] > 1:
        return
    # X = A of the transposed right operand's integers: B^T in the order of its own tiles
    dt = dict(db, rows=db["cols"], cols=db["rows"], row_cuts=db["col_cuts"], col_cuts=db["row_cuts"], proc_rows=db["proc_cols"], proc_cols=db["proc_rows"])
    dat = dict(da, rows=da["cols"], cols=da["rows"], row_cuts=da["col_cuts"], col_cuts=da["row_cuts"], proc_rows=da["proc_cols"], proc_cols=da["proc_rows"])
    dct = dict(dc, rows=dc["cols"], cols=dc["rows"], row_cuts=dc["col_cuts"], col_cuts=dc["row_cuts"], proc_rows=dc["proc_cols"], proc_cols=dc["proc_rows"])
    plan = binding.Plan(dt, dat, dct, ranks)
    turned = TileSet(dct, torch.float32, fill=float("nan"))
    plan.execute_int(cols.transposed(), rows.transposed(), binding.tiles(turned.tensors, turned.ld), 0, stream)
    assert (np.abs(turned.gather() - want.T) <= np.abs(want.T) * 5 * 2.0 ** -24).all()
    plan.destroy()


def test_gated_on_integers():
    (da, db, dc), ranks = descs("blocks", 65, 320, 200)
    rng = np.random.default_rng(12)
    forms = []
    for d, along in ((da, "rows"), (db, "cols"), (db, "cols")):
        x, form = TileSet(d, torch.float32), IntTileSet(d, along)
        x.scatter(rng.standard_normal((d["rows"], d["cols"]), dtype=np.float32) / np.float32(1 if along == "rows" else 18))
        quantize(x, **{along: form})
        forms.append(form)
    h = TileSet(dc, torch.bfloat16, fill=float("nan"))
    plan = binding.Plan(da, db, dc, ranks)
    plan.gated_int(ACTS["silu"], *[f.table for f in forms], binding.tiles(h.tensors, h.ld), torch.cuda.current_stream().cuda_stream)
    (qa, sa), (qg, sg), (qu, su) = map(whole, forms)
    g, u = qa @ qg * sa * sg, qa @ qu * sa * su
    v, slope = (t.numpy() for t in act(torch.from_numpy(g), "silu"))
    # g and u: 3 roundings each; the activation some units (8 here) of its value; the product; bf16's half step
    bound = (np.abs(u * slope * g) * 3 + np.abs(v * u) * (3 + 8 + 1)) * 2.0 ** -24 * 1.01 + np.abs(v * u) * 2.0 ** -8 * 1.01 + 1e-30
    assert (np.abs(h.gather() - v * u) <= bound).all()
    plan.destroy()
