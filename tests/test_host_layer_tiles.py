"""``IntTileSet``: its buffers and tables, and what ``quantize`` and ``write_values`` refuse with it.  Nothing here needs a GPU."""
import ctypes

import pytest

import workloads

torch = pytest.importorskip("torch")
from paper_2510_08874_amd.tiles import IntTileSet, MxTileSet, TileSet, quantize  # noqa: E402

D = workloads.desc(300, 520, [0, 100, 300], [0, 256, 256, 520], 2, 3, replication=2)
OTHERS = [dict(D, row_cuts=[0, 200, 300]), dict(D, col_cuts=[0, 256, 520]), dict(D, replication=1)]


@pytest.fixture
def addresses(monkeypatch):
    # (a meta tensor has none, and nothing gets as far as to use one)
    from paper_2510_08874_amd import binding
    monkeypatch.setattr(binding, "_ptr", lambda t: 0)


def read(p, ctype, n):
    return list(ctypes.cast(p, ctypes.POINTER(ctype))[:n])


@pytest.mark.parametrize("along", ["rows", "cols"])
def test_buffers(along):
    form = IntTileSet(D, along, device="cpu")
    shapes = [(100, 256), None, (100, 264), (200, 256), None, (200, 264)] * 2
    for t, s in zip(form.codes, shapes):
        if s is None:
            assert t is None
            continue
        n, k = s if along == "rows" else s[::-1]
        assert t.dtype == torch.int8 and t.shape[0] == n and k <= t.shape[1] < k + 16 and t.shape[1] % 16 == 0
    lengths = [100, 200] * 2 if along == "rows" else [256, 0, 264] * 2
    assert [0 if t is None else t.numel() for t in form.scales] == lengths and all(t is None or t.dtype == torch.float32 for t in form.scales)
    assert read(form.table.codes, ctypes.c_uint64, 12) == [0 if t is None else t.data_ptr() for t in form.codes]
    assert read(form.table.code_ld, ctypes.c_int64, 12) == [0 if t is None else t.shape[1] for t in form.codes]
    assert read(form.table.scales, ctypes.c_uint64, len(lengths)) == [0 if t is None else t.data_ptr() for t in form.scales]
    turned = form.transposed()                             # tile (j, i) of the transposed matrix
    order = [rep * 6 + i * 3 + j for rep in range(2) for j in range(3) for i in range(2)]
    assert read(turned.codes, ctypes.c_uint64, 12) == [0 if form.codes[x] is None else form.codes[x].data_ptr() for x in order]
    assert read(turned.code_ld, ctypes.c_int64, 12) == [0 if form.codes[x] is None else form.codes[x].shape[1] for x in order]
    assert read(turned.scales, ctypes.c_uint64, len(lengths)) == read(form.table.scales, ctypes.c_uint64, len(lengths))


def test_no_such_direction():
    with pytest.raises(ValueError, match="along"):
        IntTileSet(D, "columns", device="cpu")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8], ids=str)
def test_other_types(addresses, dtype):
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        quantize(TileSet(D, dtype, device="meta"), rows=IntTileSet(D, "rows", device="meta"))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        IntTileSet(D, "rows", device="meta").write_values(TileSet(D, dtype, device="meta"))


@pytest.mark.parametrize("other", range(len(OTHERS)))
@pytest.mark.parametrize("along", ["rows", "cols"])
def test_other_cuts(addresses, along, other):
    x, form = TileSet(D, torch.bfloat16, device="meta"), IntTileSet(OTHERS[other], along, device="meta")
    with pytest.raises(ValueError, match="cuts"):
        quantize(x, **{along: form})
    with pytest.raises(ValueError, match="cuts"):
        form.write_values(x)


def test_the_other_direction_and_device(addresses):
    x = TileSet(D, torch.float32, device="meta")
    with pytest.raises(ValueError, match="along"):
        quantize(x, rows=IntTileSet(D, "cols", device="meta"))
    with pytest.raises(ValueError, match="along"):
        quantize(x, cols=IntTileSet(D, "rows", device="meta"))
    with pytest.raises(ValueError, match="current device"):
        quantize(x, rows=IntTileSet(D, "rows", device="cpu"))
    with pytest.raises(ValueError, match="current device"):
        IntTileSet(D, "cols", device="cpu").write_values(x)


def test_two_kinds_of_forms(addresses, monkeypatch):
    from paper_2510_08874_amd import tiles
    monkeypatch.setattr(tiles, "_check_form", lambda *_: None)
    with pytest.raises(ValueError, match="two calls"):
        quantize(TileSet(D, torch.bfloat16, device="meta"), rows=IntTileSet(D, "rows", device="meta"), cols=MxTileSet(D, "cols", device="meta"))
