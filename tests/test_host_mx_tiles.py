"""What ``quantize`` and ``MxTileSet.write_values`` refuse: tiles and forms of other types, cuts, directions or devices would be
read and written out of range.  Nothing here needs a GPU."""
import pytest

import workloads

torch = pytest.importorskip("torch")
from paper_2510_08874_amd.tiles import MxTileSet, TileSet, quantize  # noqa: E402

D = workloads.desc(300, 520, [0, 100, 300], [0, 256, 520], 2, 2)
OTHERS = [workloads.desc(300, 520, [0, 100, 300], [0, 520], 2, 1), workloads.desc(300, 520, [0, 200, 300], [0, 256, 520], 2, 2),
          workloads.desc(300, 520, [0, 100, 300], [0, 256, 520], 2, 2, replication=2), workloads.desc(100, 520, [0, 50, 100], [0, 256, 520], 2, 2)]


def tiles(d=D, dtype=torch.bfloat16, device="meta"):
    return TileSet(d, dtype, device=device)


def form(d=D, along="rows", device="meta"):
    return MxTileSet(d, along, device=device)


@pytest.fixture(autouse=True)
def addresses(monkeypatch):
    # (a meta tensor has none, and nothing gets as far as to use one)
    from paper_2510_08874_amd import binding
    monkeypatch.setattr(binding, "_ptr", lambda t: 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int16], ids=str)
def test_other_types(dtype):
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        quantize(tiles(dtype=dtype), rows=form())
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        form().write_values(tiles(dtype=dtype))


@pytest.mark.parametrize("other", range(len(OTHERS)))
def test_other_cuts(other):
    for along in ("rows", "cols"):
        with pytest.raises(ValueError, match="cuts"):
            quantize(tiles(), **{along: form(OTHERS[other], along)})
        with pytest.raises(ValueError, match="cuts"):
            form(OTHERS[other], along).write_values(tiles())


def test_the_other_direction():
    with pytest.raises(ValueError, match="along"):
        quantize(tiles(), rows=form(along="cols"))
    with pytest.raises(ValueError, match="along"):
        quantize(tiles(), cols=form(along="rows"))


def test_other_devices():
    for x, q in (("cpu", "cpu"), ("meta", "cpu"), ("cpu", "meta")):
        with pytest.raises(ValueError, match="current device"):
            quantize(tiles(device=x), rows=form(device=q))
        with pytest.raises(ValueError, match="current device"):
            form(device=q).write_values(tiles(device=x))
