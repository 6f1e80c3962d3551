"""Tile buffers for the tests of the layers around a product: guards around and between rows, whatever the cuts."""
import numpy as np
import torch

import workloads
from paper_2510_08874_amd import binding

ACTS = {"silu": binding.DMM_SILU, "gelu": binding.DMM_GELU, "gelu_tanh": binding.DMM_GELU_TANH}


def bounds(d, replicas=None):
    return [(r0, r1, c0, c1) for _ in range(d["replication"] if replicas is None else replicas)
            for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]) for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:])]


class Tiles:
    """The tiles of a matrix, each in an allocation of its own that ends with the tile's last element: `offset` elements in front, rows `more`
    elements longer than they have to be, all of that filled with NaN (integers: 77)."""

    def __init__(self, d, dtype, x=None, more=0, offset=0, replicas=None, turned=False):
        self.d, self.dtype, self.offset, self.turned = d, dtype, offset, turned
        self.bounds = bounds(d, replicas)
        self.fill = 77 if dtype == torch.int8 else float("nan")
        self.bufs, self.views, self.ld = [], [], []
        for r0, r1, c0, c1 in self.bounds:
            h, w = (c1 - c0, r1 - r0) if turned else (r1 - r0, c1 - c0)
            ld = max(w + more, 1)
            self.ld.append(ld)
            if h == 0 or w == 0:
                self.bufs.append(None)
                self.views.append(None)
                continue
            buf = torch.full((offset + (h - 1) * ld + w,), self.fill, dtype=dtype, device="cuda")
            view = torch.as_strided(buf, (h, w), (ld, 1), offset)
            if x is not None:
                t = x[r0:r1, c0:c1]
                view.copy_(t.t() if turned else t)
            self.bufs.append(buf)
            self.views.append(view)

    def table(self):
        return binding.tiles(self.views, self.ld)

    def whole(self, rep=0):
        """The matrix of one replica in 64 bits."""
        out = torch.zeros(self.d["rows"], self.d["cols"], dtype=torch.float64, device="cuda")
        n = len(bounds(self.d, 1))
        for (r0, r1, c0, c1), v in list(zip(self.bounds, self.views))[rep * n:(rep + 1) * n]:
            if v is not None:
                out[r0:r1, c0:c1] = (v.t() if self.turned else v).double()
        return out

    def check_guards(self):
        """Nothing but the tiles themselves has been written."""
        for buf, v in zip(self.bufs, self.views):
            if buf is None:
                continue
            kept = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
            torch.as_strided(kept, v.shape, v.stride(), self.offset).fill_(False)
            rest = buf[kept]
            assert bool((rest == 77).all() if self.dtype == torch.int8 else torch.isnan(rest).all()), "a guard was written"


class Int8:
    """A matrix in 8-bit integers along its rows or columns, with scales of every row (column) of tiles."""

    def __init__(self, d, along, q=None, s=None, more=0, offset=0):
        self.d, self.along = d, along
        self.q = Tiles(d, torch.int8, q, more, offset, turned=along == "cols")
        cuts = d["row_cuts"] if along == "rows" else d["col_cuts"]
        self.s = []
        for _ in range(d["replication"]):
            for i, j in zip(cuts, cuts[1:]):
                self.s.append(None if i == j else torch.full((j - i,), float("nan"), dtype=torch.float32, device="cuda") if s is None else s[i:j].clone())

    def table(self):
        return binding.int_tiles(self.q.views, self.q.ld, self.s)

    def scales(self, rep=0):
        n = len(self.s) // self.d["replication"]
        return torch.cat([t for t in self.s[rep * n:(rep + 1) * n] if t is not None])


def stream():
    return torch.cuda.current_stream().cuda_stream


def uneven(n, parts):
    """Cuts on no regular grid, an empty part among them where there are three and more."""
    cuts = [0] + sorted((n * (i * i + 2 * i) // (parts * parts + 2 * parts)) for i in range(1, parts)) + [n]
    if parts >= 3:
        cuts[2] = cuts[1]
    return cuts


def descs(layout, m, k, n):
    """A, B and C of a product, and the number of ranks."""
    D = workloads.desc
    if layout == "whole":
        return (D(m, k, [0, m], [0, k], 1, 1), D(k, n, [0, k], [0, n], 1, 1), D(m, n, [0, m], [0, n], 1, 1)), 1
    if layout == "blocks":
        return (workloads.block_desc(m, k, 2, 2), workloads.block_desc(k, n, 2, 2), workloads.block_desc(m, n, 2, 2)), 4
    if layout == "column":
        return (D(m, k, [0, m], [0, k], 1, 1, replication=4), workloads.block_desc(k, n, 1, 4), workloads.block_desc(m, n, 1, 4)), 4
    if layout == "uneven":
        return (D(m, k, uneven(m, 3), uneven(k, 4), 3, 4), D(k, n, uneven(k, 3), uneven(n, 2), 3, 2), D(m, n, uneven(m, 2), uneven(n, 3), 2, 3)), 12
    if layout == "row_col":
        return (workloads.block_desc(m, k, 8, 1), D(k, n, uneven(k, 3), uneven(n, 2), 3, 2), workloads.block_desc(m, n, 4, 2)), 8
    assert layout == "replicated"
    return tuple(workloads.block_desc(r, c, 2, 2, replication=2) for r, c in ((m, k), (k, n), (m, n))), 8


def normal(rows, cols, seed, scale=1.0, dtype=torch.bfloat16):
    """The same values on every device."""
    x = np.random.default_rng(seed).standard_normal((rows, cols), dtype=np.float32) * scale
    return torch.from_numpy(x).to("cuda").to(dtype)


def act(g, name):
    """act and its slope in 64 bits."""
    if name == "silu":
        s = torch.special.expit(g)
        return g * s, s + g * s * torch.special.expit(-g)
    if name == "gelu":
        p = torch.special.erfc(-g * 0.5 ** 0.5) / 2             # (torch.special.ndtr is 1 % off at -7.9, in 64 bits)
        return g * p, p + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    c = 2 * (2 / torch.pi) ** 0.5
    s = torch.special.expit(c * (g + 0.044715 * g ** 3))
    return g * s, s + g * s * (1 - s) * c * (1 + 3 * 0.044715 * g * g)
