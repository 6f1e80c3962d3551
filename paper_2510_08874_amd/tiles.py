"""Tile buffers on the GPU: every (replica, tile) of a distributed matrix is its
own torch allocation, as every virtual rank's tile is its own HBM buffer.
Allocation, host<->device copies and slicing by cut points only."""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple, Union

import numpy as np
import torch


def _round_up(x: int, m: int) -> int:
    return ((x + m - 1) // m) * m


class TileSet:
    """All tiles of all replicas of one matrix, in the table order of the ABI:
    ``rep * (grid_rows * grid_cols) + ti * grid_cols + tj``."""

    def __init__(self, desc: Dict, torch_dtype, device="cuda", ld_multiple: int = 1, fill: Optional[float] = None):
        self.desc = desc
        self.dtype = torch_dtype
        rc, cc = desc["row_cuts"], desc["col_cuts"]
        self.gr, self.gc = len(rc) - 1, len(cc) - 1
        self.tensors: List[Optional[torch.Tensor]] = []
        self.ld: List[int] = []
        for rep in range(desc["replication"]):
            for ti in range(self.gr):
                for tj in range(self.gc):
                    h, w = rc[ti + 1] - rc[ti], cc[tj + 1] - cc[tj]
                    ld = max(_round_up(w, ld_multiple), 1)
                    self.ld.append(ld)
                    if h == 0 or w == 0:
                        self.tensors.append(None)
                        continue
                    t = torch.empty((h, ld), dtype=torch_dtype, device=device)
                    if fill is not None:
                        t.fill_(fill)
                    self.tensors.append(t)

    def index(self, rep: int, ti: int, tj: int) -> int:
        return rep * self.gr * self.gc + ti * self.gc + tj

    def bounds(self, ti: int, tj: int) -> Tuple[int, int, int, int]:
        rc, cc = self.desc["row_cuts"], self.desc["col_cuts"]
        return rc[ti], rc[ti + 1], cc[tj], cc[tj + 1]

    def scatter(self, X: np.ndarray) -> None:
        """Copy a global host matrix into every replica's tiles.  ``X`` is
        float32, or uint16 bf16 bit patterns when the tiles are bfloat16."""
        if self.dtype == torch.bfloat16:
            host = torch.from_numpy(X.view(np.int16)).view(torch.bfloat16)
        else:
            host = torch.from_numpy(X)
        for ti in range(self.gr):
            for tj in range(self.gc):
                r0, r1, c0, c1 = self.bounds(ti, tj)
                if r1 == r0 or c1 == c0:
                    continue
                dev = host[r0:r1, c0:c1].contiguous().to(self.tensors[self.index(0, ti, tj)].device)
                for rep in range(self.desc["replication"]):
                    self.tensors[self.index(rep, ti, tj)][:, :c1 - c0].copy_(dev)

    def gather(self, rep: int = 0) -> np.ndarray:
        """Global host matrix assembled from one replica's tiles (float32)."""
        out = np.zeros((self.desc["rows"], self.desc["cols"]), dtype=np.float32)
        for ti in range(self.gr):
            for tj in range(self.gc):
                r0, r1, c0, c1 = self.bounds(ti, tj)
                if r1 == r0 or c1 == c0:
                    continue
                out[r0:r1, c0:c1] = self.tensors[self.index(rep, ti, tj)][:, :c1 - c0].float().cpu().numpy()
        return out

    def gather_rows(self, rows: np.ndarray, rep: int = 0) -> np.ndarray:
        """Selected global rows (all columns) from one replica's tiles."""
        rows = np.asarray(rows)
        out = np.zeros((len(rows), self.desc["cols"]), dtype=np.float32)
        rc = self.desc["row_cuts"]
        for ti in range(self.gr):
            sel = np.nonzero((rows >= rc[ti]) & (rows < rc[ti + 1]))[0]
            if len(sel) == 0:
                continue
            local = torch.as_tensor(rows[sel] - rc[ti], device="cpu")
            for tj in range(self.gc):
                r0, r1, c0, c1 = self.bounds(ti, tj)
                if c1 == c0:
                    continue
                t = self.tensors[self.index(rep, ti, tj)]
                out[sel, c0:c1] = t[local.to(t.device), :c1 - c0].float().cpu().numpy()
        return out

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self.tensors if t is not None)


class MxTileSet:
    """The tiles of a matrix in 4 bits, along its rows or along its columns: codes and scales of every tile, in the
    table order of the ABI.  ``table`` goes to ``dmm_mx_quantize``, ``dmm_mx_dequantize`` and ``Plan.execute_mx``."""

    def __init__(self, desc: Dict, along: str, device="cuda"):
        from . import binding
        if along not in ("rows", "cols"):
            raise ValueError(f"along: {along!r}, not 'rows' or 'cols'")
        self.desc, self.along, self.binding = desc, along, binding
        self.codes: List[Optional[torch.Tensor]] = []
        self.scales: List[Optional[torch.Tensor]] = []
        rc, cc = desc["row_cuts"], desc["col_cuts"]
        for _ in range(desc["replication"]):
            for r0, r1 in zip(rc, rc[1:]):
                for c0, c1 in zip(cc, cc[1:]):
                    n, k = (r1 - r0, c1 - c0) if along == "rows" else (c1 - c0, r1 - r0)
                    chunks = _round_up(k, binding.DMM_MX_CHUNK) // binding.DMM_MX_CHUNK
                    for made, size in ((self.codes, binding.DMM_MX_CHUNK // 2), (self.scales, binding.DMM_MX_CHUNK // binding.DMM_MX_BLOCK)):
                        made.append(torch.empty((n, chunks * size), dtype=torch.uint8, device=device) if n and k else None)
        self.table = self._table(range(len(self.codes)))

    def _table(self, order):
        def columns(made):
            return [made[i] for i in order], [0 if made[i] is None else made[i].shape[1] for i in order]
        order = list(order)
        return self.binding.mx_tiles(*columns(self.codes), *columns(self.scales))

    def transposed(self):
        """The table of the transposed matrix, whose rows are this one's columns: the same buffers in another order."""
        gr, gc = len(self.desc["row_cuts"]) - 1, len(self.desc["col_cuts"]) - 1
        return self._table(rep * gr * gc + i * gc + j for rep in range(self.desc["replication"]) for j in range(gc) for i in range(gr))

    def write_values(self, X: TileSet, stream: Optional[int] = None) -> None:
        """The values that the codes stand for, into the tiles of ``X`` (bf16 or fp32)."""
        b = self.binding
        _check_form(X, self, self.along)
        b.dmm_mx_dequantize(b.matrix_desc(self.desc), self.table, b.DMM_MX_ROWS if self.along == "rows" else b.DMM_MX_COLS,
                            b.DMM_BF16 if X.dtype == torch.bfloat16 else b.DMM_F32, b.tile_table(X.tensors, X.ld),
                            torch.cuda.current_stream().cuda_stream if stream is None else stream)


class IntTileSet:
    """The tiles of a matrix in 8-bit integers, along its rows or along its columns: codes of every tile and scales of every row (column) of tiles, in
    the table order of the ABI.  ``table`` goes to ``dmm_int_quantize``, ``dmm_int_dequantize``, ``Plan.execute_int`` and ``Plan.gated_int``."""

    def __init__(self, desc: Dict, along: str, device="cuda"):
        from . import binding
        if along not in ("rows", "cols"):
            raise ValueError(f"along: {along!r}, not 'rows' or 'cols'")
        self.desc, self.along, self.binding = desc, along, binding
        self.codes: List[Optional[torch.Tensor]] = []
        self.scales: List[Optional[torch.Tensor]] = []
        rc, cc = desc["row_cuts"], desc["col_cuts"]
        for _ in range(desc["replication"]):
            for r0, r1 in zip(rc, rc[1:]):
                for c0, c1 in zip(cc, cc[1:]):
                    n, k = (r1 - r0, c1 - c0) if along == "rows" else (c1 - c0, r1 - r0)
                    self.codes.append(torch.empty((n, _round_up(k, 16)), dtype=torch.int8, device=device) if n and k else None)
            cuts = rc if along == "rows" else cc
            for i, j in zip(cuts, cuts[1:]):
                self.scales.append(torch.empty(j - i, dtype=torch.float32, device=device) if j > i else None)
        self.table = self._table(range(len(self.codes)))

    def _table(self, order):
        order = list(order)
        return self.binding.int_tiles([self.codes[i] for i in order], [0 if self.codes[i] is None else self.codes[i].shape[1] for i in order], self.scales)

    def transposed(self):
        """The table of the transposed matrix, whose rows are this one's columns: the same buffers, the codes in another order."""
        gr, gc = len(self.desc["row_cuts"]) - 1, len(self.desc["col_cuts"]) - 1
        return self._table(rep * gr * gc + i * gc + j for rep in range(self.desc["replication"]) for j in range(gc) for i in range(gr))

    def write_values(self, X: TileSet, stream: Optional[int] = None) -> None:
        """The values that the integers stand for, into the tiles of ``X`` (bf16 or fp32)."""
        b = self.binding
        _check_form(X, self, self.along)
        b.dmm_int_dequantize(b.matrix_desc(self.desc), self.table, b.DMM_MX_ROWS if self.along == "rows" else b.DMM_MX_COLS,
                             b.DMM_BF16 if X.dtype == torch.bfloat16 else b.DMM_F32, b.tiles(X.tensors, X.ld),
                             torch.cuda.current_stream().cuda_stream if stream is None else stream)


def _check_form(X: TileSet, form: Union[MxTileSet, IntTileSet], along: str) -> None:
    """The library gets addresses alone: tiles and a form that do not belong together would be read or written out of range."""
    if X.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"tiles of {X.dtype}, not of bfloat16 or float32")
    if form.along != along:
        raise ValueError(f"a form along the {form.along} where one along the {along} is meant")
    a, b = X.desc, form.desc
    if a["replication"] != b["replication"] or any(tuple(a[c]) != tuple(b[c]) for c in ("row_cuts", "col_cuts")):
        raise ValueError("the tiles and the form have different cuts or replicas")
    for device in {t.device for t in (*X.tensors, *form.codes, *form.scales) if t is not None}:
        if device.type != "cuda" or device.index != torch.cuda.current_device():
            raise ValueError(f"tiles on {device}, not on the current device")


def quantize(X: TileSet, rows: Union[MxTileSet, IntTileSet, None] = None, cols: Union[MxTileSet, IntTileSet, None] = None,
             stream: Optional[int] = None) -> None:
    """``dmm_mx_quantize`` or, into an ``IntTileSet``, ``dmm_int_quantize`` of the tiles of ``X`` along their rows, their columns or both."""
    from . import binding as b
    for form, along in ((rows, "rows"), (cols, "cols")):
        if form is not None:
            _check_form(X, form, along)
    kinds = {type(form) for form in (rows, cols) if form is not None}
    if len(kinds) > 1:
        raise ValueError("one form in 4 bits and one in 8-bit integers: two calls")
    desc, dtype, forms = b.matrix_desc(X.desc), b.DMM_BF16 if X.dtype == torch.bfloat16 else b.DMM_F32, dict(rows=rows and rows.table, cols=cols and cols.table)
    on = torch.cuda.current_stream().cuda_stream if stream is None else stream
    if kinds == {IntTileSet}:
        b.dmm_int_quantize(desc, dtype, b.tiles(X.tensors, X.ld), **forms, stream=on)
    else:
        b.dmm_mx_quantize(desc, dtype, b.tile_table(X.tensors, X.ld), **forms, stream=on)


class DeviceProblem:
    """One partitioned product resident on the GPU: the plan, the three tile
    sets and the marshalled argument arrays of ``dmm_execute``."""

    def __init__(self, cfg: Dict, A_host: Optional[np.ndarray] = None, B_host: Optional[np.ndarray] = None,
                 ld_multiple: int = 1, c_fill: Optional[float] = None, device="cuda", c_dtype: str = "f32"):
        from . import binding
        self.cfg = cfg
        self.binding = binding
        self.dtype_code = binding.DMM_BF16 if cfg["dtype"] == "bf16" else binding.DMM_F32
        tdt = torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32
        self.plan = binding.Plan(cfg["A"], cfg["B"], cfg["C"], cfg["nranks"],
                                 binding.STATIONARY_FLAGS[cfg.get("stationary", "C")] |
                                 (binding.DMM_ITERATION_OFFSET if cfg.get("iteration_offset") else 0) |
                                 (binding.DMM_MERGE_ALWAYS if cfg.get("merge_always") else 0))
        self.A = TileSet(cfg["A"], tdt, device, ld_multiple)
        self.B = TileSet(cfg["B"], tdt, device, ld_multiple)
        # C tiles are fp32, or bf16 when asked for (DMM_C_BF16 then goes with every execute)
        self.c_flags = binding.DMM_C_BF16 if c_dtype == "bf16" else 0
        self.C = TileSet(cfg["C"], torch.bfloat16 if c_dtype == "bf16" else torch.float32, device, ld_multiple,
                         fill=c_fill)
        if A_host is not None:
            self.A.scatter(A_host)
        if B_host is not None:
            self.B.scatter(B_host)
        self.args = self.plan.marshal(self.A.tensors, self.A.ld, self.B.tensors, self.B.ld,
                                      self.C.tensors, self.C.ld)

    def execute(self, flags: int = 0, stream: Optional[int] = None) -> None:
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self.plan.execute_marshalled(self.dtype_code, self.args, flags | self.c_flags, stream)

    def reduce(self, origin: int = 0, stream: Optional[int] = None) -> None:
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self.plan.reduce_replicas(self.C.tensors, self.C.ld, origin, stream)

    def broadcast(self, origin: int = 0, stream: Optional[int] = None) -> None:
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self.plan.broadcast_replica(self.C.tensors, self.C.ld, origin, stream)

    def c_global(self, rep: int = 0) -> np.ndarray:
        torch.cuda.synchronize()
        return self.C.gather(rep)

    def close(self) -> None:
        torch.cuda.synchronize()
        self.plan.destroy()
