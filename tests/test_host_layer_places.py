"""Which elements the products around a layer multiply, without a GPU: scenarios on the stand-in for the HIP runtime, as in test_host_layer.py, every one
in a process of its own.  Each address that a work table names, in a tile or in a copy of one, is taken back to the row and column of its matrix: both
operands of a product have to be at the same k, and every k of a result counts once."""
import ctypes
import os
import random
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workloads  # noqa: E402
from tests.test_host_calls import Recorder, recorder  # noqa: E402, F401
from tests.test_host_layer import COPY, ITEM, JOIN, KINDS, PRODUCTS, SEG, Space, bounds, layouts, made  # noqa: E402

ZERO = -1                                                      # where a copy was filled up
STORE, PARTS, NOTHING = range(3)                               # what becomes of a macro-tile (NOTHING: zeros, there is no k)
# of a product's operands: which come together, and the results they may go into
PAIRS = {("a", "w"): ("c", "h"), ("dg", "w"): ("ga",), ("du", "v"): ("ga",), ("a", "dg"): ("gw",), ("a", "du"): ("gv",)}


class Ground(Space):
    """Buffers that know which tile of which matrix they are.  Along K everything has bytes of a row in one piece, or rows at one pitch."""

    def __init__(self, aligned=False):
        super().__init__(aligned)
        self.names, self.tile = [], []                         # of every buffer: name; first row, first column, leading dimension, bytes, transposed
        self.arrays = None

    def know(self, name, r0, c0, ld, es, turned):
        self.names.append(name)
        self.tile.append((r0, c0, ld, es, turned))
        assert len(self.names) == len(self.start)
        self.arrays = None

    def bf(self, name, d, es=2, more=0, replicas=None, turned=False):
        from paper_2510_08874_amd import binding as b
        ptr, ld = [], []
        for r0, r1, c0, c1 in bounds(d, d["replication"] if replicas is None else replicas):
            h, w = (c1 - c0, r1 - r0) if turned else (r1 - r0, c1 - c0)
            ld.append(max(w + more, 1))
            ptr.append(self.take(((h - 1) * ld[-1] + w) * es, es) if h and w else None)
            if ptr[-1]:
                self.know(name, r0, c0, ld[-1], es, turned)
        self.last = ptr, ld
        return b.tiles(ptr, ld)

    def ints(self, name, d, along, more=0):
        from paper_2510_08874_amd import binding as b
        self.bf(name, d, 1, more, turned=along == "cols")
        cuts, scales = d["row_cuts"] if along == "rows" else d["col_cuts"], []
        for _ in range(d["replication"]):
            for i, j in zip(cuts, cuts[1:]):
                scales.append(self.take(4 * (j - i), 4) if j > i else None)
                if j > i:
                    self.know(name + " scale", i, 0, 1, 4, False)
        return b.int_tiles(*self.last, scales)

    def find(self, at):
        """Names, rows and columns of the addresses `at`."""
        if self.arrays is None:
            self.arrays = [np.array(x, dtype=np.int64) for x in (self.start, self.end, self.tile)]
        at, (start, end, tile) = np.asarray(at, dtype=np.int64), self.arrays
        i = np.searchsorted(start, at, side="right") - 1
        assert (i >= 0).all() and (at < end[i]).all(), "an address that lies in no tile"
        r0, c0, ld, es, turned = tile[i].T
        off = at - start[i]
        assert (off % es == 0).all()
        r, c = off // es // ld, off // es % ld
        return {self.names[x] for x in np.unique(i)}, r0 + np.where(turned, c, r), c0 + np.where(turned, r, c)


class Call:
    """A call's launches: what each macro-tile multiplies, and where that goes."""

    def __init__(self, rec, space, at):
        self.rec, self.space, self.front, self.back = rec, space, [], []
        self.sums = {}                                         # result, row, column -> k's of every partial sum, in the order they are added in
        ops, multiplied = rec.launches(at), False
        for op in ops:
            if op[1] == "layer_copy_kernel":
                (self.back if multiplied else self.front).extend(self.jobs(op))
            multiplied = multiplied or op[1] in PRODUCTS
        self.lows = np.array([j[1] for j in self.front])
        self.highs = np.array([j[1] + (j[4] - 1) * j[3] + j[5] for j in self.front])
        for x, op in enumerate(ops):
            if op[1] in PRODUCTS:
                self.launch(op, ops[x + 1][3] if x + 1 < len(ops) and ops[x + 1][1] == "layer_join_kernel" else None)

    def jobs(self, op):
        blocks, x = 0, 0
        while blocks < self.rec.so.rec_blocks(op[0]):
            job = COPY.unpack(ctypes.string_at(op[3] + x * COPY.size, COPY.size))
            yield job[:6]
            blocks += -(-(-(-job[5] // 16) * job[4]) // 2048)
            x += 1

    def source(self, at):
        """Where what lies at the addresses `at` comes from: there, from where it was copied, or ZERO."""
        out, known = at.copy(), np.zeros(len(at), dtype=bool)
        if not self.front:
            return out
        low, high = at.min(), at.max()
        for x in np.flatnonzero((self.lows <= high) & (self.highs > low)):
            src, dst, src_pitch, dst_pitch, rows, size = self.front[x]
            off = at - dst
            r, c = (off // dst_pitch, off % dst_pitch) if dst_pitch else (0 * off, off)
            here = (off >= 0) & (r < rows) & (c < size)
            assert not (here & known).any(), "two copies in one place"
            known |= here
            out[here] = src + r[here] * src_pitch + c[here] if src else ZERO
        return out

    def line(self, p, pitch, turned, es, other, k0, n):
        """An operand at its row (column) `other`, n of its k's from k0 on: name, the row (column) in its matrix, k's (ZERO where there is none)."""
        ks = np.arange(k0, k0 + n, dtype=np.int64)
        at = self.source(p + (ks * pitch + other * es if turned else other * pitch + ks * es))
        there = at != ZERO
        k, name, row = np.full(n, ZERO), None, None
        if there.any():
            names, r, c = self.space.find(at[there])
            assert len(names) == 1, names
            name = names.pop()
            # (of A and dC along n the columns are k, of B the rows; across m the other way round)
            k_is_row = name in ("w", "v") and not self.nt or turned and self.tn
            k[there] = r if k_is_row else c
            rows = np.unique(c if k_is_row else r)
            assert len(rows) == 1, "one row of an operand from several of its matrix'"
            row = int(rows[0])
        return name, row, k

    def launch(self, op, joins):
        i, _, _, items, _ = op
        n = int(self.rec.so.rec_blocks(i))
        segs = items + n * ITEM.size
        parts = {}
        for x in range(n):
            v = ITEM.unpack(ctypes.string_at(items + x * ITEM.size, ITEM.size))
            front, (c, ldc, g, u, ldg, ldu, sa, sb, sb2), (m_off, n_off, m_ext, n_ext, seg, n_segs, first, steps, tail_seg, n_tails, c_es, what, kind, _) = v[:9], v[9:18], v[18:]
            kind = list(KINDS)[kind]
            self.nt, self.tn = kind == "nt", kind == "tn"
            a_turned, b_turned, dual, es = KINDS[kind]
            step = 128 // es
            pieces, left, s, skip = [], steps, 0, first        # segment, k's from ... on, how many
            while left > 0:
                assert s < n_segs
                q = front if s == 0 else self.segment(segs, seg + s)
                here = min(left, q[6] - skip)
                pieces.append((q, skip * step, here * step))
                left, s, skip = left - here, s + 1, 0
            for y in range(n_tails):
                q = self.segment(segs, tail_seg + y)
                pieces.append((q, q[6] * step, q[7]))
            corners = {}
            for dm, dn in {(0, 0), (m_ext - 1, n_ext - 1)}:
                got = []
                for q, k0, size in pieces:
                    if size == 0:
                        continue
                    name_a, row, ka = self.line(q[0], q[3], a_turned, es, m_off + dm, k0, size)
                    names = []
                    for p, pitch, want in ((q[1], q[4], "w"),) + (((q[2], q[5], "v"),) if dual else ()):
                        name, col, k = self.line(p, pitch, b_turned, es, n_off + dn, k0, size)
                        assert (k == ka).all(), (kind, "operands at different k")
                        assert not dual or name == want
                        names.append((name, col))
                    if name_a is None:                         # (zeros on both sides)
                        continue
                    assert len({col for _, col in names}) == 1
                    got.append(((name_a, names[0][0]), row, names[0][1], ka[ka != ZERO]))
                assert len({(pair, r, q) for pair, r, q, _ in got}) <= 2 and len({(r, q) for _, r, q, _ in got}) <= 1
                corners[dm, dn] = got
            scales = None
            if es == 1 and what == STORE:
                scales = self.scales(sa, sb, sb2, dual, m_ext, n_ext)
            if what == PARTS:
                parts[c] = corners
            else:
                self.result({at: [of] for at, of in corners.items()}, c, ldc, c_es, g, ldg, u, ldu, scales)
        slots, y = set(parts), 0
        while slots:
            c, ldc, g, u, ldg, ldu, sa, sb, sb2, p, runs, tm, tn, m_ext, n_ext, c_es = JOIN.unpack(ctypes.string_at(joins + y * JOIN.size, JOIN.size))
            all_of = [parts[p + r * tm * tn * 4] for r in range(runs)]
            slots -= {p + r * tm * tn * 4 for r in range(runs)}
            corners = {at: [of[at] for of in all_of] for at in all_of[0]}
            scales = self.scales(sa, sb, sb2, KINDS[kind][2], m_ext, n_ext) if KINDS[kind][3] == 1 else None
            self.result(corners, c, ldc, c_es, g, ldg, u, ldu, scales)
            y += 1

    def segment(self, segs, x):
        return SEG.unpack(ctypes.string_at(segs + x * SEG.size, SEG.size))

    def scales(self, sa, sb, sb2, dual, m_ext, n_ext):
        """First and last row and column that the scales of a macro-tile belong to."""
        out = []
        for p, ext, name in ((sa, m_ext, "a scale"), (sb, n_ext, "w scale")) + (((sb2, n_ext, "v scale"),) if dual else ()):
            at = self.source(p + 4 * np.array([0, ext - 1], dtype=np.int64))
            names, r, _ = self.space.find(at)
            assert names == {name}, names
            out.append(r.tolist())
        assert out[1] == out[-1]
        return out[:2]

    def target(self, at, es):
        """Name, row and column of a result's element, through its way out of scratch memory."""
        for src, dst, src_pitch, dst_pitch, rows, size in self.back:
            r, c = divmod(at - src, src_pitch)
            if 0 <= r < rows and c < size:
                at = dst + r * dst_pitch + c
                break
        names, r, c = self.space.find([at])
        return names.pop(), int(r[0]), int(c[0])

    def result(self, corners, c, ldc, c_es, g, ldg, u, ldu, scales):
        for (dm, dn), runs in corners.items():
            name, row, col = self.target(c + (dm * ldc + dn) * c_es, c_es)
            for p, ld, kept in ((g, ldg, "g"), (u, ldu, "u")):
                if p and name == "h":
                    assert self.target(p + (dm * ld + dn) * 2, 2) == (kept, row, col)
            seen = {}
            self.sums[name, row, col] = [[(pair, tuple(k.tolist())) for pair, _, _, k in got] for got in runs]
            for pair, r, q, k in (x for got in runs for x in got):
                assert name in PAIRS[pair], (pair, name)
                assert (r, q) == (row, col), ("the product of another row or column", pair, (r, q), (row, col))
                seen.setdefault(pair, []).append(k)
            want = {"c": [("a", "w")], "h": [("a", "w")], "ga": [("dg", "w"), ("du", "v")], "gw": [("a", "dg")], "gv": [("a", "du")]}[name]
            for pair in want[:self.pairs if name == "ga" else 1]:
                k = np.sort(np.concatenate(seen.pop(pair))) if pair in seen else np.zeros(0)
                assert np.array_equal(k, np.arange(self.depth[name])), (name, pair, "every k once", len(k), self.depth[name])
            assert not seen
            if scales:
                assert (scales[0][dm > 0], scales[1][dn > 0]) == (row, col)

    depth, pairs = {}, 2


def check(rec, space, call, depth, pairs=2):
    at = len(rec.ops())
    call()
    Call.depth, Call.pairs = depth, pairs
    return Call(rec, space, at)


def every_call(rec, d, ranks, more=0, aligned=False, integers=True, gated=True, backward=True):
    """All products on these cuts, with everything they can be asked for."""
    from paper_2510_08874_amd import binding as b
    da, db, dc = d
    m, k, n = da["rows"], da["cols"], db["cols"]
    plan, out = b.Plan(*d, ranks), []
    if integers:
        s = Ground(aligned)
        a, w, v = s.ints("a", da, "rows", more), s.ints("w", db, "cols", more), s.ints("v", db, "cols", more + 2)
        c, h = s.bf("c", dc, 4, more), s.bf("h", dc, 2, more)
        out.append(check(rec, s, lambda: plan.execute_int(a, w, c, 0, 0), dict(c=k)))
        out.append(check(rec, s, lambda: plan.gated_int(b.DMM_SILU, a, w, v, h, 0), dict(h=k)))
    s = Ground(aligned)
    a, w, v = s.bf("a", da, 2, more), s.bf("w", db, 2, more), s.bf("v", db, 2, more + 2)
    h, g, u = s.bf("h", dc, 2, more), s.bf("g", dc, 2, more), s.bf("u", dc, 2, more + 1)
    for kept in ((None, None), (g, u)) if gated else ():
        out.append(check(rec, s, lambda: plan.gated(b.DMM_GELU, a, w, v, h, *kept, 0), dict(h=k)))
    if backward:
        dg, du, ga, gw, gv = s.bf("dg", dc, 2, more), s.bf("du", dc, 2, more + 1), s.bf("ga", da, 2, more, 1), s.bf("gw", db, 4, more, 1), s.bf("gv", db, 4, more, 1)
        depth = dict(ga=n, gw=m, gv=m)
        for x in ((ga, gw, gv), (ga, None, None), (None, gw, None), (None, None, gv), (ga, None, gv)):
            out.append(check(rec, s, lambda: plan.gated_backward(b.DMM_GELU, a, w, v, g, u, h, dg, du, *x, b.DMM_DB_F32, 0), depth))
        for x in ((ga, gw), (ga, None), (None, gw)):
            out.append(check(rec, s, lambda: plan.execute_backward(a, w, dg, *x, b.DMM_DB_F32, 0), depth, 1))
    plan.destroy()
    return out


def operands_meet_at_the_same_k(rec):
    """Random sizes, cuts and leading dimensions."""
    rng = random.Random(23)
    copied = 0
    for turn in range(24):
        m, k, n = (max(15, rng.choice((rng.randint(15, 300), rng.randint(15, 1200), 64 * rng.randint(1, 16)))) for _ in range(3))
        if turn % 4 == 0:
            m = rng.randint(15, 64)
        d, ranks = layouts(rng, m, k, n)
        copied += any(c.front for c in every_call(rec, d, ranks, rng.choice((0, 0, 1, 3, 8)), turn % 2 == 0))
    assert copied > 5
    every_call(rec, made("whole", 40, 140100, 30), 1, backward=False, gated=False)   # (integer sums in several runs)
    every_call(rec, made("whole", 40, 8192, 300), 1)
    every_call(rec, made("row_col", 9, 2000, 12001), 12)
    every_call(rec, made("uneven", 1301, 1103, 907), 12)


def narrow_tiles_of_weights_on_a_copy_of_the_rows(rec):
    """A weight's last tile has one to three columns, so that a read of eight runs over rows that whole steps do not have behind them, and these rows are
    multiplied behind the steps: with the left operand's columns there, in a copy as anywhere else."""
    took = 0
    for m, blocks, k, n, last in ((8, 8, 4097, 8195, 3), (8, 4, 4097, 8195, 3), (8, 1, 4097, 8195, 3), (8, 8, 4098, 8194, 2), (8, 2, 4102, 8193, 1), (8, 8, 4160, 8193, 1),
                                  (64, 8, 8193, 8195, 3), (8, 8, 4097, 16387, 3)):
        d = (workloads.block_desc(m, k, 8, 1), workloads.desc(k, n, [0, k], [0, n - last, n], 1, 2), workloads.block_desc(m, n, blocks, 1))
        took += all(c.front for c in every_call(rec, d, 8, integers=False, backward=False))
        d = (d[0], workloads.desc(k, n, [0, 1025, k], [0, n - last, n], 2, 2), d[2])
        took += all(c.front for c in every_call(rec, d, 8, integers=False, backward=False))
    assert took >= 8


def gradients_are_summed_alike_whatever_else_is_asked_for(rec):
    """The k's of a gradient come in the same order and in the same partial sums, whichever of the others are asked for as well."""
    from paper_2510_08874_amd import binding as b
    rng = random.Random(5)
    cases = [(made("whole", *x), 1, 0) for x in ((4096, 1024, 1024), (8192, 512, 768), (8192, 1024, 3072), (2048, 256, 512), (1111, 300, 500), (40, 300, 500), (9000, 130, 65))]
    cases += [(made("uneven", 1301, 1103, 907), 12, 0), (made("uneven", 2500, 300, 400), 12, 1), (made("blocks", 3000, 256, 384), 4, 0)]
    for _ in range(6):
        cases.append((*layouts(rng, 64 * rng.randint(1, 40), 64 * rng.randint(1, 12), 64 * rng.randint(1, 12)), rng.choice((0, 1, 8))))
    cut = 0
    for d, ranks, more in cases:
        da, db, dc = d
        plan, s = b.Plan(*d, ranks), Ground(True)
        a, w, v = s.bf("a", da, 2, more), s.bf("w", db, 2, more), s.bf("v", db, 2, more)
        h, g, u = (s.bf("h", dc, 2, more) for _ in range(3))
        ga, gw, gv = s.bf("ga", da, 2, more, 1), s.bf("gw", db, 4, more, 1), s.bf("gv", db, 4, more + 1, 1)
        for of in ((0, 0), (0, 1), (1, 0)):                    # rows of dG and dU: as long as each other, or not
            dg, du = s.bf("dg", dc, 2, more + of[0]), s.bf("du", dc, 2, more + of[1])
            depth, got = dict(ga=db["cols"], gw=da["rows"], gv=da["rows"]), []
            for x in ((ga, gw, gv), (ga, None, None), (None, gw, None), (None, None, gv), (ga, None, gv), (None, gw, gv)):
                got.append(check(rec, s, lambda: plan.gated_backward(b.DMM_SILU, a, w, v, g, u, h, dg, du, *x, b.DMM_DB_F32, 0), depth).sums)
            for one in got[1:]:
                both = set(one) & set(got[0])
                assert {name for name, _, _ in both} == {name for name, _, _ in one}
                assert all(one[x] == got[0][x] for x in both), [(x, [len(r) for r in one[x]], [len(r) for r in got[0][x]]) for x in both if one[x] != got[0][x]][:3]
            cut += any(len(runs) > 1 for (name, _, _), runs in got[0].items() if name != "ga")
        plan.destroy()
    assert cut > 5


def without_memory_for_copies_each_gradient_has_its_own_macro_tiles(rec):
    """Both gradients in one launch on copies; without room for these, in two launches, on the tiles that each gets alone."""
    from paper_2510_08874_amd import binding as b
    D, block = workloads.desc, workloads.block_desc
    rec.so.rec_lds.restype = ctypes.c_uint64
    plans, two = [], 0                                         # (plans live on: buffers of others are not to be had again)
    for m, k, n, a_rows, b_cols, c_cols, more in ((3712, 3073, 3649, 1, 3, 5, (0, 0, 0)), (3073, 2945, 3777, 8, 1, 1, (0, 8, 0)), (3841, 3456, 2944, 8, 1, 1, (1, 1, 0)),
                                                  (2945, 3457, 3520, 1, 3, 5, (8, 0, 8))):
        d, s = (block(m, k, a_rows, 1), block(k, n, 1, b_cols), block(m, n, 1, c_cols)), Ground(True)
        a, w, dc = (s.bf(name, x, 2, y, 1) for name, x, y in zip(("a", "w", "dg"), d, more))
        ga, gw = s.bf("ga", d[0], 2, 0, 1), s.bf("gw", d[1], 2, 0, 1)

        def launches(room, x):
            plans.append(b.Plan(*d, 8))
            rec.so.rec_set_limit(rec.so.rec_live() + room)
            at = len(rec.ops())
            try:
                plans[-1].execute_backward(a, w, dc, *x, 0, 0)
            except b.DmmError as e:
                assert e.kind == "ENOMEM"
                return None
            return [(o[1], int(rec.so.rec_lds(o[0])), int(rec.so.rec_blocks(o[0]))) for o in rec.launches(at)]

        assert [x[0] for x in launches(1 << 40, (ga, gw))] == ["layer_copy_kernel", "layer_pair_kernel"]
        for room in (5 << 20, 9 << 20, 17 << 20):
            got, alone = launches(room, (ga, gw)), [launches(room, x) for x in ((ga, None), (None, gw))]
            if got and all(alone) and [x[0] for x in got] == ["layer_gemm_kernel"] * 2:
                assert got == alone[0] + alone[1], (m, k, n, got, alone)
                two += 1
    assert two >= 4


SCENARIOS = [without_memory_for_copies_each_gradient_has_its_own_macro_tiles, gradients_are_summed_alike_whatever_else_is_asked_for, operands_meet_at_the_same_k, narrow_tiles_of_weights_on_a_copy_of_the_rows]


@pytest.mark.parametrize("scenario", [f.__name__ for f in SCENARIOS])
def test_scenario(recorder, scenario):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, scenario], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]


if __name__ == "__main__":
    {f.__name__: f for f in SCENARIOS}[sys.argv[2]](Recorder(sys.argv[1]))
