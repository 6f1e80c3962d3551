"""What the entry points for the layers around a product enqueue, without a GPU: scenarios on the stand-in for the HIP runtime, as in
test_host_calls.py, every one in a process of its own.  The work tables are read back from the stand-in's memory, and what the
kernels read and write by them is followed byte by byte."""
import bisect
import ctypes
import os
import random
import struct
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workloads  # noqa: E402
from tests.test_host_calls import Recorder, recorder  # noqa: E402, F401


# ---- inside the scenario's process --------------------------------------------------------------------

def bounds(d, replicas):
    return [(r0, r1, c0, c1) for _ in range(replicas) for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]) for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:])]


class Space:
    """Made-up device buffers that end with a tile's last element, far from each other."""

    def __init__(self, aligned=False):
        self.at, self.start, self.end, self.copies, self.results, self.aligned = 1 << 44, [], [], None, None, aligned

    def take(self, size, align):
        self.at += 0 if self.aligned else align                # (at multiples of the element's size, not of more)
        start = self.at
        self.start.append(start)
        self.end.append(start + size)
        self.at = -(-(start + size + 4096) // 512) * 512
        return start

    def tiles(self, d, es, more=0, replicas=None, turned=False):
        from paper_2510_08874_amd import binding as b
        ptr, ld = [], []
        for r0, r1, c0, c1 in bounds(d, d["replication"] if replicas is None else replicas):
            h, w = (c1 - c0, r1 - r0) if turned else (r1 - r0, c1 - c0)
            ld.append(max(w + more, 1))
            ptr.append(self.take(((h - 1) * ld[-1] + w) * es, es) if h and w else None)
        return b.tiles(ptr, ld), ptr, ld

    def integers(self, d, along, more=0):
        from paper_2510_08874_amd import binding as b
        _, ptr, ld = self.tiles(d, 1, more, turned=along == "cols")
        cuts = d["row_cuts"] if along == "rows" else d["col_cuts"]
        return b.int_tiles(ptr, ld, [self.take(4 * (j - i), 4) if j > i else None for _ in range(d["replication"]) for i, j in zip(cuts, cuts[1:])])

    def inside(self, first, last, what):
        """Bytes first ... last - 1 lie in one buffer (or in this call's copies, or its results on their way)."""
        if any(x and x[0] <= first and last <= x[1] for x in (self.copies, self.results)):
            return
        i = bisect.bisect_right(self.start, first) - 1
        assert i >= 0 and first >= self.start[i] and last <= self.end[i], f"{what}: bytes {first:#x} to {last:#x}, the buffer ends at {self.end[i]:#x}"


COPY = struct.Struct("<2Q2q4i")
PRODUCTS = ("layer_gemm_kernel", "layer_pair_kernel")
class Results(list):
    """Regions of results; `copies`: both operands lie in copies."""
    copies = False


SEG, ITEM, JOIN = struct.Struct("<3Q3I3i"), struct.Struct("<3Q3I3i" + "Qq2Q2q3Q" + "14i"), struct.Struct("<Qq2Q2q3Q" + "Q6i")
# kind of a launch: rows, columns of a right operand in its macro-tiles, by LDS; (A turned, B turned, two right operands, bytes of an element)
KINDS = {"int": (False, False, False, 1), "int_gated": (False, False, True, 1), "gated": (False, True, True, 2), "nt": (False, False, False, 2), "tn": (True, True, False, 2)}


def follow(rec, space, op):
    """Everything that a launch reads and writes: by kind of product, the regions of its results and how much of K each got; the same of partial sums."""
    i, _, _, items, _ = op
    n = int(rec.so.rec_blocks(i))
    raw = ctypes.string_at(items, n * ITEM.size)
    segs = items + n * ITEM.size

    def seg_at(x):
        return SEG.unpack(ctypes.string_at(segs + x * SEG.size, SEG.size))

    def read(p, pitch, turned, off, ext, k0, k, whole):
        if k == 0 or ext == 0:
            return
        if turned:
            first = p + k0 * pitch + off * es
            wide = (-(-ext // 8) * 8 if whole else ext) * es
            space.inside(first, first + (k - 1) * pitch + wide, f"{kind}, across K, {'whole steps' if whole else 'a tail'}")
        else:
            first = p + off * pitch + k0 * es
            space.inside(first, first + (ext - 1) * pitch + k * es, f"{kind}, along K, {'whole steps' if whole else 'a tail'}")

    got, parts = {}, {}
    for x in range(n):
        v = ITEM.unpack(raw[x * ITEM.size:(x + 1) * ITEM.size])
        front, (c, ldc, g, u, ldg, ldu, sa, sb, sb2), (m_off, n_off, m_ext, n_ext, seg, n_segs, first, steps, tail_seg, n_tails, c_es, what, kind, _) = v[:9], v[9:18], v[18:]
        kind = list(KINDS)[kind]
        a_turned, b_turned, dual, es = KINDS[kind]
        step = 128 // es
        out = got.setdefault(kind, Results())
        k_sum, left, s, skip = 0, steps, 0, first
        if steps and space.copies and space.copies[0] <= front[1] < space.copies[1]:
            out.copies = True
        while left > 0:
            rec_seg = front if s == 0 else seg_at(seg + s)
            assert s < n_segs
            here = min(left, rec_seg[6] - skip)
            assert here > 0 or rec_seg[6] == 0
            for p, pitch, turned, off, ext in ((rec_seg[0], rec_seg[3], a_turned, m_off, m_ext), (rec_seg[1], rec_seg[4], b_turned, n_off, n_ext)) + (
                    ((rec_seg[2], rec_seg[5], b_turned, n_off, n_ext),) if dual else ()):
                read(p, pitch, turned, off, ext, skip * step, here * step, True)
            k_sum += here * step
            left -= here
            s, skip = s + 1, 0
        for y in range(n_tails):
            q = seg_at(tail_seg + y)
            assert 0 <= q[7] <= step
            for p, pitch, turned, off, ext in ((q[0], q[3], a_turned, m_off, m_ext), (q[1], q[4], b_turned, n_off, n_ext)) + (
                    ((q[2], q[5], b_turned, n_off, n_ext),) if dual else ()):
                read(p, pitch, turned, off, ext, q[6] * step, q[7], False)
            k_sum += q[7]
        if es == 1:
            assert k_sum <= 131071
            if what != 2:
                for p, ext in ((sa, m_ext), (sb, n_ext)) + (((sb2, n_ext),) if dual else ()):
                    space.inside(p, p + 4 * ext, "scales")
        if what == 1:
            parts[c] = k_sum, kind
        else:
            out.append((c, ldc, c_es, m_ext, n_ext, k_sum))
            for p, ld in ((g, ldg), (u, ldu)):
                if p:
                    space.inside(p, p + ((m_ext - 1) * ld + n_ext) * 2, "what is kept")
    return got, parts


def follow_call(rec, space, at, kinds):
    """The launches of one call: [(corner, ld, bytes of an element, rows, columns, k)] of every kind."""
    space.copies, space.results, back, made, multiplied = None, None, [], [], False
    for op in rec.launches(at):
        multiplied = multiplied or op[1] in PRODUCTS
        if op[1] == "layer_copy_kernel":
            blocks, x, low, high = 0, 0, 1 << 63, 0
            while blocks < rec.so.rec_blocks(op[0]):
                src, dst, src_pitch, dst_pitch, rows, size, first, _ = COPY.unpack(ctypes.string_at(op[3] + x * COPY.size, COPY.size))
                assert first == blocks and rows > 0 and size > 0
                if multiplied:
                    back.append((src, dst, src_pitch, dst_pitch, rows, size))
                elif src:
                    space.inside(src, src + (rows - 1) * src_pitch + size, "copied")
                if not multiplied:
                    made.append((dst, dst + (rows - 1) * dst_pitch + size))
                low, high = min(low, dst), max(high, dst + (rows - 1) * dst_pitch + size)
                blocks += -(-(-(-size // 16) * rows) // 2048)
                x += 1
            assert blocks == rec.so.rec_blocks(op[0])
            if multiplied:
                continue
            # (rows are filled up to 128 bytes, and so many lie behind the last: a read of eight columns may pass a row's end)
            space.copies = (low, -(-high // 128) * 128 + 128)
    if back:
        space.results = (min(o[0] for o in back), max(o[0] + (o[4] - 1) * o[2] + o[5] for o in back))
        assert all(high <= space.results[0] or low >= space.results[1] for low, high in made)
    ops = [o for o in rec.launches(at) if o[1] in PRODUCTS or o[1] == "layer_join_kernel"]
    all_of, x = {}, 0
    while x < len(ops):
        assert ops[x][1] in PRODUCTS
        of, parts = follow(rec, space, ops[x])
        assert len(of) == (2 if ops[x][1] == "layer_pair_kernel" else 1) and not set(of) & set(all_of)
        all_of.update(of)
        x += 1
        if parts:
            assert ops[x][1] == "layer_join_kernel"
            # the joins lie behind the segments; their number follows from the slots
            join_at, slots = ops[x][3], sorted(parts)
            x += 1
            used = 0
            size = None
            y = 0
            while used < len(slots):
                c, ldc, g, u, ldg, ldu, sa, sb, sb2, p, runs, tm, tn, m_ext, n_ext, c_es = JOIN.unpack(ctypes.string_at(join_at + y * JOIN.size, JOIN.size))
                size = tm * tn * 4
                of[parts[p][1]].append((c, ldc, c_es, m_ext, n_ext, sum(parts[p + r * size][0] for r in range(runs))))
                assert len({parts[p + r * size][1] for r in range(runs)}) == 1
                used += runs
                y += 1
            assert used == len(slots)
    assert list(sorted(all_of)) == list(sorted(kinds))
    got = [all_of[kind] for kind in kinds]
    for y, of in enumerate(got):
        if not (back and of and space.results[0] <= of[0][0] < space.results[1]):
            continue
        # results in dense rows: their tiles do not meet, and what goes into the tiles is what they hold
        pitch = {o[1] * o[2] for o in of}
        assert pitch == {o[2] for o in back} and len({o[5] for o in of}) == 1
        at, pitch, es = min(o[0] for o in of), pitch.pop(), of[0][2]
        placed = sorted((*reversed(divmod(o[0] - at, pitch)), o[3], o[4] * es) for o in of)
        for i, (col, row, h, w) in enumerate(placed):
            assert col + w <= pitch and not any(c < col + w and r < row + h and row < r + hh for c, r, hh, _ in placed[i + 1:])
        rows, cols = max(r + h for _, r, h, _ in placed), max(c + w for c, _, _, w in placed)
        assert sum(h * w for _, _, h, w in placed) == rows * cols
        out = Results()
        for src, dst, _, dst_pitch, h, size in back:
            r, c = divmod(src - at, pitch)
            if r < rows and c + size <= cols and r + h <= rows:    # (what is kept of G and U lies behind H)
                out.append((dst, dst_pitch // es, es, h, size // es, of[0][5]))
            else:
                space.inside(dst, dst + (h - 1) * dst_pitch + size, "kept results")
        got[y] = out
    return got


def covers(space, out, ptr, ld, d, es, k, step, times=1, cuts=None, replicas=1):
    """Every element of the tiles is written once, with all of K (on copies, filled up to whole steps, every interval of `cuts`)."""
    seen = {}
    cuts = cuts or [0, k]
    k = (sum(-(-(j - i) // step) * step for i, j in zip(cuts, cuts[1:])) if out.copies else k) * times
    for c, ldc, c_es, h, w, k_sum in out:
        assert c_es == es and k_sum == k, (c_es, es, k_sum, k)
        i = bisect.bisect_right(space.start, c) - 1
        row, col = divmod((c - space.start[i]) // es, ldc)
        seen.setdefault(space.start[i], []).append((row, col, h, w, ldc))
    for p, l, (r0, r1, c0, c1) in zip(ptr, ld, bounds(d, replicas)):
        if p is None:
            continue
        area, corners = 0, set()
        for row, col, h, w, ldc in seen.pop(p):
            assert ldc == l and row + h <= r1 - r0 and col + w <= c1 - c0
            area += h * w
            corners.add((row, col))
        assert area == (r1 - r0) * (c1 - c0) and len(corners) == len(set(corners))
    assert not seen


def layouts(rng, m, k, n):
    D, block, jitter = workloads.desc, workloads.block_desc, workloads.jittered_cuts
    which = rng.choice(("whole", "blocks", "column", "uneven", "row_col"))
    if which == "whole":
        return (D(m, k, [0, m], [0, k], 1, 1), D(k, n, [0, k], [0, n], 1, 1), D(m, n, [0, m], [0, n], 1, 1)), 1
    if which == "blocks":
        return (block(m, k, 2, 2), block(k, n, 2, 2), block(m, n, 2, 2)), 4
    if which == "column":
        return (D(m, k, [0, m], [0, k], 1, 1, replication=4), block(k, n, 1, 4), block(m, n, 1, 4)), 4
    if which == "row_col":
        return (block(m, k, 8, 1), block(k, n, 1, 8), block(m, n, 2, 4)), 8
    s = rng.randrange(1000)
    return (D(m, k, jitter(m, 3, s), jitter(k, 5, s + 1), 3, 5), D(k, n, jitter(k, 4, s + 2), jitter(n, 2, s + 3), 4, 2), D(m, n, jitter(m, 5, s + 4), jitter(n, 3, s + 5), 5, 3)), 15


def reads_and_writes_stay_inside(rec):
    """Random sizes, cuts and leading dimensions, the smallest buffers that hold the tiles: what the kernels read and write by the work tables lies
    inside them, and every result gets all of K, once."""
    from paper_2510_08874_amd import binding as b
    rng = random.Random(11)
    for turn in range(150):
        def size(hi):
            return max(15, rng.choice((rng.randint(15, 300), rng.randint(15, hi), rng.randint(1, hi // 64) * 64)))
        m, k, n = size(2600), size(3000), size(2600)
        if turn % 10 == 0:
            m = rng.randint(15, 64)
        if turn % 15 == 0:
            k = 140000 + rng.randint(0, 300)
        d, ranks = layouts(rng, m, k, n)
        da, db, dc = d
        more = rng.choice((0, 0, 1, 3, 8))
        plan = b.Plan(*d, ranks)

        def call(kinds, f):
            at = len(rec.ops())
            f()
            return follow_call(rec, space, at, kinds)

        space = Space()
        a, w, v = space.integers(da, "rows", more), space.integers(db, "cols", more), space.integers(db, "cols", more + 2)
        c, h = space.tiles(dc, 4, more), space.tiles(dc, 2, more)
        (out,) = call(["int"], lambda: plan.execute_int(a, w, c[0], 0, 0))
        covers(space, out, c[1], c[2], dc, 4, k, 128)
        (out,) = call(["int_gated"], lambda: plan.gated_int(b.DMM_SILU, a, w, v, h[0], 0))
        covers(space, out, h[1], h[2], dc, 2, k, 128)
        if k > 10000:
            continue
        space = Space()
        a, w, v, h, g, u, dh, dg, du = [space.tiles(x, 2, more + y) for y, x in enumerate((da, db, db, dc, dc, dc, dc, dc, dc))]
        (out,) = call(["gated"], lambda: plan.gated(b.DMM_GELU, a[0], w[0], v[0], h[0], g[0], u[0], 0))
        covers(space, out, h[1], h[2], dc, 2, k, 64)
        es = rng.choice((2, 4))
        ga, gw, gv = space.tiles(da, 2, more, 1), space.tiles(db, es, more, 1), space.tiles(db, es, more, 1)
        out = call(["nt", "tn"], lambda: plan.gated_backward(b.DMM_GELU, a[0], w[0], v[0], g[0], u[0], dh[0], dg[0], du[0], ga[0], gw[0], gv[0],
                                                             b.DMM_DB_F32 if es == 4 else 0, 0))
        covers(space, out[0], ga[1], ga[2], da, 2, n, 64, 2, db["col_cuts"])
        covers(space, those(space, out[1], gw), gw[1], gw[2], db, es, m, 64)
        covers(space, those(space, out[1], gv), gv[1], gv[2], db, es, m, 64)
        out = call(["nt", "tn"], lambda: plan.execute_backward(a[0], w[0], dh[0], ga[0], gw[0], b.DMM_DB_F32 if es == 4 else 0, 0))
        covers(space, out[0], ga[1], ga[2], da, 2, n, 64, 1, db["col_cuts"])
        covers(space, out[1], gw[1], gw[2], db, es, m, 64)
        rec.check_tables()
        plan.destroy()


def those(space, out, t):
    """The results that lie in the tiles `t`."""
    got = Results(o for o in out if space.start[bisect.bisect_right(space.start, o[0]) - 1] in t[1])
    got.copies = out.copies
    return got


def narrow_tiles(rec):
    """Tiles of a few columns: a read of eight columns runs over several rows."""
    from paper_2510_08874_amd import binding as b
    for m, k, n in ((200, 200, 1), (200, 1, 200), (130, 70, 2), (64, 128, 3), (128, 64, 9), (65, 66, 67), (64, 3, 5), (192, 7, 1)):
        for cuts in ([0], [0, 1], [0, 66], [0, 3, 100]):
            rows = sorted({c for c in cuts if c < m} | {0}) + [m]
            ks = sorted({c for c in cuts if c < k} | {0}) + [k]
            d = (workloads.desc(m, k, rows, [0, k], 1, 1), workloads.desc(k, n, ks, [0, n], 1, 1), workloads.desc(m, n, [0, m], [0, n], 1, 1))
            plan = b.Plan(*d, 1)
            for more in (0, 1, 5):
                space = Space()
                a, w, v, h = [space.tiles(x, 2, more) for x in (d[0], d[1], d[1], d[2])]
                at = len(rec.ops())
                plan.gated(b.DMM_SILU, a[0], w[0], v[0], h[0], None, None, 0)
                (out,) = follow_call(rec, space, at, ["gated"])
                covers(space, out, h[1], h[2], d[2], 2, k, 64)
                ga, gw = space.tiles(d[0], 2, more), space.tiles(d[1], 4, more)
                at = len(rec.ops())
                plan.execute_backward(a[0], w[0], h[0], ga[0], gw[0], b.DMM_DB_F32, 0)
                out = follow_call(rec, space, at, ["nt", "tn"])
                covers(space, out[0], ga[1], ga[2], d[0], 2, n, 64, 1, d[1]["col_cuts"])
                covers(space, out[1], gw[1], gw[2], d[1], 4, m, 64)


def sizes_under_test_take_the_ways_they_are_meant_for(rec):
    """The sizes of the GPU tests of calls: whole tiles as they lie, tiles cut along K, copies of the operands."""
    from paper_2510_08874_amd import binding as b
    for layout, m, k, n, kernels in (("blocks", 512, 512, 768, {"layer_gemm_kernel"}), ("whole", 40, 8192, 300, {"layer_gemm_kernel", "layer_join_kernel"}),
                                     ("uneven", 1301, 1103, 907, {"layer_gemm_kernel", "layer_copy_kernel"}),
                                     ("row_col", 9, 2000, 12001, {"layer_gemm_kernel", "layer_copy_kernel"})):
        d = made(layout, m, k, n)
        plan, space = b.Plan(*d, 12), Space(True)
        a, w, v = space.integers(d[0], "rows"), space.integers(d[1], "cols"), space.integers(d[1], "cols")
        t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2], d[2], d[2], d[2], d[0], d[1])]
        c = space.tiles(d[2], 4)[0]
        for call, at_least in ((lambda: plan.execute_int(a, w, c, 0, 0), kernels), (lambda: plan.gated_int(b.DMM_GELU, a, w, v, t[3], 0), kernels),
                               (lambda: plan.gated(b.DMM_SILU, *t[:4], None, None, 0), kernels), (lambda: plan.execute_backward(t[0], t[1], t[3], t[7], t[8]), set())):
            at = len(rec.ops())
            call()
            names = [o[1] for o in rec.launches(at)]
            if layout == "row_col":                                # (results are copied behind the product, dA in front of dB)
                assert names.count("layer_copy_kernel") == 2 and names[0] == names[-1] == "layer_copy_kernel", names
            got = set(names)
            assert got >= at_least and (not at_least or "layer_copy_kernel" in at_least or "layer_copy_kernel" not in got), (layout, got)


def made(layout, m, k, n):
    """As in layer_tiles.py, which needs a GPU."""
    def uneven(n, parts):
        cuts = [0] + sorted((n * (i * i + 2 * i) // (parts * parts + 2 * parts)) for i in range(1, parts)) + [n]
        if parts >= 3:
            cuts[2] = cuts[1]
        return cuts
    D, block = workloads.desc, workloads.block_desc
    if layout == "whole":
        return D(m, k, [0, m], [0, k], 1, 1), D(k, n, [0, k], [0, n], 1, 1), D(m, n, [0, m], [0, n], 1, 1)
    if layout == "blocks":
        return block(m, k, 2, 2), block(k, n, 2, 2), block(m, n, 2, 2)
    if layout == "row_col":
        return block(m, k, 8, 1), D(k, n, uneven(k, 3), uneven(n, 2), 3, 2), block(m, n, 4, 2)
    return D(m, k, uneven(m, 3), uneven(k, 4), 3, 4), D(k, n, uneven(k, 3), uneven(n, 2), 3, 2), D(m, n, uneven(m, 2), uneven(n, 3), 2, 3)


def few_rows_run_on_few_rows(rec):
    """Up to 32 rows on tiles of 32 and up to 64 on tiles of 64 or 32 wherever memory bounds them, whole along K where tiles fill the device,
    with more steps in flight where every workgroup has a CU to itself."""
    from paper_2510_08874_amd import binding as b
    rec.so.rec_lds.restype = ctypes.c_uint64
    for m, want, n, deep in ((1, 32, 28672, True), (17, 32, 28672, True), (32, 32, 28672, True), (48, 64, 28672, True), (64, 64, 28672, True), (32, 32, 40960, False),
                             (64, 64, 40960, False)):
        d = made("whole", m, 8192, n)
        plan, space = b.Plan(*d, 1), Space(True)
        a, w, v = space.integers(d[0], "rows"), space.integers(d[1], "cols"), space.integers(d[1], "cols")
        t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2])]
        # (bytes of LDS: stages)
        for call, rows in ((lambda: plan.execute_int(a, w, t[3], b.DMM_C_BF16, 0), {7 * 160 * 128: 32, 6 * 192 * 128: 64} if deep else {3 * 160 * 128: 32, 3 * 192 * 128: 64}),
                           (lambda: plan.gated_int(b.DMM_GELU, a, w, v, t[3], 0), {4 * 288 * 128: 32, 3 * 320 * 128: 64}),
                           (lambda: plan.gated(b.DMM_SILU, *t, None, None, 0), {4 * 288 * 128: 32, 3 * 320 * 128: 64})):
            at = len(rec.ops())
            call()
            ops = rec.launches(at)
            assert [o[1] for o in ops] == ["layer_gemm_kernel"] and rows.get(rec.so.rec_lds(ops[0][0])) == want, (m, want, rec.so.rec_lds(ops[0][0]))


def rows_in_blocks_are_joined_on_a_copy(rec):
    """Few rows, cut into blocks each of which would bring in all of the weights: the rows alone are copied, C's tiles are written whole, or, where C is cut
    into blocks of rows as well, from scratch memory."""
    from paper_2510_08874_amd import binding as b
    for m, k, n, blocks, back in ((8, 4096, 16384, 4, True), (64, 4096, 16380, 4, True), (61, 4099, 8192, 4, True), (64, 4096, 4100, 1, False)):
        d = (workloads.block_desc(m, k, 8, 1), workloads.desc(k, n, [0, 1000, k], [0, n], 2, 1), workloads.block_desc(m, n, blocks, 8 // blocks))
        plan, space = b.Plan(*d, 8), Space(True)
        a, w, v = space.integers(d[0], "rows"), space.integers(d[1], "cols"), space.integers(d[1], "cols")
        t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1])]
        h, g, u = (space.tiles(d[2], 2) for _ in range(3))
        for kind, call in (("int", lambda: plan.execute_int(a, w, h[0], b.DMM_C_BF16, 0)), ("int_gated", lambda: plan.gated_int(b.DMM_GELU, a, w, v, h[0], 0)),
                           ("gated", lambda: plan.gated(b.DMM_SILU, *t, h[0], None, None, 0)), ("gated", lambda: plan.gated(b.DMM_SILU, *t, h[0], g[0], u[0], 0)),
                           ("gated", lambda: plan.gated(b.DMM_SILU, *t, h[0], None, u[0], 0))):
            at = len(rec.ops())
            call()
            (out,) = follow_call(rec, space, at, [kind])
            assert space.copies and not out.copies and bool(space.results) == back, (kind, m, k, n)
            covers(space, out, h[1], h[2], d[2], 2, k, 64)
    # a layer's gradients by few rows: dA alike, dB on copies of both its operands
    for m, k, n, back in ((83, 4160, 16384, True), (96, 4099, 8192, False)):
        d = (workloads.block_desc(m, k, 8 if back else 1, 1), workloads.desc(k, n, [0, 1000, k], [0, 3001, n], 2, 2), workloads.block_desc(m, n, 4, 2))
        plan, space = b.Plan(*d, 8), Space()
        a, w, v, h, g, u, dg, du, da = (space.tiles(x, 2) for x in (d[0], d[1], d[1], d[2], d[2], d[2], d[2], d[2], d[0]))
        dw, dv = space.tiles(d[1], 4), space.tiles(d[1], 4)
        at = len(rec.ops())
        plan.gated_backward(b.DMM_SILU, a[0], w[0], v[0], g[0], u[0], h[0], dg[0], du[0], da[0], dw[0], dv[0], b.DMM_DB_F32, 0)
        out = follow_call(rec, space, at, ["nt", "tn"])
        assert space.copies and not out[0].copies and out[1].copies and bool(space.results) == back, (m, k, n)
        covers(space, out[0], da[1], da[2], d[0], 2, n, 64, 2)
        covers(space, those(space, out[1], dw), dw[1], dw[2], d[1], 4, m, 64)
        covers(space, those(space, out[1], dv), dv[1], dv[2], d[1], 4, m, 64)


def both_gradients_in_one_launch(rec):
    """Where each alone leaves places empty, and not where both fill the device with tiles of 256 x 256."""
    from paper_2510_08874_amd import binding as b
    for m, k, n, one in ((381, 720, 1112, True), (1448, 512, 768, True), (256, 1080, 3600, True), (4096, 4096, 4096, False)):
        d = made("blocks", m, k, n)
        plan, space = b.Plan(*d, 4), Space(True)
        a, w, dc = (space.tiles(x, 2) for x in d)
        da, db = space.tiles(d[0], 2), space.tiles(d[1], 4)
        at = len(rec.ops())
        plan.execute_backward(a[0], w[0], dc[0], da[0], db[0], b.DMM_DB_F32, 0)
        names = [o[1] for o in rec.launches(at) if o[1] in PRODUCTS]
        assert names == (["layer_pair_kernel"] if one else ["layer_gemm_kernel"] * 2), (m, k, n)
        out = follow_call(rec, space, at, ["nt", "tn"])
        covers(space, out[0], da[1], da[2], d[0], 2, n, 64, 1, d[1]["col_cuts"])
        covers(space, out[1], db[1], db[2], d[1], 4, m, 64)


def a_call_without_memory_for_copies_runs_on_the_operands(rec):
    from paper_2510_08874_amd import binding as b
    d = made("uneven", 1301, 1103, 907)
    plan, space = b.Plan(*d, 12), Space(True)
    t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2])]
    rec.so.rec_fail_allocations(3, 1)                          # (behind the tables' buffers, if these come first)
    for _ in range(3):
        at = len(rec.ops())
        plan.gated(b.DMM_SILU, *t, None, None, 0)
        assert "layer_gemm_kernel" in [o[1] for o in rec.launches(at)]
        rec.check_tables()
    rec.so.rec_set_limit(0)                                    # no memory at all: refused, and as before when there is some again
    other = b.Plan(*d, 12)
    at = len(rec.ops())
    try:
        other.gated(b.DMM_SILU, *t, None, None, 0)
        assert "layer_gemm_kernel" in [o[1] for o in rec.launches(at)]     # (on buffers that are there)
    except b.DmmError as e:
        assert e.kind == "ENOMEM" and not rec.launches(at)
    rec.so.rec_set_limit(1 << 40)
    other.gated(b.DMM_SILU, *t, None, None, 0)


def captures_take_what_is_there(rec):
    """A first call is refused while a stream is captured; a call with the tables of the call before takes no memory, copies nothing and waits for nothing, on
    any stream; one with others is refused."""
    from paper_2510_08874_amd import binding as b
    for layout, m, k, n in (("blocks", 512, 512, 768), ("whole", 40, 8192, 300), ("uneven", 1301, 1103, 907)):
        d = made(layout, m, k, n)
        plan, space = b.Plan(*d, 12), Space(True)
        a, w, v = space.integers(d[0], "rows"), space.integers(d[1], "cols"), space.integers(d[1], "cols")
        t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2], d[2], d[2], d[2], d[2], d[0], d[1], d[1])]
        c = [space.tiles(d[2], 4)[0] for _ in range(2)]
        s, side = rec.stream(), rec.stream()
        calls = [lambda x, st: plan.execute_int(a, w, c[x], 0, st), lambda x, st: plan.gated_int(b.DMM_GELU, a, w, v, t[3 + x], st),
                 lambda x, st: plan.gated(b.DMM_SILU, *t[:3], t[3 + x], None, None, st),
                 lambda x, st: plan.gated_backward(b.DMM_SILU, *t[:6], t[6 - x], t[7 - x], *t[8:], stream=st),
                 lambda x, st: plan.execute_backward(t[0], t[1], t[3 + x], t[8], t[9], 0, st)]
        for call in calls:
            rec.so.rec_set_capturing(side, 1)
            at = len(rec.ops())
            try:
                call(0, side)
                assert False, "not refused"
            except b.DmmError as e:
                assert e.kind == "EINVAL" and not rec.launches(at)
            rec.so.rec_set_capturing(side, 0)
            call(0, s)
            want = [o[1] for o in rec.launches(at)]
            rec.so.rec_set_capturing(side, 1)
            at, live = len(rec.ops()), rec.so.rec_live()
            call(0, side)
            assert [o[1] for o in rec.launches(at)] == want and rec.so.rec_live() == live and not [o for o in rec.ops(at) if o[1] == "copy"]
            at = len(rec.ops())
            try:
                call(1, side)
                assert False, "not refused"
            except b.DmmError as e:
                assert e.kind == "EINVAL" and not rec.launches(at)
            rec.so.rec_set_capturing(side, 0)
        rec.check_tables()
        plan.destroy()


def partial_sums_and_copies_wait_for_each_other(rec):
    """Calls on two streams whose partial sums or copies lie in one buffer: each behind the one before; with whole tiles they need not wait."""
    from paper_2510_08874_amd import binding as b
    for layout, m, k, n, shared in (("blocks", 512, 512, 768, False), ("whole", 40, 8192, 300, True), ("uneven", 1301, 1103, 907, True)):
        d = made(layout, m, k, n)
        plan, space = b.Plan(*d, 12), Space(True)
        t = [space.tiles(x, 2)[0] for x in (d[0], d[1], d[1], d[2])]
        streams = [rec.stream(), rec.stream()]
        last = None
        for turn in range(4):
            at = len(rec.ops())
            plan.gated(b.DMM_SILU, *t, None, None, streams[turn % 2])
            ops = [o[0] for o in rec.launches(at)]
            if last is not None:
                assert rec.before(last, ops[0]) or not shared
            last = ops[-1]
        rec.check_tables()
        plan.destroy()


def many_rows_take_several_launches(rec):
    """A launch has less than 2^32 threads, and no row is left out or quantised twice."""
    from paper_2510_08874_amd import binding as b
    rec.so.rec_blocks.restype = ctypes.c_uint
    for m, n, threads in (((1 << 24) + 5, 8192, 256), ((1 << 22) + 5, 40000, 1024), ((1 << 31) - (1 << 17), 1, 64), (1 << 22, 2000, 64)):
        d, space = workloads.desc(m, n, [0, m], [0, n], 1, 1), Space(True)
        at = len(rec.ops())
        b.dmm_int_quantize(b.matrix_desc(d), b.DMM_BF16, space.tiles(d, 2)[0], rows=space.integers(d, "rows"))
        ops = rec.launches(at)
        blocks = [int(rec.so.rec_blocks(o[0])) for o in ops]
        assert {o[1] for o in ops} == {"i8_whole_rows_kernel"} and sum(blocks) == m and max(blocks) * threads < 1 << 32, (m, n, blocks)


SCENARIOS = [many_rows_take_several_launches, rows_in_blocks_are_joined_on_a_copy, both_gradients_in_one_launch,
             reads_and_writes_stay_inside, narrow_tiles, sizes_under_test_take_the_ways_they_are_meant_for, few_rows_run_on_few_rows,
             a_call_without_memory_for_copies_runs_on_the_operands, captures_take_what_is_there, partial_sums_and_copies_wait_for_each_other]


# ---- the tests ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("scenario", [f.__name__ for f in SCENARIOS])
def test_scenario(recorder, scenario):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, scenario], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]


BASE = 1 << 44


def refused(kind, call, *args, **kw):
    from paper_2510_08874_amd import binding as b
    with pytest.raises(b.DmmError) as e:
        call(*args, **kw)
    assert e.value.kind == kind, e.value


def a_plan(m=100, k=60, n=80, replication=1):
    from paper_2510_08874_amd import binding as b
    d = [workloads.desc(r, c, [0, r], [0, c], 1, 1, replication=replication) for r, c in ((m, k), (k, n), (m, n))]
    return b, d, b.Plan(*d, replication)


def good(b, d, ld=None, at=BASE, replicas=1):
    return b.tiles([at + (i << 30) for i in range(replicas)], [ld or d["cols"]] * replicas)


def good_int(b, d, along, ld=None, at=BASE, scales=BASE + (1 << 40), replicas=1):
    w = d["cols"] if along == "rows" else d["rows"]
    return b.int_tiles([at and at + (i << 30) for i in range(replicas)], [ld or w] * replicas, [scales] * replicas)


def test_refusals_of_integers():
    b, (da, db, dc), plan = a_plan()
    desc = b.matrix_desc(da)
    x, rows, cols = good(b, da), good_int(b, da, "rows"), good_int(b, da, "cols")
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_BF16, x)                                  # no form
    refused("EINVAL", b.dmm_int_quantize, desc, 3, x, rows=rows)                                # no such type
    refused("ELD", b.dmm_int_quantize, desc, b.DMM_BF16, good(b, da, 59), rows=rows)
    refused("ELD", b.dmm_int_quantize, desc, b.DMM_BF16, x, rows=good_int(b, da, "rows", 59))
    refused("ELD", b.dmm_int_quantize, desc, b.DMM_BF16, x, cols=good_int(b, da, "cols", 99))
    refused("ELD", b.dmm_int_quantize, desc, b.DMM_BF16, x, rows=good_int(b, da, "rows", 1 << 24))
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_BF16, good(b, da, at=BASE + 1), rows=rows)   # not aligned to its elements
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_F32, good(b, da, at=BASE + 2), rows=rows)
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_BF16, x, rows=good_int(b, da, "rows", at=None))
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_BF16, x, rows=good_int(b, da, "rows", scales=None))
    refused("EINVAL", b.dmm_int_quantize, desc, b.DMM_BF16, x, rows=good_int(b, da, "rows", scales=BASE + 2))
    refused("EINVAL", b.dmm_int_dequantize, desc, rows, 3, b.DMM_BF16, x)
    refused("EINVAL", b.dmm_int_dequantize, desc, rows, b.DMM_MX_ROWS, 0, x)
    refused("ELD", b.dmm_int_dequantize, desc, rows, b.DMM_MX_COLS, b.DMM_BF16, x)              # rows of 60 bytes where a column has 100
    bad = b.matrix_desc(dict(da, col_cuts=[0, 59]))
    refused("EINVAL", b.dmm_int_quantize, bad, b.DMM_BF16, x, rows=rows)
    a, w = good_int(b, da, "rows"), good_int(b, db, "cols")
    refused("EINVAL", plan.execute_int, a, w, good(b, dc), b.DMM_TIMING)
    refused("EINVAL", plan.execute_int, a, w, good(b, dc), b.DMM_DB_F32)
    refused("EINVAL", plan.execute_int, a, w, good(b, dc, at=BASE + 2), 0)                      # fp32 tiles
    refused("ELD", plan.execute_int, a, w, good(b, dc, 79), 0)
    refused("ELD", plan.execute_int, a, w, good(b, dc, 1 << 22), 0)
    refused("ELD", plan.execute_int, a, w, good(b, dc, 1 << 23), b.DMM_C_BF16)
    refused("ELD", plan.execute_int, good_int(b, da, "rows", 59), w, good(b, dc), 0)
    refused("ELD", plan.execute_int, a, good_int(b, db, "cols", 59), good(b, dc), 0)
    refused("EINVAL", plan.execute_int, a, good_int(b, db, "cols", scales=None), good(b, dc), 0)
    for act in (0, 4, -1):
        refused("EINVAL", plan.gated_int, act, a, w, w, good(b, dc))
    refused("ELD", plan.gated_int, b.DMM_SILU, a, w, good_int(b, db, "cols", 59), good(b, dc))
    refused("EINVAL", plan.gated_int, b.DMM_SILU, a, w, w, good(b, dc, at=BASE + 1))
    b, (ra, rb, rc), replicated = a_plan(replication=2)
    a, w = good_int(b, ra, "rows", replicas=2), good_int(b, rb, "cols", replicas=2)
    refused("EINVAL", replicated.execute_int, a, w, good(b, rc, replicas=2), b.DMM_C_BF16)
    refused("EINVAL", replicated.gated_int, b.DMM_SILU, a, w, w, good(b, rc, replicas=2))


def test_sizes_that_do_not_fit_32_bits():
    most = (1 << 31) - (1 << 16)
    b, (da, db, dc), plan = a_plan(most + 1, 1, 1)
    a, w, h = good(b, da), good(b, db), good(b, dc)
    refused("ELIMIT", plan.gated, b.DMM_SILU, a, w, w, h)
    refused("ELIMIT", plan.gated_backward, b.DMM_SILU, a, w, w, h, h, h, h, h, a, w, w)
    refused("ELIMIT", plan.execute_backward, a, w, h, a, w)
    refused("ELIMIT", plan.execute_int, good_int(b, da, "rows"), good_int(b, db, "cols"), h, 0)
    refused("ELIMIT", plan.gated_int, b.DMM_SILU, good_int(b, da, "rows"), good_int(b, db, "cols"), good_int(b, db, "cols"), h)
    for rows, cols in ((most + 1, 1), (1, most + 1)):
        d = workloads.desc(rows, cols, [0, rows], [0, cols], 1, 1)
        form, along = (good_int(b, d, "rows"), "rows") if cols == 1 else (good_int(b, d, "cols"), "cols")
        refused("ELIMIT", b.dmm_int_quantize, b.matrix_desc(d), b.DMM_BF16, good(b, d), **{along: form})
        refused("ELIMIT", b.dmm_int_dequantize, b.matrix_desc(d), form, b.DMM_MX_ROWS if along == "rows" else b.DMM_MX_COLS, b.DMM_BF16, good(b, d))


def test_refusals_of_bf16_layers():
    b, (da, db, dc), plan = a_plan()
    a, w, h = good(b, da), good(b, db), good(b, dc)
    for act in (0, 4, -1):
        refused("EINVAL", plan.gated, act, a, w, w, h)
        refused("EINVAL", plan.gated_backward, act, a, w, w, h, h, h, h, h)
    for x in range(6):
        args = [good(b, d, d["cols"] - 1 if x == y else None) for y, d in enumerate((da, db, db, dc, dc, dc))]
        refused("ELD", plan.gated, b.DMM_SILU, *args)
        args = [good(b, d, 1 << 23 if x == y else None) for y, d in enumerate((da, db, db, dc, dc, dc))]
        refused("ELD", plan.gated, b.DMM_SILU, *args)
        args = [good(b, d, at=BASE + (x == y)) for y, d in enumerate((da, db, db, dc, dc, dc))]
        refused("EINVAL", plan.gated, b.DMM_SILU, *args)
    everything = (da, db, db, dc, dc, dc, dc, dc, da, db, db)
    for x in range(11):
        args = [good(b, d, d["cols"] - 1 if x == y else None) for y, d in enumerate(everything)]
        refused("ELD", plan.gated_backward, b.DMM_SILU, *args)
        args = [good(b, d, at=BASE + (x == y)) for y, d in enumerate(everything)]
        refused("EINVAL", plan.gated_backward, b.DMM_SILU, *args)
    full = [good(b, d) for d in everything]
    refused("EINVAL", plan.gated_backward, b.DMM_SILU, *full, b.DMM_C_BF16)                     # no such flag here
    for x in (9, 10):                                                                           # fp32 where bf16 alone is aligned
        refused("EINVAL", plan.gated_backward, b.DMM_SILU, *[t if y != x else good(b, db, at=BASE + 2) for y, t in enumerate(full)], b.DMM_DB_F32)
    refused("EINVAL", plan.gated_backward, b.DMM_SILU, None, *full[1:])                         # a weight's gradient without A
    refused("EINVAL", plan.gated_backward, b.DMM_SILU, full[0], None, *full[2:])                # A's without a weight
    refused("EINVAL", plan.gated_backward, b.DMM_SILU, full[0], full[1], None, *full[3:])
    refused("EINVAL", plan.execute_backward, a, w, h, None, None)                               # nothing to do
    refused("EINVAL", plan.execute_backward, None, w, h, a, w)
    refused("EINVAL", plan.execute_backward, a, None, h, a, w)
    refused("EINVAL", plan.execute_backward, a, w, h, a, w, b.DMM_NO_REDUCE)
    refused("ELD", plan.execute_backward, a, w, good(b, dc, 79), a, w)
    refused("ELD", plan.execute_backward, a, w, h, a, good(b, db, 1 << 22), b.DMM_DB_F32)
    refused("EINVAL", plan.execute_backward, a, w, h, a, good(b, db, at=BASE + 2), b.DMM_DB_F32)
    b, (ra, rb, rc), replicated = a_plan(replication=2)
    a, w, h = (good(b, d, replicas=2) for d in (ra, rb, rc))
    refused("EINVAL", replicated.gated, b.DMM_SILU, a, w, w, h)
    refused("EINVAL", replicated.gated_backward, b.DMM_SILU, a, w, w, h, h, h, h, h)


if __name__ == "__main__":
    {f.__name__: f for f in SCENARIOS}[sys.argv[2]](Recorder(sys.argv[1]))
