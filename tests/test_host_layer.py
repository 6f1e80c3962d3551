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

    def __init__(self):
        self.at, self.start, self.end, self.copies = 1 << 44, [], [], None

    def take(self, size, align):
        self.at += align                                       # (at multiples of the element's size, not of more)
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
        """Bytes first ... last - 1 lie in one buffer (or in this call's copies)."""
        if self.copies and self.copies[0] <= first and last <= self.copies[1]:
            return
        i = bisect.bisect_right(self.start, first) - 1
        assert i >= 0 and first >= self.start[i] and last <= self.end[i], f"{what}: bytes {first:#x} to {last:#x}, the buffer ends at {self.end[i]:#x}"


COPY = struct.Struct("<2Q2q4i")
SEG, ITEM, JOIN = struct.Struct("<3Q3I3i"), struct.Struct("<3Q3I3i" + "Qq2Q2q3Q" + "12i"), struct.Struct("<Qq2Q2q3Q" + "Q6i")
# kind of a launch: rows, columns of a right operand in its macro-tiles, by LDS; (A turned, B turned, two right operands, bytes of an element)
KINDS = {"int": (False, False, False, 1), "int_gated": (False, False, True, 1), "gated": (False, True, True, 2), "nt": (False, False, False, 2), "tn": (True, True, False, 2)}


def follow(rec, space, op, kind):
    """Everything that a launch reads and writes; the regions of its results, and how much of K each got."""
    a_turned, b_turned, dual, es = KINDS[kind]
    step = 128 // es
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

    out, parts = [], {}
    for x in range(n):
        v = ITEM.unpack(raw[x * ITEM.size:(x + 1) * ITEM.size])
        front, (c, ldc, g, u, ldg, ldu, sa, sb, sb2), (m_off, n_off, m_ext, n_ext, seg, n_segs, first, steps, tail_seg, n_tails, c_es, what) = v[:9], v[9:18], v[18:]
        k_sum, left, s, skip = 0, steps, 0, first
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
            parts[c] = k_sum
        else:
            out.append((c, ldc, c_es, m_ext, n_ext, k_sum))
            for p, ld in ((g, ldg), (u, ldu)):
                if p:
                    space.inside(p, p + ((m_ext - 1) * ld + n_ext) * 2, "what is kept")
    return out, parts


def follow_call(rec, space, at, kinds):
    """The launches of one call: [(corner, ld, bytes of an element, rows, columns, k)] of every kind."""
    space.copies = None
    for op in rec.launches(at):
        if op[1] == "layer_copy_kernel":
            blocks, x, low, high = 0, 0, 1 << 63, 0
            while blocks < rec.so.rec_blocks(op[0]):
                src, dst, src_pitch, dst_pitch, rows, size, first, _ = COPY.unpack(ctypes.string_at(op[3] + x * COPY.size, COPY.size))
                assert first == blocks and rows > 0 and size > 0
                if src:
                    space.inside(src, src + (rows - 1) * src_pitch + size, "copied")
                low, high = min(low, dst), max(high, dst + (rows - 1) * dst_pitch + size)
                blocks += -(-(-(-size // 16) * rows) // 2048)
                x += 1
            assert blocks == rec.so.rec_blocks(op[0])
            # (rows are filled up to 128 bytes, and so many lie behind the last: a read of eight columns may pass a row's end)
            space.copies = (low, -(-high // 128) * 128 + 128)
    ops = [o for o in rec.launches(at) if o[1] in ("layer_gemm_kernel", "layer_join_kernel")]
    got, x = [], 0
    for kind in kinds:
        assert ops[x][1] == "layer_gemm_kernel"
        out, parts = follow(rec, space, ops[x], kind)
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
                out.append((c, ldc, c_es, m_ext, n_ext, sum(parts[p + r * size] for r in range(runs))))
                used += runs
                y += 1
            assert used == len(slots)
        got.append(out)
    assert x == len(ops)
    return got


def covers(space, out, ptr, ld, d, es, k, step, times=1, cuts=None, replicas=1):
    """Every element of the tiles is written once, with all of K (on copies, filled up to whole steps, every interval of `cuts`)."""
    seen = {}
    cuts = cuts or [0, k]
    k = (sum(-(-(j - i) // step) * step for i, j in zip(cuts, cuts[1:])) if space.copies else k) * times
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
    which = rng.choice(("whole", "blocks", "column", "uneven"))
    if which == "whole":
        return (D(m, k, [0, m], [0, k], 1, 1), D(k, n, [0, k], [0, n], 1, 1), D(m, n, [0, m], [0, n], 1, 1)), 1
    if which == "blocks":
        return (block(m, k, 2, 2), block(k, n, 2, 2), block(m, n, 2, 2)), 4
    if which == "column":
        return (D(m, k, [0, m], [0, k], 1, 1, replication=4), block(k, n, 1, 4), block(m, n, 1, 4)), 4
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
        covers(space, [o for o in out[1] if in_tiles(space, o[0], gw)], gw[1], gw[2], db, es, m, 64)
        covers(space, [o for o in out[1] if in_tiles(space, o[0], gv)], gv[1], gv[2], db, es, m, 64)
        out = call(["nt", "tn"], lambda: plan.execute_backward(a[0], w[0], dh[0], ga[0], gw[0], b.DMM_DB_F32 if es == 4 else 0, 0))
        covers(space, out[0], ga[1], ga[2], da, 2, n, 64, 1, db["col_cuts"])
        covers(space, out[1], gw[1], gw[2], db, es, m, 64)
        rec.check_tables()
        plan.destroy()


def in_tiles(space, p, t):
    return space.start[bisect.bisect_right(space.start, p) - 1] in t[1]


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


SCENARIOS = [reads_and_writes_stay_inside, narrow_tiles]


# ---- the tests ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("scenario", [f.__name__ for f in SCENARIOS])
def test_scenario(recorder, scenario):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, scenario], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]


if __name__ == "__main__":
    {f.__name__: f for f in SCENARIOS}[sys.argv[2]](Recorder(sys.argv[1]))
