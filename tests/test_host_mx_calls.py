"""What `dmm_mx_execute` and the other entry points for 4-bit matrices and orthogonalised updates enqueue, without a
GPU: scenarios on the stand-in for the HIP runtime, as in test_host_calls.py, every one in a process of its own."""
import ctypes
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workloads  # noqa: E402
from tests.test_host_calls import Recorder, recorder, tables  # noqa: E402, F401


# ---- inside the scenario's process --------------------------------------------------------------------

def whole(h, w, replication=1):
    return workloads.desc(h, w, [0, h], [0, w], 1, 1, replication=replication)


def form(d, along, base):
    """Made-up addresses of a matrix in 4 bits."""
    from paper_2510_08874_amd import binding
    codes, scales, cld, sld = [], [], [], []
    for _ in range(d["replication"]):
        for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]):
            for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:]):
                h, w = (r1 - r0, c1 - c0) if along == 1 else (c1 - c0, r1 - r0)
                chunks = -(-w // 128)
                codes.append(base)
                scales.append(base + h * 64 * chunks)
                cld.append(64 * chunks)
                sld.append(4 * chunks)
                base += -(-h * 68 * chunks // 512) * 512 + 512
    return binding.mx_tiles(codes, cld, scales, sld)


class MxProduct:
    """A plan and made-up 4-bit operands; outputs by `where`."""

    def __init__(self, descs, nranks, flags=0):
        from paper_2510_08874_amd import binding
        self.b, self.descs, self.plan = binding, descs, binding.Plan(*descs, nranks, flags)
        self.a, self.bt = form(descs[0], 1, 1 << 44), form(descs[1], 2, 3 << 43)

    def c(self, where=0):
        return tables(self.descs[2], (1 << 45) + (where << 40), 4)

    def run(self, where=0, flags=0, stream=0):
        self.plan.execute_mx(self.a, self.bt, self.b.tile_table(*self.c(where)), flags, stream)


def replicated(m=500, k=1024, n=300):
    block = workloads.block_desc
    return MxProduct(tuple(block(r, c, 2, 2, replication=2) for r, c in ((m, k), (k, n), (m, n))), 8)


def a_replicated_product_is_captured_after_other_calls(rec):
    """The sum of C's replicas has its tables on the device with those of the product, whatever the plan did with replicas
    before: a call that did not sum, sums and copies of other replicas.  While a stream is captured nothing is copied and no
    memory is taken."""
    p, s, other = replicated(), rec.stream(), rec.stream()
    before = (lambda: p.run(0, p.b.DMM_NO_REDUCE, other), lambda: p.run(0, 0, s), lambda: p.plan.reduce_replicas(*p.c(3), 1, other),
              lambda: p.plan.broadcast_replica(*p.c(0), 1, s))
    for call in before:
        call()
        rec.so.rec_set_capturing(s, 1)
        for flags, kernels in ((0, ["mx_gemm_kernel", "reduce_replicas_kernel"]), (p.b.DMM_NO_REDUCE, ["mx_gemm_kernel"])):
            at, live = len(rec.ops()), rec.so.rec_live()
            p.run(0, flags, s)
            assert [o[1] for o in rec.ops(at) if o[1] != "event"] == kernels
            assert rec.so.rec_live() == live
        rec.so.rec_set_capturing(s, 0)
        rec.check_tables()


def a_refused_quantisation_launches_nothing(rec):
    """A tile with too many workgroups for a launch behind tiles that would have been launched: no output is touched."""
    from paper_2510_08874_amd import binding as b
    high = workloads.desc((1 << 29) + 4000, 8, [i * 100 for i in range(41)] + [(1 << 29) + 4000], [0, 8], 41, 1)
    wide = workloads.desc(600, 1 << 30, [0, 300, 600], [0, 8, 1 << 30], 2, 2)
    for d, along in ((high, 1), (wide, 2)):
        desc, q, t = b.matrix_desc(d), form(d, along, 1 << 44), b.tile_table(*tables(d, 1 << 45, 2))
        for call in (lambda: b.dmm_mx_quantize(desc, 1, t, **{("rows", "cols")[along - 1]: q}), lambda: b.dmm_mx_dequantize(desc, q, along, 1, t)):
            try:
                call()
                assert False, "not refused"
            except b.DmmError as e:
                assert e.kind == "ELIMIT"
            assert not rec.ops()


def few_rows_run_on_tiles_of_few_rows(rec):
    """Up to 32 rows: the kernel without stages or, against much B, tiles of 32 rows; no estimate is below what it takes to
    read B.  From 33 to 64 rows tiles of 64 or, with one on almost every CU, of 128."""
    rec.so.rec_lds.restype = ctypes.c_uint64
    rows_of = {76800: 32, 61440: 64, 81920: 128, 155648: 128, 163840: 256}    # bytes of LDS: stages and slots of scales
    for m, k, n, want in ((1, 8192, 28672, 32), (8, 8192, 28672, 32), (32, 8192, 28672, 32), (1, 8192, 131072, 32), (32, 8192, 131072, 32),
                          (20, 4096, 28000, 32), (32, 640, 20000, 32), (2, 1000, 60000, 32), (32, 12000, 10000, 32), (16, 4096, 14336, 32),
                          (3, 2100, 9001, 32), (31, 1157, 8897, 32), (32, 700, 12865, 32),
                          (1, 4096, 4096, 0), (16, 1024, 1024, 0), (2, 16384, 2048, 0),
                          (64, 8192, 28672, 128), (48, 4096, 28000, 128), (33, 4096, 14336, 64), (64, 4096, 4096, 64), (64, 1024, 28672, 64)):
        p, at = MxProduct((whole(m, k), whole(k, n), whole(m, n)), 1), len(rec.ops())
        p.run()
        first = rec.launches(at)[0]
        got = 0 if first[1] == "mx_skinny_kernel" else rows_of[rec.so.rec_lds(first[0])]
        assert got == want, (m, k, n, got, want)
    # a few rows dealt to row blocks: every block reads all of B, from a cache but once
    for m in (4, 16, 256):
        block = workloads.block_desc
        p, at = MxProduct((block(m, 8192, 8, 1), block(8192, 28672, 1, 8), block(m, 28672, 4, 2)), 8), len(rec.ops())
        p.run()
        assert rows_of[rec.so.rec_lds(rec.launches(at)[0][0])] == 32


def long_sums_are_cut(rec):
    """The sizes at which sums over ranges of K are tested run in ranges of K."""
    from tests.test_gpu_mx_sums import CUT, WHOLE
    for m, k, n in CUT + WHOLE:
        p, at = MxProduct((whole(m, k), whole(k, n), whole(m, n)), 1), len(rec.ops())
        p.run()
        assert ("mx_join_kernel" in [o[1] for o in rec.launches(at)]) == ((m, k, n) in CUT), (m, k, n)


SCENARIOS = [long_sums_are_cut, few_rows_run_on_tiles_of_few_rows, a_replicated_product_is_captured_after_other_calls, a_refused_quantisation_launches_nothing]


# ---- the tests ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("scenario", [f.__name__ for f in SCENARIOS])
def test_scenario(recorder, scenario):  # noqa: F811
    run = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, scenario], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]


@pytest.mark.parametrize("ld", [1 << 22, 1 << 61, (1 << 62) + 77, (1 << 63) - 1], ids=str)
def test_rows_that_lie_too_far_apart_are_refused(ld):
    """2^24 bytes and more, also where the bytes would pass 64 bits."""
    from paper_2510_08874_amd import binding as b
    d = whole(130, 300), whole(300, 77), whole(130, 77)
    plan, at = b.Plan(*d, 1), 3 << 40
    for flags in (0, b.DMM_C_BF16):
        if ld == 1 << 22 and flags:
            continue                                          # (2^23 bytes are none too many)
        with pytest.raises(b.DmmError) as e:
            plan.execute_mx(form(d[0], 1, 1 << 44), form(d[1], 2, 3 << 43), b.tile_table([at], [ld]), flags)
        assert e.value.kind == "ELD"
    for x in range(3):
        lds = [300, 77, 77]
        lds[x] = ld
        with pytest.raises(b.DmmError) as e:
            plan.execute(b.DMM_F32, [at], [lds[0]], [at], [lds[1]], [at], [lds[2]])
        assert e.value.kind == "ELD"


if __name__ == "__main__":
    {f.__name__: f for f in SCENARIOS}[sys.argv[2]](Recorder(sys.argv[1]))
