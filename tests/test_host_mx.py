"""What the entry points for 4-bit matrices refuse (made-up device addresses: nothing is launched), and the
oracle of the format against its definition written out by hand."""
import ctypes

import numpy as np
import pytest

import workloads
from oracle import mx as oracle
from paper_2510_08874_amd import binding

BASE = 1 << 40


def whole(h, w, replication=1):
    return workloads.desc(h, w, [0, h], [0, w], 1, 1, replication=replication)


def form(d, along, code_ld=None, scale_ld=None, codes=None, scales=None):
    n, cld, sld = 0, [], []
    for _ in range(d["replication"]):
        for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]):
            for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:]):
                chunks = -(-((c1 - c0) if along == 1 else (r1 - r0)) // 128)
                cld.append(64 * chunks)
                sld.append(4 * chunks)
                n += 1
    return binding.mx_tiles([BASE + 4096 * i if codes is None else codes for i in range(n)], cld if code_ld is None else [code_ld] * n,
                            [BASE + (1 << 30) + 4096 * i if scales is None else scales for i in range(n)], sld if scale_ld is None else [scale_ld] * n)


def refused(kind, call, *args, **kw):
    with pytest.raises(binding.DmmError) as e:
        call(*args, **kw)
    assert e.value.kind == kind, e.value


D = whole(130, 300)
X = binding.tile_table([BASE + (2 << 30)], [300])
DESC = binding.matrix_desc(D)


@pytest.mark.parametrize("kind,form_args", [
    ("ELD", dict(code_ld=128)), ("ELD", dict(code_ld=200)), ("ELD", dict(scale_ld=8)), ("ELD", dict(scale_ld=14)),
    ("ELD", dict(code_ld=1 << 24)), ("ELD", dict(scale_ld=1 << 24)), ("EINVAL", dict(codes=BASE + 8)), ("EINVAL", dict(scales=BASE + 2)),
    ("EINVAL", dict(codes=0)), ("EINVAL", dict(scales=0)),
], ids=str)
def test_forms_that_are_refused(kind, form_args):
    bad, good = form(D, 1, **form_args), form(D, 1)
    refused(kind, binding.dmm_mx_quantize, DESC, 1, X, rows=bad)
    refused(kind, binding.dmm_mx_dequantize, DESC, bad, 1, 1, X)
    b = whole(300, 77)
    plan = binding.Plan(D, b, whole(130, 77), 1)
    c = binding.tile_table([BASE + (3 << 30)], [77])
    refused(kind, plan.execute_mx, bad, form(b, 2), c)
    e = whole(40, 130)
    other = binding.Plan(e, D, whole(40, 300), 1)
    refused(kind, other.execute_mx, form(e, 1), form(D, 2, **(dict(form_args, code_ld=64) if form_args.get("code_ld") == 128 else
                                                              dict(form_args, scale_ld=4) if form_args.get("scale_ld") == 8 else form_args)),
            binding.tile_table([BASE + (3 << 30)], [300]))
    assert good is not None


def test_arguments_that_are_refused():
    q = form(D, 1)
    refused("EINVAL", binding.dmm_mx_quantize, DESC, 1, X)
    refused("EINVAL", binding.dmm_mx_quantize, DESC, 3, X, rows=q)
    refused("ELD", binding.dmm_mx_quantize, DESC, 1, binding.tile_table([BASE], [299]), rows=q)
    refused("EINVAL", binding.dmm_mx_quantize, DESC, 1, binding.tile_table([None], [300]), rows=q)
    refused("EINVAL", binding.dmm_mx_quantize, DESC, 1, binding.tile_table([BASE + 1], [300]), rows=q)
    refused("EINVAL", binding.dmm_mx_quantize, DESC, 2, binding.tile_table([BASE + 2], [300]), rows=q)
    for along in (0, 3):
        refused("EINVAL", binding.dmm_mx_dequantize, DESC, q, along, 1, X)
    refused("EINVAL", binding.dmm_mx_dequantize, DESC, q, 1, 0, X)
    bad = binding.matrix_desc(dict(D, row_cuts=(0, 131)))
    refused("EINVAL", binding.dmm_mx_quantize, bad, 1, X, rows=q)
    bad = binding.matrix_desc(dict(D, col_cuts=(0, 200, 100, 300)))
    refused("EINVAL", binding.dmm_mx_quantize, bad, 1, X, rows=q)
    refused("EINVAL", binding.dmm_mx_quantize, binding.matrix_desc(dict(D, replication=0)), 1, X, rows=q)
    L = binding.lib()
    assert L.dmm_mx_quantize(None, 1, X[0], X[1], ctypes.byref(q), None, None) == binding.DMM_EINVAL
    assert L.dmm_mx_dequantize(ctypes.byref(DESC), None, 1, 1, X[0], X[1], None) == binding.DMM_EINVAL
    empty = binding.dmm_mx_tiles()
    assert L.dmm_mx_quantize(ctypes.byref(DESC), 1, X[0], X[1], ctypes.byref(empty), None, None) == binding.DMM_EINVAL


def test_products_that_are_refused():
    a, b, c = D, whole(300, 77), whole(130, 77)
    plan = binding.Plan(a, b, c, 1)
    qa, qb, t = form(a, 1), form(b, 2), binding.tile_table([BASE + (3 << 30)], [77])
    for flags in (binding.DMM_TIMING, binding.DMM_NO_MERGE, binding.DMM_SEPARATE_REDUCE, 1, 0x2000):
        refused("EINVAL", plan.execute_mx, qa, qb, t, flags)
    refused("ELD", plan.execute_mx, qa, qb, binding.tile_table([BASE], [76]))
    refused("ELD", plan.execute_mx, qa, qb, binding.tile_table([BASE], [1 << 22]))
    refused("EINVAL", plan.execute_mx, qa, qb, binding.tile_table([None], [77]))
    refused("EINVAL", plan.execute_mx, qa, qb, binding.tile_table([BASE + 2], [77]))
    refused("EINVAL", plan.execute_mx, qa, qb, binding.tile_table([BASE + 1], [77]), binding.DMM_C_BF16)
    rep = [whole(130, 256, 2), whole(256, 77, 2), whole(130, 77, 2)]
    plan = binding.Plan(*rep, 2)
    refused("EINVAL", plan.execute_mx, form(rep[0], 1), form(rep[1], 2), binding.tile_table([BASE, BASE + 65536], [77, 77]), binding.DMM_C_BF16)


@pytest.mark.parametrize("a_cols,b_rows,replication", [([0, 64, 300], [0, 300], 1), ([0, 300], [0, 130, 300], 1), ([0, 128, 300], [0, 100, 300], 1),
                                                       ([0, 300], [0, 300], 2)], ids=str)
def test_blocks_that_do_not_meet_are_refused(a_cols, b_rows, replication):
    """Cuts of K, or replicas' shares of it, that do not lie at multiples of 128."""
    a = workloads.desc(50, 300, [0, 50], a_cols, 1, 1, replication=replication)
    b = workloads.desc(300, 40, b_rows, [0, 40], 1, 1, replication=replication)
    c = whole(50, 40, replication)
    plan = binding.Plan(a, b, c, 2)
    tiles = binding.tile_table([BASE + (3 << 30) + 65536 * i for i in range(replication)], [40] * replication)
    refused("EINVAL", plan.execute_mx, form(a, 1), form(b, 2), tiles)


def test_oracle_of_the_format():
    x = np.zeros((2, 40))
    x[0, :14] = [6.0, 5.0, -5.0, 3.5, 2.5, 1.75, 1.25, -0.75, 0.25, -0.25, 0.2, 7.9, -100.0 / 16, 0.26]
    x[0, 33], x[1, 0], x[1, 39] = -1.0, 2.0 ** -140, np.inf
    codes, scales = oracle.quantize(x)
    assert codes.shape == (2, 128) and scales.tolist() == [[127, 125, 0, 0], [0, 255, 0, 0]]
    assert codes[0, :14].tolist() == [7, 6, 14, 6, 4, 4, 2, 10, 0, 8, 0, 7, 15, 1] and codes[0, 33] == 8 + 6
    assert codes[1, 0] == 0 and not codes[0, 40:].any()
    v = oracle.values(codes, scales, 40)
    assert v[0, :5].tolist() == [6.0, 4.0, -4.0, 4.0, 2.0] and v[0, 33] == -1.0 and np.isnan(v[1, 32:]).all() and not v[1, :32].any()
    assert np.array_equal(oracle.unpack(oracle.pack(codes)), codes)
