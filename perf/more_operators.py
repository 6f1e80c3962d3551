"""The operators of a feed-forward layer beside the products of `cases.py`: products of 8-bit integers with a scale
for every token and channel, the gated block, and the gradients of bf16 products.

  quantize          a partitioned matrix to 8-bit integers with a scale for every row (token) or column (channel), and
                    back to values
  product           C = A B of such matrices, partitioned and replicated like the operands of `dmm_execute`
  gated_i8          H = act(A Wg) * (A Wu) of such matrices
  gated             the same in bf16; a training step keeps G = A Wg and U = A Wu
  gated_backward    dG, dU, dA, dWg and dWu from dH, G and U
  linear_backward   dA = dC B^T and dB = A^T dC

A row's scale is its largest magnitude over 127, whatever tiles it is cut into; an element is the integer nearest
to its value over the scale, half-way values to the even one.  act is silu, gelu (with the error function) or gelu_tanh.
dG and dU are results in bf16, and the other gradients are products of these.

A case is a dict of plain values; `layout` says how the matrices are cut and dealt to the ranks.
"""
from __future__ import annotations

import math

import torch

own = False

CHUNK = 1024                                                   # products of so many pairs of 8-bit integers add up exactly in fp32


def listed():
    return [
        # the activations of a few new tokens in front of a layer: the smallest call, where latency counts
        dict(name="i8_quantize_tokens", op="quantize", layout="1x1", rows=16, cols=8192, dtype="bf16", along="rows"),
        # a fp32 weight of odd sizes in uneven blocks, a scale for every channel
        dict(name="i8_quantize_weight_ragged", op="quantize", layout="uneven", rows=4099, cols=11003, dtype="f32", along="cols"),
        # one new token through a tensor-parallel layer
        dict(name="i8_product_token", op="product", layout="column", ranks=8, m=1, k=8192, n=28672, c_dtype="bf16"),
        # the same layer on a long prompt batch
        dict(name="i8_product_prefill", op="product", layout="column", ranks=8, m=16384, k=8192, n=28672, c_dtype="bf16"),
        # a batch of sequences that get a token each, both projections in column blocks
        dict(name="i8_gated_tokens", op="gated_i8", layout="column", ranks=8, m=48, k=8192, n=28672, act="silu"),
        # uneven blocks, odd sizes
        dict(name="i8_gated_ragged", op="gated_i8", layout="uneven", ranks=15, m=2501, k=1999, n=1777, act="gelu"),
        # a few tokens through the block in bf16
        dict(name="gated_tokens", op="gated", layout="column", ranks=8, m=4, k=8192, n=28672, act="silu", keep=False),
        # the forward half of a training step at the sizes of the MLP benchmark (the largest call)
        dict(name="gated_training", op="gated", layout="column", ranks=8, m=8192, k=12288, n=49152, act="silu", keep=True),
        # the backward half of a step in 2-D blocks
        dict(name="gated_backward_step", op="gated_backward", layout="2x2", ranks=4, m=4096, k=4096, n=8192, act="silu"),
        # uneven blocks, odd sizes
        dict(name="gated_backward_ragged", op="gated_backward", layout="uneven", ranks=15, m=2501, k=1999, n=1777, act="gelu_tanh"),
        # the projection behind the block: its gradients, the weight's in fp32 for the optimiser
        dict(name="linear_backward_down", op="linear_backward", layout="row_col", ranks=8, m=8192, k=8192, n=4096, db_dtype="f32"),
        # misaligned odd blocks
        dict(name="linear_backward_ragged", op="linear_backward", layout="uneven", ranks=15, m=1999, k=2731, n=1021, db_dtype="bf16"),
    ]


def draw(rng):
    """One more case of the ranges above: sizes spread over their logarithm, most of them odd or ragged."""
    def size(lo, hi):
        x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        step = rng.choice((1, 1, 8, 64, 128))
        return max(lo, min(hi, (x + step - 1) // step * step))

    def most(case, names, cost, limit):
        # the largest size is halved until the case costs no more than the limit
        while cost(case) > limit:
            big = max(names, key=lambda d: case[d])
            case[big] = case[big] // 2
        return case

    def product(c):
        return 2.0 * c["m"] * c["k"] * c["n"]

    def dealt(case):
        layout = rng.choice(("column", "row_col", "2x2", "uneven"))
        return dict(case, layout=layout, ranks=15 if layout == "uneven" else 4 if layout == "2x2" else 8)

    act = rng.choice(("silu", "silu", "gelu", "gelu_tanh"))
    kind = rng.choice(("quantize", "quantize", "product_token", "product", "product", "product_long", "product_replicated", "gated_i8_token", "gated_i8",
                       "gated_token", "gated", "gated", "gated_backward", "gated_backward", "linear_backward", "linear_backward"))
    if kind == "quantize":
        return most(dict(op="quantize", layout=rng.choice(("1x1", "1x8", "4x2", "uneven")), rows=size(1, 16384), cols=size(32, 28672),
                         dtype=rng.choice(("bf16", "f32")), along=rng.choice(("rows", "cols"))), ("rows", "cols"), lambda c: c["rows"] * c["cols"], 8192 * 16384)
    c_dtype = rng.choice(("bf16", "f32"))
    if kind == "product_token":
        return dict(op="product", layout=rng.choice(("column", "row_col")), ranks=8, m=size(1, 64), k=size(1024, 16384), n=size(1024, 28672), c_dtype=c_dtype)
    if kind == "product":
        return most(dealt(dict(op="product", m=size(64, 16384), k=size(512, 16384), n=size(512, 28672), c_dtype=c_dtype)), "mkn", product, 7e12)
    if kind == "product_long":
        return dict(op="product", layout=rng.choice(("row_col", "2x2")), ranks=rng.choice((4, 8)), m=size(64, 1536), k=size(8192, 49152), n=size(64, 1536),
                    c_dtype=c_dtype)
    if kind == "product_replicated":
        return dict(op="product", layout="replicated", ranks=8, m=size(512, 6144), k=size(512, 8192) // 2 * 2, n=size(512, 6144), c_dtype="f32")
    if kind == "gated_i8_token":
        return dict(op="gated_i8", layout="column", ranks=8, m=size(1, 64), k=size(1024, 16384), n=size(1024, 28672), act=act)
    if kind == "gated_i8":
        return most(dealt(dict(op="gated_i8", m=size(64, 8192), k=size(512, 16384), n=size(512, 28672), act=act)), "mkn", product, 4e12)
    if kind == "gated_token":
        return dict(op="gated", layout="column", ranks=8, m=size(1, 64), k=size(1024, 16384), n=size(1024, 28672), act=act, keep=False)
    if kind == "gated":
        return most(dealt(dict(op="gated", m=size(64, 8192), k=size(512, 16384), n=size(512, 28672), act=act, keep=rng.choice((True, False)))),
                    "mkn", product, 4e12)
    if kind == "gated_backward":
        return most(dealt(dict(op="gated_backward", m=size(32, 8192), k=size(256, 8192), n=size(256, 16384), act=act)), "mkn", product, 1e12)
    return most(dealt(dict(op="linear_backward", m=size(32, 8192), k=size(256, 16384), n=size(256, 16384), db_dtype=c_dtype)), "mkn", product, 2e12)


# ---- partitionings ---------------------------------------------------------------------------------

def _cuts(n, parts):
    size = -(-n // parts)
    return tuple(min(i * size, n) for i in range(parts + 1))


def _uneven(n, parts):
    """Cuts that fall on no regular grid: the parts grow like 2 : 3 : 4 ..."""
    total = parts * (parts + 3) // 2
    return tuple(n * (i * (i + 3) // 2) // total for i in range(parts)) + (n,)


def _desc(rows, cols, row_cuts, col_cuts, replication=1):
    return dict(rows=rows, cols=cols, row_cuts=row_cuts, col_cuts=col_cuts, proc_rows=len(row_cuts) - 1,
                proc_cols=len(col_cuts) - 1, replication=replication)


def _matrix(layout, rows, cols):
    """One matrix, its tile grid by name."""
    if layout == "uneven":
        return _desc(rows, cols, _uneven(rows, 3), _uneven(cols, 2))
    r, c = (int(x) for x in layout.split("x"))
    return _desc(rows, cols, _cuts(rows, r), _cuts(cols, c))


def _product_descs(case):
    m, k, n, p, layout = (case[x] for x in ("m", "k", "n", "ranks", "layout"))
    r, q = (4, 2) if p == 8 else (2, 2)
    if layout == "column":          # A on every rank, B and C in column blocks
        return _desc(m, k, (0, m), (0, k), p), _desc(k, n, (0, k), _cuts(n, p)), _desc(m, n, (0, m), _cuts(n, p))
    if layout == "row_col":         # row blocks times column blocks, C in 2-D blocks
        return _desc(m, k, _cuts(m, p), (0, k)), _desc(k, n, (0, k), _cuts(n, p)), _desc(m, n, _cuts(m, r), _cuts(n, q))
    if layout == "2x2":             # 2-D blocks throughout
        return _desc(m, k, _cuts(m, r), _cuts(k, q)), _desc(k, n, _cuts(k, r), _cuts(n, q)), _desc(m, n, _cuts(m, r), _cuts(n, q))
    if layout == "uneven":          # 3 x 5, 4 x 2 and 5 x 3 uneven blocks
        return (_desc(m, k, _uneven(m, 3), _uneven(k, 5)), _desc(k, n, _uneven(k, 4), _uneven(n, 2)), _desc(m, n, _uneven(m, 5), _uneven(n, 3)))
    # 2.5D: all three matrices twice, every replica of C sums over half of k
    return (_desc(m, k, _cuts(m, 2), _cuts(k, 2), 2), _desc(k, n, _cuts(k, 2), _cuts(n, 2), 2), _desc(m, n, _cuts(m, 2), _cuts(n, 2), 2))


def _bounds(d):
    return [(r0, r1, c0, c1) for r0, r1 in zip(d["row_cuts"], d["row_cuts"][1:]) for c0, c1 in zip(d["col_cuts"], d["col_cuts"][1:])]


def _split(X, d):
    """The tiles of one replica, each a buffer of its own."""
    return [X[r0:r1, c0:c1].contiguous() for r0, r1, c0, c1 in _bounds(d)]


def _join(tiles, d):
    gc = len(d["col_cuts"]) - 1
    return torch.cat([torch.cat(tiles[i:i + gc], 1) for i in range(0, (len(d["row_cuts"]) - 1) * gc, gc)], 0)


def _replicas(tiles, d):
    """The tiles of all replicas, each a buffer of its own."""
    return tiles + [t.clone() for _ in range(d["replication"] - 1) for t in tiles]


def _first(tiles, d):
    """The matrix that replica 0 holds, in fp32."""
    return _join(tiles[:len(_bounds(d))], d).float()


def _empty_tiles(d, dtype, replicas=None):
    return [torch.empty((r1 - r0, c1 - c0), dtype=dtype, device="cuda") for r0, r1, c0, c1 in _bounds(d) * (replicas or d["replication"])]


def _torch_type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---- the operators in elementary operations --------------------------------------------------------

def _quantize(X):
    """Integers and scales of the rows of X."""
    top = X.double().abs().amax(1, keepdim=True)
    q = torch.round(X.double() * 127 / torch.where(top > 0, top, 1.0))
    return q.to(torch.int8), (top / 127).float().squeeze(1)


def _values(q, s, along):
    return q.double() * (s.double().unsqueeze(1) if along == "rows" else s.double())


def _sums(a, b):
    """The product of two integer matrices, exactly."""
    total = 0
    for k in range(0, a.shape[1], CHUNK):
        total = total + torch.matmul(a[:, k:k + CHUNK].float(), b[k:k + CHUNK].float()).double()
    return total


def _activate(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1 + torch.erf(g * 2 ** -0.5))
    return 0.5 * g * (1 + torch.tanh((2 / math.pi) ** 0.5 * (g + 0.044715 * g ** 3)))


def _slope(g, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(g * 2 ** -0.5)) + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    t = torch.tanh((2 / math.pi) ** 0.5 * (g + 0.044715 * g ** 3))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * (2 / math.pi) ** 0.5 * (1 + 0.134145 * g * g)


# ---- inputs ----------------------------------------------------------------------------------------

def _signal(rows, cols, gen, dtype, size=1.0):
    """Activations or gradients: normal values whose columns differ in size."""
    X = torch.randn(rows, cols, generator=gen, device="cuda")
    X *= size * torch.exp(0.7 * torch.randn(1, cols, generator=gen, device="cuda"))
    return X.to(dtype)


def _weight(k, n, gen):
    return (torch.randn(k, n, generator=gen, device="cuda") * k ** -0.5).to(torch.bfloat16)


def _inputs(case, seed):
    """What the seed decides, as whole matrices."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    if op == "quantize":
        return (_signal(case["rows"], case["cols"], gen, _torch_type(case["dtype"])),)
    m, k, n = case["m"], case["k"], case["n"]
    A = _signal(m, k, gen, torch.bfloat16, 0.6)
    if op in ("product", "linear_backward"):
        B = _weight(k, n, gen)
        return (A, B) if op == "product" else (A, B, _signal(m, n, gen, torch.bfloat16, 1e-3))
    Wg, Wu = _weight(k, n, gen), _weight(k, n, gen)
    if op != "gated_backward":
        return A, Wg, Wu
    return A, Wg, Wu, A @ Wg, A @ Wu, _signal(m, n, gen, torch.bfloat16, 1e-3)


class _Int8:
    """A matrix in 8-bit integers along its rows or its columns: the integers of every tile (along the columns a tile
    lies transposed, so that a row of them is a column of the matrix), and the scales of every row (column) of tiles."""

    def __init__(self, X, d, along):
        q, s = _quantize(X if along == "rows" else X.t())
        cuts = d["row_cuts"] if along == "rows" else d["col_cuts"]
        self.along = along
        self.q = _replicas([q[r0:r1, c0:c1].contiguous() if along == "rows" else q[c0:c1, r0:r1].contiguous() for r0, r1, c0, c1 in _bounds(d)], d)
        scales = [s[i:j].contiguous() for i, j in zip(cuts, cuts[1:])]
        self.s = scales + [t.clone() for _ in range(d["replication"] - 1) for t in scales]

    def whole(self, d):
        """Integers (in the matrix' own orientation) and scales."""
        tiles = self.q[:len(_bounds(d))]
        n = len(d["row_cuts"] if self.along == "rows" else d["col_cuts"]) - 1
        return _join(tiles if self.along == "rows" else [t.t() for t in tiles], d), torch.cat(self.s[:n])


def prepare(case, seed):
    """The tiles on the GPU; the plans, descriptors and argument tables that a program keeps."""
    op = case["op"]
    given = _inputs(case, seed)
    state = dict(case=case, op=op)
    if op == "quantize":
        d = _matrix(case["layout"], case["rows"], case["cols"])
        state.update(d=d, x=_split(given[0], d))
    else:
        da, db, dc = descs = _product_descs(case)
        state["descs"] = descs
        if op in ("product", "gated_i8"):
            state["a"] = _Int8(given[0], da, "rows")
            state["b"] = [_Int8(B, db, "cols") for B in given[1:]]
        else:
            state["a"] = _replicas(_split(given[0], da), da)
            weights = 1 if op == "linear_backward" else 2
            state["b"] = [_replicas(_split(B, db), db) for B in given[1:1 + weights]]
            state["c"] = [_split(C, dc) for C in given[1 + weights:]]
    if own:
        _prepare_own(state)
    return state


def _table(binding, tiles):
    return binding.tiles(tiles, [max(t.shape[1], 1) for t in tiles])


def _i8_table(binding, x):
    return binding.int_tiles(x.q, [t.shape[1] for t in x.q], x.s)


def _prepare_own(state):
    from paper_2510_08874_amd import binding
    case, op = state["case"], state["op"]
    state.update(binding=binding, stream=torch.cuda.current_stream().cuda_stream)
    if op == "quantize":
        d, rows = state["d"], case["along"] == "rows"
        q = [torch.empty((r1 - r0, c1 - c0) if rows else (c1 - c0, r1 - r0), dtype=torch.int8, device="cuda") for r0, r1, c0, c1 in _bounds(d)]
        cuts = d["row_cuts"] if rows else d["col_cuts"]
        s = [torch.empty(j - i, dtype=torch.float32, device="cuda") for i, j in zip(cuts, cuts[1:])]
        out = _empty_tiles(d, state["x"][0].dtype)
        state.update(desc=binding.matrix_desc(d), dtype=binding.DMM_BF16 if case["dtype"] == "bf16" else binding.DMM_F32, x_table=_table(binding, state["x"]),
                     q=q, s=s, q_table=binding.int_tiles(q, [t.shape[1] for t in q], s), out=out, out_table=_table(binding, out))
        return
    da, db, dc = state["descs"]
    state["plan"] = binding.Plan(da, db, dc, case["ranks"])
    if "act" in case:
        state["act"] = dict(silu=binding.DMM_SILU, gelu=binding.DMM_GELU, gelu_tanh=binding.DMM_GELU_TANH)[case["act"]]
    if op in ("product", "gated_i8"):
        state["tables"] = [_i8_table(binding, x) for x in (state["a"], *state["b"])]
        state["out"] = _empty_tiles(dc, _torch_type(case.get("c_dtype", "bf16")))
        state.update(out_table=_table(binding, state["out"]), flags=binding.DMM_C_BF16 if case.get("c_dtype", "bf16") == "bf16" else 0)
        return
    state["tables"] = [_table(binding, x) for x in (state["a"], *state["b"], *state["c"])]
    bf16 = torch.bfloat16
    if op == "gated":
        state["out"] = [_empty_tiles(dc, bf16) for _ in range(3 if case["keep"] else 1)]
    elif op == "gated_backward":
        state["out"] = [_empty_tiles(dc, bf16), _empty_tiles(dc, bf16), _empty_tiles(da, bf16, 1), _empty_tiles(db, bf16, 1), _empty_tiles(db, bf16, 1)]
    else:
        state["out"] = [_empty_tiles(da, bf16, 1), _empty_tiles(db, _torch_type(case["db_dtype"]), 1)]
        state["flags"] = binding.DMM_DB_F32 if case["db_dtype"] == "f32" else 0
    state["out_tables"] = [_table(binding, t) for t in state["out"]]


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    """One pass: the tiles of every result."""
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    b, op, stream = state["binding"], state["op"], state["stream"]
    if op == "quantize":
        rows = state["case"]["along"] == "rows"
        b.dmm_int_quantize(state["desc"], state["dtype"], state["x_table"], rows=state["q_table"] if rows else None, cols=None if rows else state["q_table"],
                          stream=stream)
        b.dmm_int_dequantize(state["desc"], state["q_table"], b.DMM_MX_ROWS if rows else b.DMM_MX_COLS, state["dtype"], state["out_table"], stream=stream)
        return state["out"]
    plan, tables = state["plan"], state["tables"]
    if op == "product":
        plan.execute_int(*tables, state["out_table"], state["flags"], stream)
    elif op == "gated_i8":
        plan.gated_int(state["act"], *tables, state["out_table"], stream)
    elif op == "gated":
        h, *kept = state["out_tables"]
        plan.gated(state["act"], *tables, h, *kept, stream=stream)
    elif op == "gated_backward":
        plan.gated_backward(state["act"], *tables, *state["out_tables"], stream=stream)
    else:
        plan.execute_backward(*tables, *state["out_tables"], flags=state["flags"], stream=stream)
    return state["out"]


def _run_plain(state):
    case, op = state["case"], state["op"]
    if op == "quantize":
        d, along = state["d"], case["along"]
        X = _join(state["x"], d)
        q, s = _quantize(X if along == "rows" else X.t())
        return _split(_values(q if along == "rows" else q.t(), s, along).to(X.dtype), d)
    da, db, dc = state["descs"]
    if op in ("product", "gated_i8"):
        (a, sa), b = state["a"].whole(da), [x.whole(db) for x in state["b"]]
        if op == "gated_i8":
            g, u = ((_sums(a, q) * sa.double().unsqueeze(1) * s.double()).float() for q, s in b)
            return _split((_activate(g, case["act"]) * u).bfloat16(), dc)
        (q, s), t = b[0], _torch_type(case["c_dtype"])
        if dc["replication"] == 1:
            return _split((_sums(a, q) * sa.double().unsqueeze(1) * s.double()).to(t), dc)
        # replica 0 has the sum, the others keep their partial sums
        half = case["k"] // 2
        parts = [(_sums(a[:, i], q[i]) * sa.double().unsqueeze(1) * s.double()) for i in (slice(0, half), slice(half, None))]
        return _split((parts[0] + parts[1]).to(t), dc) + _split(parts[1].to(t), dc)
    A, B = _first(state["a"], da), [_first(x, db) for x in state["b"]]
    if op == "gated":
        g, u = torch.matmul(A, B[0]), torch.matmul(A, B[1])
        h = _activate(g, case["act"]) * u
        return [_split(x.bfloat16(), dc) for x in ((h, g, u) if case["keep"] else (h,))]
    if op == "linear_backward":
        dC = _join(state["c"][0], dc).float()
        return [_split(torch.matmul(dC, B[0].t()).bfloat16(), da), _split(torch.matmul(A.t(), dC).to(_torch_type(case["db_dtype"])), db)]
    g, u, dh = (_join(x, dc).float() for x in state["c"])
    dg, du = (dh * u * _slope(g, case["act"])).bfloat16(), (dh * _activate(g, case["act"])).bfloat16()
    dgf, duf = dg.float(), du.float()
    return [_split(dg, dc), _split(du, dc), _split((torch.matmul(dgf, B[0].t()) + torch.matmul(duf, B[1].t())).bfloat16(), da),
            _split(torch.matmul(A.t(), dgf).bfloat16(), db), _split(torch.matmul(A.t(), duf).bfloat16(), db)]


def work(case):
    op = case["op"]
    size = {"bf16": 2.0, "f32": 4.0}
    if op == "quantize":
        # the matrix is read, its integers and scales written, and its values written
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * size[case["dtype"]] + 1) + 4.0 * case["rows" if case["along"] == "rows" else "cols"], "flops": 4.0 * n}
    m, k, n = (float(case[x]) for x in "mkn")
    if op == "product":
        c = 2 if case["layout"] == "replicated" else 1
        return {"bytes": m * k + k * n + 4 * (m + n) + size[case["c_dtype"]] * c * m * n, "flops": 2 * m * k * n}
    if op == "gated_i8":
        return {"bytes": m * k + 2 * k * n + 4 * (m + 2 * n) + 2 * m * n, "flops": 4 * m * k * n}
    if op == "gated":
        return {"bytes": 2 * (m * k + 2 * k * n + (3 if case["keep"] else 1) * m * n), "flops": 4 * m * k * n}
    if op == "gated_backward":
        # A, both weights, G, U and dH are read, a gradient of each but H written
        return {"bytes": 2 * (2 * m * k + 4 * k * n + 5 * m * n), "flops": 8 * m * k * n}
    return {"bytes": 2 * (2 * m * k + k * n + m * n) + size[case["db_dtype"]] * k * n, "flops": 4 * m * k * n}


# ---- the same from the definition, in 64 bits -------------------------------------------------------

def _exact_quantized(X, axis):
    """Every element as the nearest multiple of its row's (column's) scale, half-way ones the even multiple; the scale is a fp32 number."""
    X = X.double()
    top = torch.linalg.vector_norm(X, ord=float("inf"), dim=axis, keepdim=True)
    ratio = (X / top.clamp_min(1e-300)) * 127
    low = torch.floor(ratio)
    rest = ratio - low
    up = (rest > 0.5) | ((rest == 0.5) & (low.remainder(2) == 1))
    # (should the quotient have been rounded onto a half, or off it: twice the distance from the lower multiple decides, both sides exact)
    close = (rest - 0.5).abs() < 1e-9
    twice, border = 254 * X, (2 * low + 1) * top
    up = torch.where(close, (twice > border) | ((twice == border) & (low.remainder(2) == 1)), up)
    return low + up, (top / 127).float().double()


def _exact_act(g, act):
    if act == "silu":
        return g * torch.special.expit(g)
    if act == "gelu":
        return g * torch.special.ndtr(g)
    return g * torch.special.expit(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))


def _exact_slope(g, act):
    if act == "silu":
        p = torch.special.expit(g)
        return p + g * p * torch.special.expit(-g)
    if act == "gelu":
        return torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = 2 * math.sqrt(2 / math.pi)
    p = torch.special.expit(c * (g + 0.044715 * g * g * g))
    return p + g * p * (1 - p) * c * (1 + 3 * 0.044715 * g * g)


def exact(case, seed):
    op = case["op"]
    given = _inputs(case, seed)
    if op == "quantize":
        q, s = _exact_quantized(given[0], 1 if case["along"] == "rows" else 0)
        return _split(q * s, _matrix(case["layout"], case["rows"], case["cols"]))
    da, db, dc = _product_descs(case)
    if op in ("product", "gated_i8"):
        a, sa = _exact_quantized(given[0], 1)
        b = [_exact_quantized(B, 0) for B in given[1:]]
        if op == "gated_i8":
            g, u = ((a @ q) * (sa * s) for q, s in b)
            return _split(_exact_act(g, case["act"]) * u, dc)
        q, s = b[0]
        whole = _split((a @ q) * (sa * s), dc)
        if dc["replication"] == 1:
            return whole
        upper = case["k"] // 2
        return whole + _split((a[:, upper:] @ q[upper:]) * (sa * s), dc)
    X = [x.double() for x in given]
    if op == "gated":
        g, u = X[0] @ X[1], X[0] @ X[2]
        return [_split(x, dc) for x in ((_exact_act(g, case["act"]) * u, g, u) if case["keep"] else (_exact_act(g, case["act"]) * u,))]
    if op == "linear_backward":
        return [_split(X[2] @ X[1].t(), da), _split(X[0].t() @ X[2], db)]
    A, Wg, Wu, g, u, dh = X
    dg, du = dh * u * _exact_slope(g, case["act"]), dh * _exact_act(g, case["act"])
    rg, ru = dg.bfloat16().double(), du.bfloat16().double()
    return [_split(dg, dc), _split(du, dc), _split(rg @ Wg.t() + ru @ Wu.t(), da), _split(A.t() @ rg, db), _split(A.t() @ ru, db)]
