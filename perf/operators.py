"""The layer operators around the sparse x dense product, as cases that can be timed: the product with bias, activation
and residual in its epilogue, the gated pair of products, the backward pass of both, and the product of two dense
matrices sampled at the stored cells. A case's inputs, one pass in plain torch operations or through the library's
entry points (`own`), the result in 64 bits, and the bytes and operations that a pass cannot do without.

Matrices come in two laws. "weights": a pruned weight matrix, cells kept at random with a given density, some rows
pruned away altogether. "graph": a power-law adjacency matrix (row lengths min(Zipf(1.8), cap), uniform columns). Dense
operands are row-major with the features of one layer as rows and the tokens (or the channels of a graph's nodes) as columns.
"""
import math

import numpy as np
import torch

own = False

ZIPF_S, ZIPF_CAP = 1.8, 10_000                 # row lengths of the power-law matrices
EMPTY_EVERY = 37                               # every 37th row of a pruned weight matrix holds nothing
TYPES = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f64": 8, "f32": 4, "bf16": 2, "f16": 2}
OPS = ("epilogue", "gated", "epilogue_backward", "gated_backward", "sddmm")
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # the smallest layer that a loop calls for one vector: launches and latency are what it costs
        {"name": "epilogue-vector-small", "op": "epilogue", "law": "weights", "rows": 4096, "cols": 4096, "density": 1 / 256, "dtype": "f64",
         "R": 1, "act": "relu", "bias": "rows", "residual": False, "preact": False},
        # serving a handful of sequences: the pruned projection back to the residual stream, one token of each
        {"name": "epilogue-tokens", "op": "epilogue", "law": "weights", "rows": 4096, "cols": 16384, "density": 0.1, "dtype": "bf16",
         "R": 8, "act": "none", "bias": "rows", "residual": True, "preact": False},
        # the same projection over a prompt
        {"name": "epilogue-prompt", "op": "epilogue", "law": "weights", "rows": 4096, "cols": 16384, "density": 0.1, "dtype": "bf16",
         "R": 500, "act": "none", "bias": "rows", "residual": True, "preact": False},
        # a graph layer: features aggregated over the neighbours, one bias per channel, the pre-activation kept for training
        {"name": "epilogue-features", "op": "epilogue", "law": "graph", "rows": 170_003, "cols": 170_003, "density": 0.0, "dtype": "f32",
         "R": 50, "act": "relu", "bias": "cols", "residual": False, "preact": True},
        # one token through both projections of a pruned feed-forward block
        {"name": "gated-token", "op": "gated", "law": "weights", "rows": 16384, "cols": 4096, "density": 0.1, "dtype": "bf16",
         "R": 1, "act": "silu", "bias": "none", "preact": False},
        # training step of a block of half the width, pre-activations kept
        {"name": "gated-prompt", "op": "gated", "law": "weights", "rows": 8192, "cols": 2048, "density": 0.2, "dtype": "f16",
         "R": 1000, "act": "gelu_tanh", "bias": "rows", "preact": True},
        # gradients of a small layer in double precision, odd sizes
        {"name": "epilogue-backward-small", "op": "epilogue_backward", "law": "weights", "rows": 1003, "cols": 1501, "density": 0.05, "dtype": "f64",
         "R": 33, "act": "gelu", "bias": "rows"},
        # gradients of the graph layer: edge weights, features and channel biases
        {"name": "epilogue-backward-features", "op": "epilogue_backward", "law": "graph", "rows": 170_003, "cols": 170_003, "density": 0.0, "dtype": "f32",
         "R": 50, "act": "relu", "bias": "cols"},
        # gradients of the gated block over a batch of tokens
        {"name": "gated-backward-prompt", "op": "gated_backward", "law": "weights", "rows": 8192, "cols": 2048, "density": 0.2, "dtype": "bf16",
         "R": 512, "act": "silu", "bias": "rows"},
        # the same in fp32 at odd sizes
        {"name": "gated-backward-odd", "op": "gated_backward", "law": "weights", "rows": 2051, "cols": 1027, "density": 0.05, "dtype": "f32",
         "R": 129, "act": "gelu", "bias": "rows"},
        # scores of a layer at a random pattern of cells
        {"name": "sddmm-pattern", "op": "sddmm", "law": "weights", "rows": 4096, "cols": 4096, "density": 0.1, "dtype": "bf16", "R": 128},
        # an edge score for every edge of a large graph
        {"name": "sddmm-graph", "op": "sddmm", "law": "graph", "rows": 1_048_576, "cols": 1_048_576, "density": 0.0, "dtype": "f32", "R": 64},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    case = {"op": op, "law": rng.choice(["weights", "weights", "graph"]), "dtype": rng.choice(["bf16", "bf16", "f16", "f32", "f32", "f64"])}
    if case["law"] == "weights":
        case["rows"], case["cols"] = _log_uniform(rng, 200, 16384), _log_uniform(rng, 200, 16384)
        if rng.random() < 0.5:
            case["rows"], case["cols"] = (max(64, 64 * round(n / 64)) for n in (case["rows"], case["cols"]))
        # the share of kept cells, so that a matrix has no more entries than the largest listed one
        case["density"] = min(round(math.exp(rng.uniform(math.log(0.01), math.log(0.5))), 4), 6_700_000 / (case["rows"] * case["cols"]))
        widest = 1000
    else:
        case["rows"], case["density"] = _log_uniform(rng, 2000, 1_000_000), 0.0
        case["cols"] = max(1000, int(case["rows"] * rng.uniform(0.5, 1.2)))
        widest = 128
    entries = _entries(case)
    widest = max(1, min(widest, int(3.3e9 / (entries * (2 if op.startswith("gated") else 1)))))
    r = _log_uniform(rng, 1, widest)
    case["R"] = r if r < 16 or rng.random() < 0.5 else 8 * (r // 8)
    if op != "sddmm":
        case["act"] = rng.choice(ACTS)
        case["bias"] = rng.choice(["rows", "none"] if op.startswith("gated") else ["rows", "cols", "none"])
    if op == "epilogue":
        case["residual"] = rng.random() < 0.5
    if op in ("epilogue", "gated"):
        case["preact"] = rng.random() < 0.3
    return case


# ------------------------------------------------------------------------------------------------- inputs

def _zipf_law(case):
    cap = max(1, min(ZIPF_CAP, case["cols"] // 4))
    k = np.arange(1, cap, dtype=np.float64)
    zeta = float(np.sum(np.arange(1, 200_000, dtype=np.float64) ** -ZIPF_S)) + 200_000.0 ** (1 - ZIPF_S) / (ZIPF_S - 1)
    return k ** -ZIPF_S / zeta


def _lengths(case):
    """Row lengths of a power-law matrix: the law's quantiles, the tail beyond the cap lumped on it."""
    u = (np.arange(case["rows"]) + 0.5) / case["rows"]
    return np.searchsorted(np.cumsum(_zipf_law(case)), u, side="right") + 1


def _entries(case):
    """Stored cells of one matrix of a case."""
    rows, cols = case["rows"], case["cols"]
    if case["law"] == "weights":
        return max(1, int((rows - (rows + EMPTY_EVERY - 1) // EMPTY_EVERY) * cols * case["density"]))
    return int(_lengths(case).sum())


def _matrix(case, gen):
    """A matrix in CSR: int32 row boundaries and columns, values of the case's type."""
    rows, cols = case["rows"], case["cols"]
    n = _entries(case)
    if case["law"] == "weights":
        kept = torch.arange(rows, device="cuda")
        kept = kept[kept % EMPTY_EVERY != 0]
        cells = torch.randperm(kept.numel() * cols, generator=gen, device="cuda")[:n].sort().values
        cells = kept[cells // cols] * cols + cells % cols
        scale = 1.0 / math.sqrt(max(1.0, cols * case["density"]))
    else:                                      # a row's columns: consecutive places, from a random one on, of a random order of the columns
        length = torch.from_numpy(_lengths(case)).cuda()[torch.randperm(rows, generator=gen, device="cuda")]
        row = torch.repeat_interleave(torch.arange(rows, device="cuda"), length, output_size=n)
        first = torch.randint(0, cols, (rows,), generator=gen, device="cuda") - (torch.cumsum(length, 0) - length)
        place = (first[row] + torch.arange(n, device="cuda")) % cols
        cells = (row * cols + torch.randperm(cols, generator=gen, device="cuda")[place]).sort().values
        scale = 0.25
    row, col = cells // cols, cells % cols
    pos = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    pos[1:] = torch.cumsum(torch.bincount(row, minlength=rows), 0)
    val = (torch.randn(cells.numel(), generator=gen, device="cuda") * scale).to(TYPES[case["dtype"]])
    m = {"rows": rows, "cols": cols, "pos": pos, "crd": col.to(torch.int32), "val": val}
    if own:                                    # what a program keeps of its weights: the descriptor, and the structure of the transpose for training
        import paper_2102_05187_b200 as comet
        m["A"] = comet.SpTensor.from_arrays((rows, cols), (0, 1), (comet.D, comet.CU), [torch.full((1,), rows, dtype=torch.int32, device="cuda"), pos],
                                            [None, m["crd"]], val)
        if case["op"].endswith("backward"):
            m["At"] = comet.transpose_symbolic(m["A"])
    return m


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, cols, R, dt, op = case["rows"], case["cols"], case["R"], TYPES[case["dtype"]], case["op"]

    def dense(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dt)

    s = {"case": dict(case), "A": _matrix(case, gen)}
    if op.startswith("gated"):
        s["U"] = _matrix(case, gen)
    if op == "sddmm":
        s["P"], s["Q"] = dense(rows, R, scale=R ** -0.5), dense(cols, R)
        s["out"] = torch.empty(s["A"]["val"].numel(), dtype=dt, device="cuda")
        return s
    s["B"] = dense(cols, R)
    if op.endswith("backward"):
        s["dC"] = dense(rows, R)
        s["Z"] = dense(rows, R)                # the pre-activations that the forward pass kept
        if op == "gated_backward":
            s["Zu"] = dense(rows, R)
        return s
    if case["bias"] != "none":
        s["bias"] = dense(rows if case["bias"] == "rows" else R, scale=0.5)
        if op == "gated":
            s["bias_u"] = dense(rows, scale=0.5)
    if case.get("residual"):
        s["residual"] = dense(rows, R)
    s["C"] = torch.empty(rows, R, dtype=dt, device="cuda")
    if case["preact"]:
        s["Z"] = torch.empty_like(s["C"])
        if op == "gated":
            s["Zu"] = torch.empty_like(s["C"])
    return s


# ------------------------------------------------------------------------------------------------- plain form

def _wide(t):
    return t.double() if t.dtype == torch.float64 else t.float()


def _row_of(m):
    return torch.repeat_interleave(torch.arange(m["rows"], device="cuda"), m["pos"].diff(), output_size=m["crd"].numel())


def _product(m, dense, transposed=False):
    """A @ dense (or A^T @ dense) over the stored cells, not rounded."""
    to, of = _row_of(m), m["crd"].long()
    if transposed:
        to, of = of, to
    out = dense.new_zeros(m["cols"] if transposed else m["rows"], dense.shape[1])
    return out.index_add_(0, to, dense[of] * _wide(m["val"])[:, None])


def _sampled(m, left, right):
    """sum_r left[row, r] right[col, r] for every stored cell."""
    return (left[_row_of(m)] * right[m["crd"].long()]).sum(1)


def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        g = 1 / (1 + torch.exp(-z))
        return g * (1 + z * (1 - g))
    return torch.ones_like(z)


def _plain(s):
    case, op, A = s["case"], s["case"]["op"], s["A"]
    dt = TYPES[case["dtype"]]
    if op == "sddmm":
        return _sampled(A, _wide(s["P"]), _wide(s["Q"])).to(dt)
    act, B = case["act"], _wide(s["B"])
    if op == "epilogue":
        z = _product(A, B)
        if case["bias"] != "none":
            z = z + (_wide(s["bias"])[:, None] if case["bias"] == "rows" else _wide(s["bias"])[None, :])
        c = _act(act, z)
        if case["residual"]:
            c = c + _wide(s["residual"])
        return {"C": c.to(dt), "Z": z.to(dt)} if case["preact"] else {"C": c.to(dt)}
    if op == "gated":
        zg, zu = _product(A, B), _product(s["U"], B)
        if case["bias"] != "none":
            zg, zu = zg + _wide(s["bias"])[:, None], zu + _wide(s["bias_u"])[:, None]
        out = {"C": (_act(act, zg) * zu).to(dt)}
        return {**out, "Zg": zg.to(dt), "Zu": zu.to(dt)} if case["preact"] else out
    dC, z = _wide(s["dC"]), _wide(s["Z"])
    if op == "epilogue_backward":
        dz = dC * _act_slope(act, z)
        out = {"dval": _sampled(A, dz, B).to(dt), "dB": _product(A, dz, transposed=True).to(dt)}
        return {**out, "dbias": dz.sum(1 if case["bias"] == "rows" else 0).to(dt)} if case["bias"] != "none" else out
    zu = _wide(s["Zu"])
    dg, du = dC * zu * _act_slope(act, z), dC * _act(act, z)
    out = {"dval_g": _sampled(A, dg, B).to(dt), "dval_u": _sampled(s["U"], du, B).to(dt),
           "dB": (_product(A, dg, transposed=True) + _product(s["U"], du, transposed=True)).to(dt)}
    return {**out, "dbias_g": dg.sum(1).to(dt), "dbias_u": du.sum(1).to(dt)} if case["bias"] != "none" else out


# ------------------------------------------------------------------------------------------------- the library's calls

def _own(s):
    import paper_2102_05187_b200 as comet
    case, op, A = s["case"], s["case"]["op"], s["A"]["A"]
    if op == "sddmm":
        comet.sddmm(A, s["P"], s["Q"], out_val=s["out"])
        return s["out"]
    act = {"none": comet.ACT_NONE, "relu": comet.ACT_RELU, "gelu": comet.ACT_GELU, "gelu_tanh": comet.ACT_GELU_TANH, "silu": comet.ACT_SILU}[case["act"]]
    along = {"none": None, "rows": comet.BIAS_ROWS, "cols": comet.BIAS_COLS}[case["bias"]]
    if op == "epilogue":
        comet.spmm_epilogue(A, s["B"], act=act, bias=s.get("bias"), bias_along=along, residual=s.get("residual"), preact=s.get("Z"), out=s["C"])
        return {"C": s["C"], "Z": s["Z"]} if case["preact"] else {"C": s["C"]}
    if op == "gated":
        comet.spmm_gated(A, s["U"]["A"], s["B"], act=act, bias_g=s.get("bias"), bias_u=s.get("bias_u"),
                         preact=(s["Z"], s["Zu"]) if case["preact"] else None, out=s["C"])
        return {"C": s["C"], "Zg": s["Z"], "Zu": s["Zu"]} if case["preact"] else {"C": s["C"]}
    if op == "epilogue_backward":
        dval, dB, dbias = comet.spmm_epilogue_backward(A, s["A"]["At"], s["B"], s["dC"], act=act, preact=s["Z"], bias_along=along)
        out = {"dval": dval, "dB": dB}
        return {**out, "dbias": dbias} if case["bias"] != "none" else out
    dval_g, dval_u, dB, dbias_g, dbias_u = comet.spmm_gated_backward(A, s["A"]["At"], s["U"]["A"], s["U"]["At"], s["B"], s["dC"], (s["Z"], s["Zu"]), act=act,
                                                                     need_bias=along is not None)
    out = {"dval_g": dval_g, "dval_u": dval_u, "dB": dB}
    return {**out, "dbias_g": dbias_g, "dbias_u": dbias_u} if case["bias"] != "none" else out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work and the result in 64 bits

def work(case):
    rows, cols, R, es, n, op = case["rows"], case["cols"], case["R"], BYTES[case["dtype"]], _entries(case), case["op"]
    sides = 2 if op.startswith("gated") else 1
    index, values, x, y = 4 * n + 4 * (rows + 1), n * es, cols * R * es, rows * R * es
    bias = 0 if case.get("bias", "none") == "none" else es * (R if case["bias"] == "cols" else rows)
    if op == "sddmm":
        return {"bytes": index + values + x + y, "flops": 2 * n * R}
    if op in ("epilogue", "gated"):
        return {"bytes": sides * (index + values + bias) + x + y * (1 + bool(case.get("residual")) + sides * bool(case["preact"])), "flops": 2 * n * R * sides}
    transposed = 8 * n + 4 * (cols + 1)        # the structure of the transpose: a row number and an entry number for each stored cell
    return {"bytes": sides * (index + 2 * values + transposed + bias + y) + y + 2 * x, "flops": 4 * n * R * sides}


def _cells64(m):
    """Row and column numbers of the stored cells, from the row boundaries by search."""
    at = torch.arange(m["crd"].numel(), device="cuda")
    return torch.searchsorted(m["pos"].long(), at, right=True) - 1, m["crd"].long()


def _matmul64(m, dense, turned=False):
    i, j = _cells64(m)
    v, dense = m["val"].double(), dense.double()
    if turned:
        i, j = j, i
    shape = (m["cols"], m["rows"]) if turned else (m["rows"], m["cols"])
    if shape[0] * shape[1] <= 1 << 27:
        full = torch.zeros(shape, dtype=torch.float64, device="cuda")
        full[i, j] = v
        return full @ dense
    return torch.sparse.mm(torch.sparse_coo_tensor(torch.stack([i, j]), v, shape).coalesce(), dense)


def _cells_dot64(m, left, right):
    i, j = _cells64(m)
    left, right = left.double().t().contiguous(), right.double().t().contiguous()
    out = torch.zeros(i.numel(), dtype=torch.float64, device="cuda")
    for p, q in zip(left, right):
        out.addcmul_(p[i], q[j])
    return out


def _layer64(name, z):
    f = torch.nn.functional
    return {"none": lambda t: t * 1.0, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh"), "silu": f.silu}[name](z)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    A = s["A"]
    if op == "sddmm":
        return _cells_dot64(A, s["P"], s["Q"])
    if op in ("epilogue", "gated"):
        z = _matmul64(A, s["B"])
        if case["bias"] != "none":
            z += s["bias"].double().view((-1, 1) if case["bias"] == "rows" else (1, -1))
        if op == "epilogue":
            c = _layer64(case["act"], z) + (s["residual"].double() if case["residual"] else 0.0)
            return {"C": c, "Z": z} if case["preact"] else {"C": c}
        zu = _matmul64(s["U"], s["B"])
        if case["bias"] != "none":
            zu += s["bias_u"].double().view(-1, 1)
        c = _layer64(case["act"], z) * zu
        return {"C": c, "Zg": z, "Zu": zu} if case["preact"] else {"C": c}
    leaves = [s["Z"].double().requires_grad_()] + ([s["Zu"].double().requires_grad_()] if op == "gated_backward" else [])
    c = _layer64(case["act"], leaves[0])
    for u in leaves[1:]:
        c = c * u
    dz = torch.autograd.grad(c, leaves, s["dC"].double())
    if op == "epilogue_backward":
        out = {"dval": _cells_dot64(A, dz[0], s["B"]), "dB": _matmul64(A, dz[0], turned=True)}
        return {**out, "dbias": dz[0].sum(1 if case["bias"] == "rows" else 0)} if case["bias"] != "none" else out
    out = {"dval_g": _cells_dot64(A, dz[0], s["B"]), "dval_u": _cells_dot64(s["U"], dz[1], s["B"]),
           "dB": _matmul64(A, dz[0], turned=True) + _matmul64(s["U"], dz[1], turned=True)}
    return {**out, "dbias_g": dz[0].sum(1), "dbias_u": dz[1].sum(1)} if case["bias"] != "none" else out
