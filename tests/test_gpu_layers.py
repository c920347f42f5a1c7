"""The layer operators against their definitions in 64 bits: products with bias, activation and residual in the epilogue, gated pairs, the
sampled product, the gradients (against the formula and against differences), empty and very long rows, formats, strides,
alignments, infinities outside the stored cells, streams, captured graphs and a block run as it would be used."""
import ctypes as C

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import (ACTS, TYPES, Matrix, act64, act_bound, assert_within, place, random_mask, slope64, stored, u_of, values,  # noqa: E402
                        z_bound)


def check_epilogue(m, dt, R, act, bias, residual, preact, rng, pad=0, off=0):
    rows, cols = m.mask.shape
    B, B64 = values((cols, R), dt, rng)
    kw, b64 = {}, torch.zeros(rows, 1, dtype=torch.float64)
    if bias != "none":
        b, b64 = values(rows if bias == "rows" else R, dt, rng, 0.5)
        kw.update(bias=b.cuda(), bias_along=comet.BIAS_ROWS if bias == "rows" else comet.BIAS_COLS)
        b64 = b64.view(-1, 1) if bias == "rows" else b64.view(1, -1)
    r64 = torch.zeros(1, dtype=torch.float64)
    if residual:
        r, r64 = values((rows, R), dt, rng)
        kw["residual"] = place(r, pad, off)
    out = place(torch.full((rows, R), float("nan"), dtype=dt), pad, off, fill=7.0)
    pre = place(torch.full((rows, R), float("nan"), dtype=dt), pad, off, fill=7.0) if preact else None
    got = comet.spmm_epilogue(m.t, place(B, pad, off), act=ACTS[act], preact=pre, out=out, **kw)
    z = m.dense @ B64 + b64
    N = m.dense.abs() @ B64.abs() + b64.abs()
    dz = z_bound(dt, m.longest, N, z)
    c = act64(act, z) + r64
    dc = act_bound(dt, dz, z) + 2 * u_of(dt) * (c.abs() + r64.abs())
    assert_within(got, c, stored(dt, c, dc), f"C ({act}, bias {bias})")
    if preact:
        assert_within(pre, z, stored(dt, z, dz), "Z")
    return out, pre, pad


def untouched(view, pad):
    """The padding columns behind a view's rows still hold the fill."""
    if pad:
        rows, R = view.shape
        whole = torch.as_strided(view, (rows, R + pad), view.stride(), view.storage_offset())
        assert bool((whole[:, R:] == 7.0).all()), "padding was written"


SIZES = [  # rows, cols, density, R, pad, off
    (1, 1, 1.0, 1, 0, 0), (5, 3, 0.5, 1, 0, 0), (64, 48, 0.3, 2, 0, 0), (37, 1000, 0.4, 3, 0, 0), (130, 70, 0.2, 7, 1, 0), (100, 90, 0.1, 8, 0, 0),
    (33, 65, 0.5, 16, 8, 8), (257, 129, 0.03, 33, 0, 1), (70, 300, 0.3, 64, 0, 0), (19, 700, 0.9, 100, 4, 0), (50, 40, 0.2, 127, 1, 3),
    (40, 80, 0.25, 129, 0, 0), (24, 200, 0.5, 256, 0, 0), (9, 30, 0.5, 515, 5, 0), (300, 20, 0.02, 1000, 0, 0),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_epilogue_sizes(cuda_device, dtype, size):
    rows, cols, density, R, pad, off = size
    rng = np.random.default_rng(rows * 7 + R)
    m = Matrix(random_mask(rows, cols, density, rng, empty=(0, rows - 1) if rows > 2 else ()), TYPES[dtype], rng, scale=0.3)
    for out, pre, p in [check_epilogue(m, TYPES[dtype], R, "gelu", "rows", True, True, rng, pad, off),
                        check_epilogue(m, TYPES[dtype], R, "none", "none", False, False, rng, pad, off)]:
        untouched(out, p)
        if pre is not None:
            untouched(pre, p)


TILES = [  # rows, cols, density, R: 16-bit matrices that the tensor-core forms take, around the edges of their tiles, with few and many tiles
    (128, 64, 1.0, 64), (128, 64, 0.5, 8), (127, 63, 0.9, 72), (129, 65, 0.4, 128), (1, 512, 1.0, 8), (257, 1000, 0.3, 256), (200, 4096, 0.05, 8),
    (300, 2048, 0.02, 136), (640, 1100, 0.1, 264), (130, 5000, 0.9, 24), (520, 130, 0.6, 520), (1500, 700, 0.05, 1000), (5000, 200, 0.1, 192),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", TILES, ids=lambda s: "x".join(map(str, s)))
def test_tiles(cuda_device, dtype, size):
    rows, cols, density, R = size
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows + cols)
    empty = (0, rows // 2, rows - 1) if rows > 2 else ()
    scale = (cols * density) ** -0.5
    m = Matrix(random_mask(rows, cols, density, rng, empty), dt, rng, scale=scale)
    check_epilogue(m, dt, R, "none", "none", False, False, rng)
    for out, pre, p in [check_epilogue(m, dt, R, "gelu", "rows", True, True, rng, pad=8), check_epilogue(m, dt, R, "silu", "cols", False, True, rng, pad=16)]:
        untouched(out, p)
        if pre is not None:
            untouched(pre, p)
    u = Matrix(random_mask(rows, cols, density / 2, rng, empty[:1]), dt, rng, scale=scale)
    check_gated(m, u, dt, R, "silu", True, rng, pad=8)
    check_gated(u, m, dt, R, "none", False, rng)
    check_backward(m, dt, R, "gelu_tanh", "rows", rng, pad=8)
    P, P64 = values((rows, R), dt, rng)
    Q, Q64 = values((cols, R), dt, rng)
    check_sddmm(m, P, P64, Q, Q64, dt, pad=8)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("R", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("size", [(3000, 900, 0.3), (150, 5000, 0.5), (700, 33_000, 0.05), (20_000, 64, 0.5)], ids=lambda s: "x".join(map(str, s)))
def test_few_columns(cuda_device, dtype, R, size):
    """Matrices with enough entries that B's short rows are laid down in shared memory, in one panel or several."""
    rows, cols, density = size
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows + R)
    m = Matrix(random_mask(rows, cols, density, rng, empty=(0, rows - 1, rows // 2)), dt, rng, scale=(cols * density) ** -0.5)
    check_epilogue(m, dt, R, "silu", "rows", True, True, rng, pad=R % 3)
    u = Matrix(random_mask(rows, cols, density / 2, rng), dt, rng, scale=(cols * density) ** -0.5)
    check_gated(m, u, dt, R, "gelu_tanh", True, rng)
    (B, B64), (dC, dC64), (zg, zg64), (zu, zu64) = (values(s, dt, rng) for s in ((cols, R), (rows, R), (rows, R), (rows, R)))
    if rows >= cols:                                       # the gradient's matrix is the tall one
        dB = comet.spmm_gated_backward(m.t, comet.transpose_symbolic(m.t), u.t, comet.transpose_symbolic(u.t), None, dC.cuda(), (zg.cuda(), zu.cuda()),
                                       act=comet.ACT_NONE, need_val=False)[2]
        dg, du = dC64 * zu64, dC64 * zg64
        want = m.dense.t() @ dg + u.dense.t() @ du
        N = m.dense.abs().t() @ dg.abs() + u.dense.abs().t() @ du.abs()
        e = N * (u_of(dt) * 4 + (torch.finfo(dt).eps / 2 if dt in (torch.bfloat16, torch.float16) else 0))
        assert_within(dB, want, stored(dt, want, 1.01 * e + z_bound(dt, m.tallest + u.tallest, N * 1.01, want)), "dB")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("R", [4, 33, 130])
def test_many_short_rows(cuda_device, dtype, R):
    """Graph-like matrices: more than half a million entries in rows of about 25, some empty, a few long ones."""
    rows, cols, dt = 24_000, 1800, TYPES[dtype]
    rng = np.random.default_rng(R)
    mask = random_mask(rows, cols, 0.0145, rng, empty=(0, rows - 1, *range(500, 560)))
    mask[7], mask[9_001, :1500], mask[rows - 2] = True, True, True
    m = Matrix(mask, dt, rng, scale=0.2)
    for act, bias, residual, preact, pad in [("gelu", "rows", True, True, 1), ("none", "none", False, False, 0), ("relu", "cols", True, False, 8)]:
        out, pre, p = check_epilogue(m, dt, R, act, bias, residual, preact, rng, pad)
        untouched(out, p)
        if pre is not None:
            untouched(pre, p)
    u = Matrix(random_mask(rows, cols, 0.0145, rng), dt, rng, scale=0.2)
    check_gated(m, u, dt, R, "silu", True, rng, pad=2)
    check_gated(u, m, dt, R, "gelu", False, rng)
    B, _ = values((cols, R), dt, rng)
    r = torch.randn(rows, R, device="cuda").to(dt)
    want = comet.spmm_epilogue(m.t, B.cuda(), act=ACTS["silu"], residual=r)
    comet.spmm_epilogue(m.t, B.cuda(), act=ACTS["silu"], residual=r, out=r)
    assert torch.equal(r, want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_of_many_short_columns(cuda_device, dtype, act):
    """The same for dB, whose matrix is the transpose: short columns; and the gated pair's sum of two products."""
    rows, cols, R, dt = 1800, 24_000, 20, TYPES[dtype]
    rng = np.random.default_rng(5)
    m = Matrix(random_mask(rows, cols, 0.0145, rng, empty=(3,)), dt, rng, scale=0.2)
    check_backward(m, dt, R, act, "cols", rng, pad=4)
    u = Matrix(random_mask(rows, cols, 0.0145, rng), dt, rng, scale=0.2)
    (dC, dC64), (zg, zg64), (zu, zu64) = (values((rows, R), dt, rng) for _ in range(3))
    dB = comet.spmm_gated_backward(m.t, comet.transpose_symbolic(m.t), u.t, comet.transpose_symbolic(u.t), None, dC.cuda(), (zg.cuda(), zu.cuda()), act=ACTS[act],
                                   need_val=False)[2]
    dg, du = dC64 * zu64 * slope64(act, zg64), dC64 * act64(act, zg64)
    sg = stored(dt, dg, 28 * u_of(dt) * (dC64 * zu64).abs() * (1 + zg64.abs()))
    su = stored(dt, du, 20 * u_of(dt) * dC64.abs() * zg64.abs())
    want = m.dense.t() @ dg + u.dense.t() @ du
    N = m.dense.abs().t() @ (dg.abs() + sg) + u.dense.abs().t() @ (du.abs() + su)
    bound = m.dense.abs().t() @ sg + u.dense.abs().t() @ su + 2 * z_bound(dt, m.tallest + u.tallest, N, want)     # each product may be rounded before they are added
    assert_within(dB, want, stored(dt, want, bound), "dB")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("bias", ["none", "rows", "cols"])
def test_epilogue_variants(cuda_device, dtype, act, bias):
    rng = np.random.default_rng(5)
    m = Matrix(random_mask(61, 83, 0.2, rng, empty=(3,)), TYPES[dtype], rng)
    for residual, preact in [(False, True), (True, False)]:
        check_epilogue(m, TYPES[dtype], 24, act, bias, residual, preact, rng)


@pytest.mark.parametrize("fmt", ["csr", "dcsr", "coo", "csr10"])
@pytest.mark.parametrize("density", [0.0, 0.002, 0.2])
def test_formats(cuda_device, fmt, density):
    rng = np.random.default_rng(17)
    mask = random_mask(210, 60, density, rng, empty=range(40, 160))
    m = Matrix(mask, torch.float32, rng, fmt)
    check_epilogue(m, torch.float32, 20, "silu", "rows", True, True, rng)
    P, P64 = values((210, 20), torch.float32, rng)
    Q, Q64 = values((60, 20), torch.float32, rng)
    check_sddmm(m, P, P64, Q, Q64, torch.float32)
    At = comet.transpose_symbolic(m.t)
    check_transpose(m, At)


def check_transpose(m, At):
    r, c = m.rc
    order = torch.argsort(c * m.mask.shape[0] + r)         # column by column, rows ascending
    assert At.nnz == r.numel()
    assert torch.equal(At.pos(1).cpu().long(), torch.cat([torch.zeros(1, dtype=torch.long), torch.bincount(c, minlength=m.mask.shape[1]).cumsum(0)]))
    if r.numel():
        assert torch.equal(At.crd(1).cpu().long(), r[order]) and torch.equal(At.val.cpu().long(), order)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("R", [1, 5, 24, 130])
def test_long_rows(cuda_device, dtype, R):
    """Rows around the length from which a CTA shares them out (512), and far beyond it."""
    rng = np.random.default_rng(R)
    mask = random_mask(40, 6000, 0.002, rng)
    for i, n in [(0, 511), (1, 512), (2, 513), (7, 1500), (8, 6000), (9, 6000), (39, 3001)]:
        mask[i] = False
        mask[i, rng.permutation(6000)[:n]] = True
    m = Matrix(mask, TYPES[dtype], rng, scale=0.05)
    check_epilogue(m, TYPES[dtype], R, "none", "rows", False, False, rng)


@pytest.mark.parametrize("dtype", ["f64", "f32", "bf16"])
@pytest.mark.parametrize("R", [1, 12, 70])
def test_huge_rows(cuda_device, dtype, R):
    """Rows of more than 16,384 entries, which are cut into items for launches of their own; the other rows as ever."""
    rng = np.random.default_rng(3 * R)
    cols = 40_000
    mask = random_mask(12, cols, 0.001, rng, empty=(4,))
    for i, n in [(1, 16384), (2, 16385), (6, 40_000), (11, 20_480)]:
        mask[i] = False
        mask[i, rng.permutation(cols)[:n]] = True
    m = Matrix(mask, TYPES[dtype], rng, scale=0.02)
    check_epilogue(m, TYPES[dtype], R, "relu", "cols", True, True, rng)
    u = Matrix(random_mask(12, cols, 0.01, rng), TYPES[dtype], rng, scale=0.02)
    check_gated(m, u, TYPES[dtype], R, "silu", True, rng)
    check_gated(u, m, TYPES[dtype], R, "none", False, rng)


def check_gated(g, u, dt, R, act, full, rng, pad=0, off=0):
    rows, cols = g.mask.shape
    B, B64 = values((cols, R), dt, rng)
    kw, bias64 = {}, [torch.zeros(rows, 1, dtype=torch.float64)] * 2
    pre = None
    if full:
        (bg, bg64), (bu, bu64) = values(rows, dt, rng, 0.5), values(rows, dt, rng, 0.5)
        kw.update(bias_g=bg.cuda(), bias_u=bu.cuda())
        bias64 = [bg64.view(-1, 1), bu64.view(-1, 1)]
        pre = [place(torch.full((rows, R), float("nan"), dtype=dt), pad, off, 7.0) for _ in range(2)]
        kw["preact"] = pre
    out = place(torch.full((rows, R), float("nan"), dtype=dt), pad, off, 7.0)
    comet.spmm_gated(g.t, u.t, place(B, pad, off), act=ACTS[act], out=out, **kw)
    z, dz = [], []
    for m, b in zip((g, u), bias64):
        z.append(m.dense @ B64 + b)
        dz.append(z_bound(dt, m.longest, m.dense.abs() @ B64.abs() + b.abs(), z[-1]))
    f = act64(act, z[0])
    c = f * z[1]
    df = act_bound(dt, dz[0], z[0])
    dc = df * z[1].abs() + (f.abs() + df) * dz[1] + 2 * u_of(dt) * c.abs()
    assert_within(out, c, stored(dt, c, dc), "C")
    untouched(out, pad)
    if pre:
        for q in range(2):
            assert_within(pre[q], z[q], stored(dt, z[q], dz[q]), f"Z{q}")
            untouched(pre[q], pad)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gated_sizes(cuda_device, dtype, size):
    rows, cols, density, R, pad, off = size
    rng = np.random.default_rng(rows * 5 + R)
    g = Matrix(random_mask(rows, cols, density, rng, empty=(0,) if rows > 2 else ()), TYPES[dtype], rng, scale=0.3)
    u = Matrix(random_mask(rows, cols, density / 2, rng), TYPES[dtype], rng, scale=0.3)
    for act, full in [("silu", True), ("gelu_tanh", False)]:
        check_gated(g, u, TYPES[dtype], R, act, full, rng, pad, off)


def check_sddmm(m, P, P64, Q, Q64, dt, pad=0, off=0):
    r, c = m.rc
    R = P.shape[1]
    out = torch.full((r.numel() + 4,), 7.0, dtype=dt, device="cuda")
    comet.sddmm(m.t, place(P, pad, off), place(Q, pad, off), out_val=out[: r.numel()])
    want = (P64[r] * Q64[c]).sum(1)
    N = (P64[r].abs() * Q64[c].abs()).sum(1)
    # fp32: at most 64 terms in a lane, a rounding of its sum, five additions across lanes; the others: R terms at most
    bound = (R + 8) * u_of(dt) * N if dt != torch.float32 else 72 * u_of(dt) * N + u_of(dt) * want.abs()
    assert_within(out[: r.numel()], want, stored(dt, want, bound), "sddmm")
    assert bool((out[r.numel():] == 7.0).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sddmm_sizes(cuda_device, dtype, size):
    rows, cols, density, R, pad, off = size
    rng = np.random.default_rng(rows * 3 + R)
    m = Matrix(random_mask(rows, cols, density, rng, empty=(0, rows - 1) if rows > 2 else ()), TYPES[dtype], rng)
    P, P64 = values((rows, R), TYPES[dtype], rng)
    Q, Q64 = values((cols, R), TYPES[dtype], rng)
    check_sddmm(m, P, P64, Q, Q64, TYPES[dtype], pad, off)


@pytest.mark.parametrize("gap", [1, 30, 31, 32, 33, 100, 1000])
def test_sddmm_runs_of_empty_rows(cuda_device, gap):
    """Stored rows far apart: the search for an entry's row looks past the 32 rows it holds."""
    rng = np.random.default_rng(gap)
    mask = np.zeros((12 * (gap + 1) + 3, 50), dtype=bool)
    mask[gap::gap + 1] = rng.random((mask[gap::gap + 1].shape)) < 0.2
    m = Matrix(mask, torch.float32, rng)
    P, P64 = values((mask.shape[0], 8), torch.float32, rng)
    Q, Q64 = values((50, 8), torch.float32, rng)
    check_sddmm(m, P, P64, Q, Q64, torch.float32)


# ---------------------------------------------------------------------------------------------- gradients

def check_backward(m, dt, R, act, bias, rng, pad=0, off=0):
    rows, cols = m.mask.shape
    (B, B64), (g, g64), (z, z64) = values((cols, R), dt, rng), values((rows, R), dt, rng), values((rows, R), dt, rng)
    along = {"none": None, "rows": comet.BIAS_ROWS, "cols": comet.BIAS_COLS}[bias]
    At = comet.transpose_symbolic(m.t)
    dval, dB, dbias = comet.spmm_epilogue_backward(m.t, At, place(B, pad, off), place(g, pad, off), act=ACTS[act], preact=place(z, pad, off), bias_along=along)
    dz = g64 * slope64(act, z64)
    ddz = 24 * u_of(dt) * g64.abs() * (1 + z64.abs()) if act != "none" else torch.zeros_like(dz)   # evaluating the slope
    check_product_gradients(m, dt, dval, dB, dz, ddz, B64, rounded=act != "none")
    if along is not None:
        dim = 1 if bias == "rows" else 0
        # 8 terms at most in fp32, then double
        bound = ddz.sum(dim) + 10 * u_of(dt) * (dz.abs() + ddz).sum(dim) + u_of(dt) * dz.sum(dim).abs()
        assert_within(dbias, dz.sum(dim), stored(dt, dz.sum(dim), bound), "dbias")


def check_product_gradients(m, dt, dval, dB, dz, ddz, B64, rounded):
    """dval and dB (of one matrix) from dz, which the kernels round to the operands' type where it has an activation's slope in it."""
    r, c = m.rc
    R = B64.shape[1]
    e = stored(dt, dz, ddz) if rounded else ddz
    want = (dz[r] * B64[c]).sum(1)
    N = (dz[r].abs() * B64[c].abs()).sum(1)
    bound = (e[r] * B64[c].abs()).sum(1) + (R + 10) * u_of(dt) * N * 1.01
    assert_within(dval, want, stored(dt, want, bound), "dval")
    if dB is None:
        return None
    want = m.dense.t() @ dz
    N = m.dense.abs().t() @ (dz.abs() + e)
    bound = m.dense.abs().t() @ e + z_bound(dt, m.tallest, N, want)
    assert_within(dB, want, stored(dt, want, bound), "dB")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_epilogue_backward_sizes(cuda_device, dtype, size):
    rows, cols, density, R, pad, off = size
    rng = np.random.default_rng(rows + R)
    m = Matrix(random_mask(rows, cols, density, rng, empty=(0, rows - 1) if rows > 2 else ()), TYPES[dtype], rng, scale=0.3)
    check_backward(m, TYPES[dtype], R, "gelu", "rows", rng, pad, off)
    check_backward(m, TYPES[dtype], R, "none", "cols", rng, pad, off)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("bias", ["none", "rows", "cols"])
def test_epilogue_backward_variants(cuda_device, dtype, act, bias):
    rng = np.random.default_rng(11)
    m = Matrix(random_mask(1300, 40, 0.1, rng, empty=(3,)), TYPES[dtype], rng)
    check_backward(m, TYPES[dtype], 40, act, bias, rng)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gated_backward_sizes(cuda_device, dtype, size):
    rows, cols, density, R, pad, off = size
    dt, act = TYPES[dtype], ["silu", "gelu", "relu", "none", "gelu_tanh"][R % 5]
    rng = np.random.default_rng(rows * 2 + R)
    g = Matrix(random_mask(rows, cols, density, rng, empty=(0,) if rows > 2 else ()), dt, rng, scale=0.3)
    u = Matrix(random_mask(rows, cols, density / 2, rng), dt, rng, scale=0.3)
    (B, B64), (dC, dC64), (zg, zg64), (zu, zu64) = (values(s, dt, rng) for s in ((cols, R), (rows, R), (rows, R), (rows, R)))
    Gt, Ut = comet.transpose_symbolic(g.t), comet.transpose_symbolic(u.t)
    dval_g, dval_u, dB, dbg, dbu = comet.spmm_gated_backward(g.t, Gt, u.t, Ut, place(B, pad, off), place(dC, pad, off),
                                                            (place(zg, pad, off), place(zu, pad, off)), act=ACTS[act], need_bias=True)
    dg, du = dC64 * zu64 * slope64(act, zg64), dC64 * act64(act, zg64)
    eg, eu = 28 * u_of(dt) * (dC64 * zu64).abs() * (1 + zg64.abs()), 20 * u_of(dt) * dC64.abs() * zg64.abs()
    check_product_gradients(g, dt, dval_g, None, dg, eg, B64, True)
    check_product_gradients(u, dt, dval_u, None, du, eu, B64, True)
    want = g.dense.t() @ dg + u.dense.t() @ du
    sg, su = stored(dt, dg, eg), stored(dt, du, eu)
    N = g.dense.abs().t() @ (dg.abs() + sg) + u.dense.abs().t() @ (du.abs() + su)
    bound = g.dense.abs().t() @ sg + u.dense.abs().t() @ su + z_bound(dt, g.tallest + u.tallest, N, want)
    assert_within(dB, want, stored(dt, want, bound), "dB")
    for got, d, e in [(dbg, dg, eg), (dbu, du, eu)]:
        assert_within(got, d.sum(1), stored(dt, d.sum(1), e.sum(1) + 10 * u_of(dt) * (d.abs() + e).sum(1) + u_of(dt) * d.sum(1).abs()), "dbias")


@pytest.mark.parametrize("act", list(ACTS))
def test_gradients_against_differences(cuda_device, act):
    """fp64: the directional derivative of sum(C * W) by central differences. With step h the difference is off by h^2 / 6 times the third
    derivative (below 50 times the sum of magnitudes here) and by 2^-53 / h of it: 1e-9 for h = 1e-5 (ReLU: no z changes its sign within the
    step, which is checked)."""
    rng = np.random.default_rng(23)
    rows, cols, R, h = 15, 12, 6, 1e-5
    m, u = (Matrix(random_mask(rows, cols, 0.4, rng), torch.float64, rng) for _ in range(2))
    B, b, W = (torch.as_tensor(rng.standard_normal(s)).cuda() for s in ((cols, R), (rows,), (rows, R)))
    dB, db = (torch.as_tensor(rng.standard_normal(s)).cuda() for s in ((cols, R), (rows,)))
    dv, dv2 = (torch.as_tensor(rng.standard_normal(k.val.numel())).cuda() for k in (m, u))

    def single(t):
        A = m.t.with_values(m.val.cuda() + t * dv)
        z = torch.empty(rows, R, dtype=torch.float64, device="cuda")
        c = comet.spmm_epilogue(A, B + t * dB, act=ACTS[act], bias=b + t * db, preact=z)
        return float((c * W).sum()), z

    def gated(t):
        A, A2 = m.t.with_values(m.val.cuda() + t * dv), u.t.with_values(u.val.cuda() + t * dv2)
        z = (torch.empty(rows, R, dtype=torch.float64, device="cuda"), torch.empty(rows, R, dtype=torch.float64, device="cuda"))
        c = comet.spmm_gated(A, A2, B + t * dB, act=ACTS[act], bias_g=b + t * db, bias_u=b, preact=z)
        return float((c * W).sum()), z

    Mt, Ut = comet.transpose_symbolic(m.t), comet.transpose_symbolic(u.t)
    _, z = single(0.0)
    assert torch.equal(single(h)[1] > 0, single(-h)[1] > 0) and torch.equal(gated(h)[1][0] > 0, gated(-h)[1][0] > 0)
    gv, gB, gb = comet.spmm_epilogue_backward(m.t, Mt, B, W, act=ACTS[act], preact=z, bias_along=comet.BIAS_ROWS)
    terms = [(gv * dv), (gB * dB), (gb * db)]
    slope = (single(h)[0] - single(-h)[0]) / (2 * h)
    assert abs(sum(float(t.sum()) for t in terms) - slope) <= 2e-8 * sum(float(t.abs().sum()) for t in terms)
    _, z = gated(0.0)
    gg, gu, gB, gb, _ = comet.spmm_gated_backward(m.t, Mt, u.t, Ut, B, W, z, act=ACTS[act], need_bias=True)
    terms = [(gg * dv), (gu * dv2), (gB * dB), (gb * db)]
    slope = (gated(h)[0] - gated(-h)[0]) / (2 * h)
    assert abs(sum(float(t.sum()) for t in terms) - slope) <= 2e-8 * sum(float(t.abs().sum()) for t in terms)


# ---------------------------------------------------------------------------------------------- edges

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("R", [3, 64, 256])
def test_only_stored_cells_count(cuda_device, dtype, R):
    """Infinities and NaN in rows of B that a row does not store leave its result alone; those it stores reach it. The sums over the stored cells
    may be taken in another order where such values are about, so they are held to the definition, each within z_bound and one rounding."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(R)
    mask = random_mask(200, 160, 0.3, rng)
    mask[:, 5] = False
    mask[150:, 5] = True
    mask[:, 6] = False
    mask[10, 6] = True
    mask[:, 7] = False
    m = Matrix(mask, dt, rng)
    B, _ = values((160, R), dt, rng)
    clean = comet.spmm_epilogue(m.t, B.cuda(), act=ACTS["silu"])
    B[5], B[6, 0], B[7, R - 1] = float("nan"), float("inf"), -float("inf")
    got = comet.spmm_epilogue(m.t, B.cuda(), act=ACTS["none"])
    assert bool(torch.isnan(got[150:]).all())
    assert bool(torch.isinf(got[10, 0])) or bool(torch.isnan(got[10, 0]))
    B64 = torch.nan_to_num(B.double(), nan=0.0, posinf=0.0, neginf=0.0)
    z, N = (m.dense @ B64)[:150], (m.dense.abs() @ B64.abs())[:150]
    bound = stored(dt, z, z_bound(dt, m.longest, N, z))
    bound[10, 0] = float("inf")
    assert_within(torch.where(torch.isfinite(bound), got[:150].cpu().double(), z), z, bound, "rows without the infinities")
    assert bool(torch.isfinite(clean).all())


def test_no_entries_no_rows_no_columns(cuda_device):
    rng = np.random.default_rng(0)
    for rows, cols in [(6, 4), (6, 0), (0, 4)]:
        m = Matrix(np.zeros((rows, cols), dtype=bool), torch.float32, rng)
        b = torch.arange(rows, dtype=torch.float32, device="cuda")
        B = torch.randn(cols, 9, device="cuda")
        res = torch.randn(rows, 9, device="cuda")
        got = comet.spmm_epilogue(m.t, B, bias=b, residual=res)
        assert torch.equal(got, b[:, None] + res)
        assert comet.sddmm(m.t, torch.randn(rows, 9, device="cuda"), B).val.numel() == 0
        if cols:
            At = comet.transpose_symbolic(m.t)
            dval, dB, dbias = comet.spmm_epilogue_backward(m.t, At, B, res, bias_along=comet.BIAS_COLS)
            assert dval.numel() == 0 and bool((dB == 0).all()) and torch.allclose(dbias, res.sum(0), atol=1e-5)


def test_residual_in_place_and_repeatable(cuda_device):
    rng = np.random.default_rng(2)
    m = Matrix(random_mask(300, 900, 0.3, rng), torch.float32, rng, scale=0.1)
    B, r = torch.randn(900, 48, device="cuda"), torch.randn(300, 48, device="cuda")
    want = comet.spmm_epilogue(m.t, B, act=ACTS["gelu"], residual=r)
    out = r.clone()
    comet.spmm_epilogue(m.t, B, act=ACTS["gelu"], residual=out, out=out)
    assert torch.equal(out, want)
    z = torch.randn(300, 48, device="cuda")
    At = comet.transpose_symbolic(m.t)
    first = comet.spmm_epilogue_backward(m.t, At, B, r, act=ACTS["silu"], preact=z, bias_along=comet.BIAS_COLS)
    for a, b in zip(first, comet.spmm_epilogue_backward(m.t, At, B, r, act=ACTS["silu"], preact=z, bias_along=comet.BIAS_COLS)):
        assert torch.equal(a, b)


def test_values_may_change_after_the_transpose(cuda_device):
    rng = np.random.default_rng(4)
    m = Matrix(random_mask(50, 60, 0.3, rng), torch.float64, rng)
    At = comet.transpose_symbolic(m.t)
    val = m.val.cuda() * 3.0 + 1.0
    dC = torch.randn(50, 8, dtype=torch.float64, device="cuda")
    _, dB, _ = comet.spmm_epilogue_backward(m.t.with_values(val), At, None, dC, need_val=False)
    dense = torch.zeros(50, 60, dtype=torch.float64, device="cuda")
    dense[m.rc[0].cuda(), m.rc[1].cuda()] = val
    assert torch.allclose(dB, dense.t() @ dC, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("kind", ["huge row", "tiles", "short rows", "few columns"])
def test_streams_and_captured_graphs(cuda_device, kind):
    """Calls on side streams, and two captured graphs of one handle replayed side by side, in every form that a call may take."""
    rng = np.random.default_rng(6)
    rows, cols, density, R, dt = {"huge row": (400, 20_000, 0.02, 40, torch.float32), "tiles": (1024, 2048, 0.3, 128, torch.bfloat16),
                                  "short rows": (24_000, 1800, 0.0145, 40, torch.float32), "few columns": (3000, 900, 0.3, 1, torch.float16)}[kind]
    mask = random_mask(rows, cols, density, rng)
    if kind == "huge row":
        mask[3, :18_000] = True                            # a row that takes temporary memory
    m = Matrix(mask, dt, rng, scale=0.1)
    At = comet.transpose_symbolic(m.t)
    B = [torch.randn(cols, R, device="cuda").to(dt) for _ in range(2)]
    dC = [torch.randn(rows, R, device="cuda").to(dt) for _ in range(2)]
    z = [torch.randn(rows, R, device="cuda").to(dt) for _ in range(2)]

    def step(k):
        c = comet.spmm_epilogue(m.t, B[k], act=ACTS["gelu"])
        return [c] + [g for g in comet.spmm_epilogue_backward(m.t, At, B[k], dC[k], act=ACTS["gelu"], preact=z[k], bias_along=comet.BIAS_COLS)]

    want = [step(0), step(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k] = step(k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], [None, None]
    for k, g in enumerate(graphs):
        with torch.cuda.graph(g):
            outs[k] = step(k)
    for _ in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(outs, want) for a, b in zip(g, w))


def test_large_offsets(cuda_device):
    """Rows of B and C whose byte offsets pass 32 bits."""
    rows, ld = 70_000, 40_000                              # 70,000 x 40,000 fp16: 5.6 GB
    big = torch.empty(rows * ld, dtype=torch.float16, device="cuda").view(rows, ld)
    R = 16
    B = big[:, :R]
    B.copy_(torch.randn(rows, R, device="cuda"))
    rng = np.random.default_rng(1)
    r = np.repeat(np.arange(0, rows, 7), 3)
    c = np.sort(rng.integers(0, rows, (len(r) // 3, 3)) // 3 * 3 + np.arange(3), axis=1).clip(0, rows - 1)
    c[:, 1:] = np.maximum(c[:, 1:], c[:, :-1] + 1)
    c = np.minimum(c, rows - 3 + np.arange(3)).reshape(-1)
    pos = np.concatenate([[0], np.cumsum(np.bincount(r, minlength=rows))])
    i32 = lambda a: torch.as_tensor(a).to(torch.int32).cuda()  # noqa: E731
    val = torch.randn(len(r), device="cuda").half()
    A = comet.SpTensor.from_arrays((rows, rows), (0, 1), (comet.D, comet.CU), [i32([rows]), i32(pos)], [None, i32(c)], val)
    C_ = big[:, 128:128 + R]
    comet.spmm_epilogue(A, B, out=C_)
    rt, ct = torch.as_tensor(r).cuda(), torch.as_tensor(c).long().cuda()
    terms = B.double()[ct] * val.double()[:, None]
    want = torch.zeros(rows, R, dtype=torch.float64, device="cuda").index_add_(0, rt, terms)
    N = torch.zeros(rows, R, dtype=torch.float64, device="cuda").index_add_(0, rt, terms.abs())
    assert bool(((C_.double() - want).abs() <= 2.0 ** -11 * want.abs() + 12 * 2.0 ** -24 * N + 2.0 ** -24).all())
    got = comet.sddmm(A, C_, B).val.double()
    want = (C_.double()[rt] * B.double()[ct]).sum(1)
    N = (C_.double()[rt] * B.double()[ct]).abs().sum(1)
    assert bool(((got - want).abs() <= 2.0 ** -11 * want.abs() + 24 * 2.0 ** -24 * N + 2.0 ** -24).all())


# ---------------------------------------------------------------------------------------------- together, and refusals

def test_pruned_feed_forward_block(cuda_device):
    """The operators as one block uses them: H = silu(G X) * (U X + b), Y = D H + X, and all gradients of sum(Y * W), against autograd on the
    dense block in 64 bits. fp64: every gradient within 1e-12 of the sum of its terms' magnitudes, taken as its largest value times the widths."""
    rng = np.random.default_rng(8)
    hid, ff, T = 96, 256, 40
    g, u = (Matrix(random_mask(ff, hid, 0.2, rng), torch.float64, rng, scale=0.2) for _ in range(2))
    d = Matrix(random_mask(hid, ff, 0.2, rng, empty=(7,)), torch.float64, rng, scale=0.1)
    X, W = (torch.as_tensor(rng.standard_normal((hid, T))).cuda() for _ in range(2))
    b = torch.as_tensor(rng.standard_normal(ff)).cuda()
    z = tuple(torch.empty(ff, T, dtype=torch.float64, device="cuda") for _ in range(2))
    H = comet.spmm_gated(g.t, u.t, X, act=comet.ACT_SILU, bias_u=b, preact=z)
    Y = comet.spmm_epilogue(d.t, H, residual=X)
    dD, dH, _ = comet.spmm_epilogue_backward(d.t, comet.transpose_symbolic(d.t), H, W)
    dG, dU, dX, _, db = comet.spmm_gated_backward(g.t, comet.transpose_symbolic(g.t), u.t, comet.transpose_symbolic(u.t), X, dH, z, act=comet.ACT_SILU,
                                                  need_bias=True)
    dX = dX + W
    leaves = [t.dense.cuda().requires_grad_() for t in (g, u, d)] + [X.clone().requires_grad_(), b.clone().requires_grad_()]
    G, U, Dn, x, bb = leaves
    y = Dn @ (torch.nn.functional.silu(G @ x) * (U @ x + bb[:, None])) + x
    assert torch.allclose(Y, y, rtol=1e-12, atol=1e-12)
    grads = torch.autograd.grad((y * W).sum(), leaves)
    for got, want, m in [(dG, grads[0], g), (dU, grads[1], u), (dD, grads[2], d)]:
        want = want[m.rc[0].cuda(), m.rc[1].cuda()]
        assert float((got - want).abs().max()) <= 1e-12 * float(want.abs().max()) * T
    assert float((dX - grads[3]).abs().max()) <= 1e-12 * float(grads[3].abs().max()) * ff
    assert float((db - grads[4]).abs().max()) <= 1e-12 * float(grads[4].abs().max()) * T


def test_refusals(cuda_device):
    rng = np.random.default_rng(9)
    m = Matrix(random_mask(10, 8, 0.5, rng), torch.float32, rng)
    B = torch.randn(8, 6, device="cuda")
    At = comet.transpose_symbolic(m.t)
    dC = torch.randn(10, 6, device="cuda")
    with pytest.raises(TypeError):
        comet.spmm_epilogue(m.t, B.double())
    with pytest.raises(TypeError):
        comet.spmm_epilogue(m.t, B, bias=torch.zeros(10, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, B.cpu())
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, torch.randn(9, 6, device="cuda"))
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, torch.randn(6, 8, device="cuda").t())
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, torch.randn(8, 1, device="cuda").expand(8, 6))
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, B, bias=torch.zeros(6, device="cuda"))
    with pytest.raises(ValueError):
        comet.spmm_epilogue(m.t, B, residual=torch.zeros(10, 5, device="cuda"))
    with pytest.raises(comet.CometError) as e:
        comet.spmm_epilogue(m.t, B, act=9)
    assert e.value.status == -1
    with pytest.raises(ValueError):
        comet.spmm_epilogue_backward(m.t, None, B, dC)
    with pytest.raises(ValueError):
        comet.spmm_epilogue_backward(m.t, At, None, dC)
    with pytest.raises(ValueError):
        comet.spmm_epilogue_backward(m.t, At, B, dC, act=comet.ACT_GELU)
    with pytest.raises(comet.CometError):                  # not the transpose of this matrix
        comet.spmm_epilogue_backward(m.t, m.t, B, dC)
    other = Matrix(random_mask(10, 8, 0.9, rng), torch.float32, rng)
    if other.t.nnz != m.t.nnz:
        with pytest.raises(comet.CometError):
            comet.spmm_epilogue_backward(m.t, comet.transpose_symbolic(other.t), B, dC)
    with pytest.raises(TypeError):
        comet.spmm_epilogue(At, dC)
    with pytest.raises(comet.CometError):                  # the structure of a transpose is no matrix of values
        comet.spmm(At, dC.to(torch.int32))
    with pytest.raises(ValueError):
        comet.spmm_gated(m.t, Matrix(random_mask(9, 8, 0.5, rng), torch.float32, rng).t, B)
    with pytest.raises(ValueError):
        comet.spmm_gated(m.t, Matrix(random_mask(10, 8, 0.5, rng), torch.float64, rng).t, B)
    with pytest.raises(ValueError):
        comet.sddmm(m.t, dC, B, out_val=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        m.t.with_values(torch.zeros(m.t.nnz + 1, device="cuda"))
    half = Matrix(random_mask(10, 8, 0.5, rng), torch.bfloat16, rng)
    with pytest.raises(comet.CometError) as e:             # 16-bit values are for the layer operators alone
        comet.spmm(half.t, B.bfloat16())
    assert e.value.status == -2
    with pytest.raises(comet.CometError):
        comet.spmv(half.t, B[:, 0].contiguous().bfloat16())
    X = comet.pack([torch.zeros(1, dtype=torch.int32, device="cuda")] * 3, torch.ones(1, device="cuda"), (2, 2, 2), (0, 1, 2), (comet.CU,) * 3)
    with pytest.raises(ValueError):
        comet.spmm_epilogue(X, B)


def test_refusals_of_the_library(cuda_device):
    """The same straight through the C ABI: misaligned pointers, leading dimensions, NULL pointers, formats."""
    from paper_2102_05187_b200.binding import EpilogueStruct, SpTensorStruct
    rng = np.random.default_rng(10)
    m = Matrix(random_mask(10, 8, 0.5, rng), torch.float32, rng)
    lib, h = comet.load_library(), comet.default_handle()
    buf = torch.zeros(4096, device="cuda")
    p = buf.data_ptr()
    e = EpilogueStruct(0, 0, 0, 0, 0, 0, 0)
    call = lambda A=m.t._ref, B=p, R=4, ldb=4, ep=e, Cp=p + 8192, ldc=4: lib.comet_spmm_epilogue(h._h, A, B, R, ldb, None if ep is None else C.byref(ep), Cp, ldc, 0)  # noqa: E731
    assert call() == 0
    assert call(B=0) == -1 and call(Cp=0) == -1 and call(ep=None) == -1 and call(R=0) == -1 and call(ldb=3) == -1 and call(ldc=3) == -1
    assert call(A=None) == -1
    assert call(B=p + 2) == -9 and call(Cp=p + 8193) == -9
    assert call(ldb=1 << 28) == -5
    assert call(ep=EpilogueStruct(0, 2, 0, 0, 0, 0, 0)) == -1 and call(ep=EpilogueStruct(-1, 0, 0, 0, 0, 0, 0)) == -1
    assert call(ep=EpilogueStruct(0, 0, p + 1, 0, 0, 0, 0)) == -9 and call(ep=EpilogueStruct(0, 0, 0, p, 3, 0, 0)) == -1
    assert call(ep=EpilogueStruct(0, 0, 0, 0, 0, p, 3)) == -1
    bad = SpTensorStruct.from_buffer_copy(m.t.c)
    bad.attr[1] = comet.D
    assert call(A=C.byref(bad)) == -2
    bad = SpTensorStruct.from_buffer_copy(m.t.c)
    bad.dtype = 4
    assert call(A=C.byref(bad)) == -2
    assert lib.comet_sddmm(h._h, m.t._ref, p, 4, p, 4, 4, 0, 0) == -1 and lib.comet_sddmm(h._h, m.t._ref, p, 3, p, 4, 4, p, 0) == -1
    out = SpTensorStruct()
    assert lib.comet_transpose_symbolic(h._h, None, 0, C.byref(out)) == -1 and lib.comet_transpose_symbolic(h._h, m.t._ref, 0, None) == -1
    assert lib.comet_spmm_gated(h._h, m.t._ref, m.t._ref, p, 4, 4, 0, 0, 0, p, 0, 4, p + 8192, 4, 0) == -1
    assert lib.comet_spmm_epilogue_backward(h._h, m.t._ref, None, p, 4, 4, 0, 0, 0, p, 4, 0, 0, 0, p + 8192, 4, 0) == -1
    torch.cuda.synchronize()
