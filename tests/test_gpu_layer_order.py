"""[CN,S] matrices as comet_validate accepts them: rows in order, a row's columns in any order, cells stored more than once. The layer operators add such
entries up in every form that they take, at sizes where compressed matrices take the forms that rely on ascending columns."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import CN, TYPES, S, act64, act_bound, assert_within, stored, u_of, values, z_bound  # noqa: E402

KINDS = {  # rows, cols, entries, type, columns of B; the form that a [D,CU] matrix of these sizes takes
    "tiles": (700, 1000, 160_000, "bf16", 264),
    "tiles, split": (130, 4200, 200_000, "f16", 250),
    "panels": (400, 25_600, 5_200_000, "f64", 2),
    "panels, 16 bits": (900, 25_600, 11_000_000, "bf16", 8),
    "one panel": (900, 5000, 700_000, "f32", 3),
    "rows": (300, 700, 40_000, "f32", 50),
    "short rows": (24_000, 1800, 600_000, "f32", 64),
}


def unordered(rows, cols, n, dt, rng, repeats):
    """Sorted rows, columns as they come; about one cell in fifty stored twice and one three times, or none."""
    r, c = rng.integers(0, rows, n), rng.integers(0, cols, n)
    if repeats:
        again = rng.integers(0, n, n // 50)
        r, c = np.concatenate([r, r[again], r[:1]]), np.concatenate([c, c[again], c[:1]])
    else:
        cell = rng.permutation(np.unique(r * cols + c))
        r, c = cell // cols, cell % cols
    order = np.argsort(r, kind="stable")
    r, c = r[order], c[order]
    v, v64 = values(r.size, dt, rng, (n / rows) ** -0.5)
    i32 = lambda a: torch.as_tensor(a).to(torch.int32).cuda()  # noqa: E731
    t = comet.SpTensor.from_arrays((rows, cols), (0, 1), (CN, S), [i32(np.array([0, r.size])), None], [i32(r), i32(c)], v.cuda())
    comet.validate(t)
    return t, torch.as_tensor(r), torch.as_tensor(c), v64


def dense_of(rows, cols, r, c, v):
    return torch.zeros(rows, cols, dtype=torch.float64).index_put_((r, c), v, accumulate=True)


@pytest.mark.parametrize("kind", list(KINDS))
def test_entries_in_any_order(cuda_device, kind, monkeypatch):
    rows, cols, n, dtype, R = KINDS[kind]
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows + R)
    if kind == "short rows":                               # long rows by blocks of B's rows, at these sizes too
        for name, value in [("LONG_MIN_NNZ", 1), ("LONG_MIN_B_MB", 0), ("LONG_ROW", 16), ("LONG_TILE", 32), ("PIECE", 8), ("BLOCKS", 4)]:
            monkeypatch.setenv("COMET_SPMM_" + name, str(value))
    B, B64 = values((cols, R), dt, rng)
    g, gr, gc, gv = unordered(rows, cols, n, dt, rng, True)
    u, ur, uc, uv = unordered(rows, cols, n // 2, dt, rng, True)
    z, dz = [], []
    for r, c, v in ((gr, gc, gv), (ur, uc, uv)):
        z.append(dense_of(rows, cols, r, c, v) @ B64)
        N = dense_of(rows, cols, r, c, v.abs()) @ B64.abs()
        dz.append(z_bound(dt, int(torch.bincount(r).max()), N, z[-1]))
    assert_within(comet.spmm_epilogue(g, B.cuda()), z[0], stored(dt, z[0], dz[0]), "product")
    f, df = act64("silu", z[0]), act_bound(dt, dz[0], z[0])
    want = f * z[1]
    assert_within(comet.spmm_gated(g, u, B.cuda()), want, stored(dt, want, df * z[1].abs() + (f.abs() + df) * dz[1] + 2 * u_of(dt) * want.abs()), "pair")
    P, P64 = values((rows, R), dt, rng)
    got = comet.sddmm(g, P.cuda(), B.cuda()).val
    want, N = (P64[gr] * B64[gc]).sum(1), (P64[gr].abs() * B64[gc].abs()).sum(1)
    assert_within(got, want, stored(dt, want, (R + 8) * u_of(dt) * N), "sampled")


@pytest.mark.parametrize("kind", ["tiles", "panels", "short rows"])
def test_gradients_of_entries_in_any_order(cuda_device, kind):
    rows, cols, n, dtype, R = KINDS[kind]
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows)
    t, r, c, v = unordered(rows, cols, n, dt, rng, False)
    dC, dC64 = values((rows, R), dt, rng)
    dB = comet.spmm_epilogue_backward(t, comet.transpose_symbolic(t), None, dC.cuda(), need_val=False)[1]
    dense = dense_of(rows, cols, r, c, v)
    want, N = dense.t() @ dC64, dense.abs().t() @ dC64.abs()
    assert_within(dB, want, stored(dt, want, z_bound(dt, int(torch.bincount(c).max()), N, want)), "dB")


def test_a_cell_stored_twice_has_no_transpose(cuda_device):
    t = unordered(50, 60, 400, torch.float32, np.random.default_rng(1), True)[0]
    with pytest.raises(comet.CometError) as e:
        comet.transpose_symbolic(t)
    assert e.value.status == -4
