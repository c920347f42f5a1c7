"""Few-column calls of the layer operators whose dense operand takes several panels of shared memory: around the widths at which a panel is full, parts
of rows that end inside a panel and go on in the next one, the gated pair and the sum of two products over both."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import TYPES, Matrix, assert_within, stored, u_of, values, z_bound  # noqa: E402
from test_gpu_layers import check_epilogue, check_gated  # noqa: E402

# Panels hold 200 KB less a row: 12,784 rows of 16 bytes, 25,584 of 8, 51,184 of 4 and 102,384 of 2, in steps of 16. Enough entries for the form:
# nnz (4 + size) >= 148 cols R size.
WIDTHS = [  # type, columns of B, columns of A, rows, density
    ("bf16", 8, 25_570, 900, 0.5), ("f16", 5, 25_598, 700, 0.5), ("f64", 2, 25_580, 500, 0.5), ("f32", 4, 25_598, 900, 0.4), ("f32", 3, 38_353, 700, 0.4),
    ("bf16", 4, 51_180, 450, 0.5), ("f32", 2, 51_190, 450, 0.4), ("f64", 1, 51_169, 260, 0.5), ("bf16", 2, 102_380, 225, 0.5), ("f32", 1, 102_398, 225, 0.4),
    ("f16", 1, 204_780, 115, 0.5), ("f64", 2, 12_784, 450, 0.5), ("f64", 2, 12_785, 450, 0.5), ("f64", 2, 12_799, 450, 0.5), ("f64", 2, 12_801, 450, 0.5),
]


def mask_of(rows, cols, density, rng):
    """Cells kept at random, thinner towards the right, so that parts of rows end on both sides of a panel's edge; a row without entries, one in the last
    columns alone, one in the first alone and one full."""
    m = rng.random((rows, cols), dtype=np.float32) < np.linspace(1.3 * density, 0.7 * density, cols, dtype=np.float32)
    m[1] = False
    m[2, :-7] = False
    m[3, 5:] = False
    m[4] = True
    return m


@pytest.mark.parametrize("dtype,R,cols,rows,density", WIDTHS)
def test_full_panels(cuda_device, dtype, R, cols, rows, density):
    dt = TYPES[dtype]
    es = torch.finfo(dt).bits // 8
    rng = np.random.default_rng(cols + R)
    m = Matrix(mask_of(rows, cols, density, rng), dt, rng, scale=(cols * density) ** -0.5)
    assert m.t.nnz * (4 + es) >= 148 * cols * R * es, "the sizes are of another form"
    check_epilogue(m, dt, R, "silu", "rows", True, True, rng, pad=R % 3)
    check_epilogue(m, dt, R, "none", "none", False, False, rng)
    u = Matrix(mask_of(rows, cols, 0.3, rng), dt, rng, scale=(cols * density) ** -0.5)
    check_gated(m, u, dt, R, "gelu_tanh", True, rng)


@pytest.mark.parametrize("dtype,R,cols,rows,density", [w for w in WIDTHS if w[2] in (25_570, 25_580, 25_598, 51_169, 12_785)])
def test_full_panels_of_the_transpose(cuda_device, dtype, R, cols, rows, density):
    """dB of the gated pair: both sources' dense operands pass through shared memory one after the other, in several panels each."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(cols)
    m, u = (Matrix(mask_of(rows, cols, d, rng).T.copy(), dt, rng, scale=(cols * density) ** -0.5) for d in (density, 0.4))
    (dC, dC64), (zg, zg64), (zu, zu64) = (values((cols, R), dt, rng) for _ in range(3))
    dB = comet.spmm_gated_backward(m.t, comet.transpose_symbolic(m.t), u.t, comet.transpose_symbolic(u.t), None, dC.cuda(), (zg.cuda(), zu.cuda()),
                                   act=comet.ACT_NONE, need_val=False)[2]
    dg, du = dC64 * zu64, dC64 * zg64
    want = m.dense.t() @ dg + u.dense.t() @ du
    N = m.dense.abs().t() @ dg.abs() + u.dense.abs().t() @ du.abs()
    e = N * (u_of(dt) * 4 + (torch.finfo(dt).eps / 2 if dt in (torch.bfloat16, torch.float16) else 0))
    tiny = 2.0 ** -25 * (m.dense.abs().sum(0) + u.dense.abs().sum(0))[:, None] if dt == torch.float16 else 0.0      # dZ below fp16's normal range
    assert_within(dB, want, stored(dt, want, 1.01 * e + tiny + z_bound(dt, m.tallest + u.tallest, N * 1.01, want)), "dB")


@pytest.mark.parametrize("dtype,R,cols,rows,density", [("bf16", 8, 2000, 400, 0.5), ("f32", 1, 3000, 700, 0.4), ("f64", 2, 25_580, 500, 0.5), ("bf16", 8, 25_570, 900, 0.5)])
def test_only_stored_cells_count_in_panels(cuda_device, dtype, R, cols, rows, density):
    """Infinities and NaN in rows of B that a row of A does not store leave its result alone, in the panel that holds them and in the others."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(cols)
    mask = mask_of(rows, cols, density, rng)
    bad = [0, 9, cols // 2 - 1, cols // 2, cols - 9, cols - 1]
    mask[:, bad] = False
    mask[rows - 50:, bad[2]] = True
    m = Matrix(mask, dt, rng, scale=(cols * density) ** -0.5)
    B, _ = values((cols, R), dt, rng)
    for k, j in enumerate(bad):
        B[j] = [float("nan"), float("inf"), float("nan"), -float("inf"), float("inf"), float("nan")][k]
    B64 = torch.nan_to_num(B.double(), nan=0.0, posinf=0.0, neginf=0.0)
    got = comet.spmm_epilogue(m.t, B.cuda()).cpu()
    assert bool(torch.isnan(got[rows - 50:]).all())
    z = m.dense @ B64
    bound = stored(dt, z, z_bound(dt, m.longest, m.dense.abs() @ B64.abs(), z))
    assert_within(got[:rows - 50], z[:rows - 50], bound[:rows - 50], "rows without them")
