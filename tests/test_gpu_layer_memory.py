"""Products of the layer operators that get no temporary memory at all, or not the n-th block of it: they fall back to kernels that need none, and are held to
their definitions as ever."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import TYPES, Matrix, random_mask, values  # noqa: E402
from test_gpu_faults import FailingHandle  # noqa: E402
from test_gpu_layers import check_epilogue, check_gated, check_sddmm  # noqa: E402


class Every:
    """Equal to every request's number."""

    def __eq__(self, other):
        return True


KINDS = {  # rows, cols, density, columns, type
    "tiles": (512, 1024, 0.8, 136, "bf16"),
    "tiles, unaligned": (512, 1024, 0.8, 133, "f16"),
    "short rows": (24_000, 1800, 0.0145, 21, "f32"),
    "short rows, 16 bits": (24_000, 1800, 0.0145, 20, "bf16"),
    "short rows, fp64": (24_000, 1800, 0.0145, 6, "f64"),
    "huge row": (40, 40_000, 0.01, 9, "f32"),
    "few columns": (3000, 900, 0.3, 2, "f32"),
}


@pytest.mark.parametrize("kind", list(KINDS))
def test_products_without_memory(cuda_device, kind):
    rows, cols, density, R, dtype = KINDS[kind]
    dt = TYPES[dtype]
    rng = np.random.default_rng(7)
    h = FailingHandle()
    mask = random_mask(rows, cols, density, rng)
    if kind == "huge row":
        mask[3, :30_000] = True
    m, u = (Matrix(k, dt, rng, scale=(cols * density) ** -0.5) for k in (mask, random_mask(rows, cols, density, rng)))
    m.t.handle = u.t.handle = h
    P, P64 = values((rows, R), dt, rng)
    Q, Q64 = values((cols, R), dt, rng)
    steps = [lambda: check_epilogue(m, dt, R, "gelu", "rows", True, True, rng), lambda: check_epilogue(m, dt, R, "none", "none", False, False, rng),
             lambda: check_epilogue(m, dt, R, "silu", "cols", True, False, rng), lambda: check_gated(m, u, dt, R, "silu", True, rng),
             lambda: check_sddmm(m, P, P64, Q, Q64, dt)]
    for step in steps:
        h.arm(None)
        step()
        total, live = h.calls, len(h._live)
        for fail_at in [Every(), *range(total)]:
            h.arm(fail_at)
            step()
            torch.cuda.synchronize()
            assert len(h._live) == live, "blocks leaked"
    h.arm(None)


@pytest.mark.parametrize("kind,turned,fits", [("tiles", False, True), ("short rows, 16 bits", True, True), ("short rows, 16 bits", False, False)])
def test_the_transposed_product_without_memory_for_its_form(cuda_device, kind, turned, fits):
    """dB by lists of tiles or by fp32 copies: with the first block refused, a block for the values in the transpose's order does. The transpose of a matrix of short
    rows has long ones, which want that block from the start."""
    rows, cols, density, R, dtype = KINDS[kind]
    if turned:
        rows, cols = cols, rows
    dt = TYPES[dtype]
    rng = np.random.default_rng(8)
    h = FailingHandle()
    m = Matrix(random_mask(rows, cols, density, rng), dt, rng, scale=0.05)
    m.t.handle = h
    dC, dC64 = values((rows, R), dt, rng)
    dC = dC.cuda()
    At = comet.transpose_symbolic(m.t)
    want, N = m.dense.t() @ dC64, m.dense.abs().t() @ dC64.abs()
    h.arm(0)
    if not fits:
        with pytest.raises(comet.CometError) as e:
            comet.spmm_epilogue_backward(m.t, At, None, dC, need_val=False)
        assert e.value.status == -6
        h.arm(None)
        return
    dB = comet.spmm_epilogue_backward(m.t, At, None, dC, need_val=False)[1].cpu().double()
    h.arm(None)
    bound = (m.tallest + 8) * 2.0 ** -24 * N
    assert bool(((dB - want).abs() <= bound + torch.finfo(dt).eps / 2 * (want.abs() + bound) + 2.0 ** -25).all())


@pytest.mark.parametrize("dtype,rows,cols,density,R", [("f32", 512, 1000, 0.4, 50), ("f32", 300, 1500, 0.3, 129), ("f16", 512, 1000, 0.4, 17)])
def test_workers_per_row_take_operands_as_they_are(cuda_device, dtype, rows, cols, density, R):
    """One launch, no copy of rows that do not start on 16 bytes, no temporary memory."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(9)
    h = FailingHandle()
    m, u = (Matrix(random_mask(rows, cols, density, rng), dt, rng, scale=0.05) for _ in range(2))
    m.t.handle = u.t.handle = h
    h.arm(None)
    for check in (lambda: check_epilogue(m, dt, R, "gelu", "rows", True, True, rng), lambda: check_gated(m, u, dt, R, "silu", True, rng)):
        before = h.kernel_launches()
        check()
        assert h.kernel_launches() - before == 1
    assert h.calls == 0
