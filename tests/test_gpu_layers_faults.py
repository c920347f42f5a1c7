"""An allocator that refuses its n-th request turns the layer operators into a clean COMET_ERR_ALLOC, in each form that they take: nothing stays
allocated, and the handle goes on working."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import Matrix, random_mask  # noqa: E402
from test_gpu_faults import FailingHandle  # noqa: E402

KINDS = {  # rows, cols, density, columns, type, format
    "tiles": (512, 1024, 0.8, 133, torch.bfloat16, "csr"),
    "short rows": (24_000, 1800, 0.0145, 21, torch.float32, "csr"),
    "short rows, 16 bits": (24_000, 1800, 0.0145, 20, torch.float16, "csr"),
    "huge row": (40, 40_000, 0.01, 9, torch.float32, "csr"),
    "compressed": (300, 400, 0.1, 5, torch.float64, "dcsr"),
}


@pytest.mark.parametrize("kind", list(KINDS))
def test_every_allocation_failure(cuda_device, kind):
    rows, cols, density, R, dt, fmt = KINDS[kind]
    rng = np.random.default_rng(3)
    h = FailingHandle()
    mask = random_mask(rows, cols, density, rng)
    if kind == "huge row":
        mask[3, :30_000] = True
    m, u = Matrix(mask, dt, rng, fmt, scale=0.1), Matrix(random_mask(rows, cols, density, rng), dt, rng, fmt, scale=0.1)
    for k in (m, u):
        k.t.handle = h
    B, dC, z = (torch.randn(n, R, device="cuda").to(dt) for n in (cols, rows, rows))
    h.arm(None)
    At, Ut = comet.transpose_symbolic(m.t), comet.transpose_symbolic(u.t)
    steps = [
        lambda: [comet.spmm_epilogue(m.t, B, act=comet.ACT_GELU, residual=dC)],
        lambda: [comet.spmm_gated(m.t, u.t, B)],
        lambda: list(comet.spmm_epilogue_backward(m.t, At, B, dC, act=comet.ACT_SILU, preact=z, bias_along=comet.BIAS_COLS)),
        lambda: list(comet.spmm_gated_backward(m.t, At, u.t, Ut, B, dC, (z, z), need_bias=True)),
        lambda: [comet.sddmm(m.t, dC, B).val],
        lambda: [comet.transpose_symbolic(m.t).val],
    ]
    for n, step in enumerate(steps):
        h.arm(None)
        want = step()
        total = h.calls
        torch.cuda.synchronize()
        for k in range(total):
            live = len(h._live)
            h.arm(k)
            try:
                got = step()
            except comet.CometError as e:
                assert e.status == -6, (n, k, e)
            else:                                          # a product has a form that needs no copy of its operand
                assert all(torch.allclose(a.float(), b.float(), rtol=2e-2, atol=2e-2) for a, b in zip(got, want)), (n, k)
                del got
            torch.cuda.synchronize()
            assert len(h._live) == live, f"step {n}, allocation {k}: blocks leaked"
        h.arm(None)
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
