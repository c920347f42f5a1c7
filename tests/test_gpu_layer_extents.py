"""Layer operators at the far end of their extents: more columns of B than one launch has tiles, more columns of A than the lists of tiles can count."""
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import CU, D  # noqa: E402


def csr(rows, cols, pos, crd, val):
    i32 = lambda t: t.to(torch.int32)  # noqa: E731
    return comet.SpTensor.from_arrays((rows, cols), (0, 1), (D, CU), [torch.full((1,), rows, dtype=torch.int32, device="cuda"), i32(pos)], [None, i32(crd)], val)


def within(got, want, N, n):
    """fp32 sums of n terms, rounded to bf16 once."""
    bound = (n + 8) * 2.0 ** -24 * N
    bad = (got.double() - want).abs() > bound + 2.0 ** -8 * (want.abs() + bound) + 2.0 ** -133
    assert not bool(bad.any()), int(bad.sum())


@pytest.mark.parametrize("R", [65_535 * 64, 65_535 * 64 + 8, 65_535 * 256 + 200, (1 << 24) - 8])
def test_columns_of_b(cuda_device, R):
    """A matrix of 64 x 64, half full: 32 strips of B of up to 2.1 GB. The columns at both ends and on both sides of whole numbers of tiles are compared."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    dense = torch.randn(64, 64, generator=gen, device="cuda").bfloat16()
    dense[torch.rand(64, 64, generator=gen, device="cuda") < 0.5] = 0
    at = dense.nonzero()
    pos = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.bincount(at[:, 0], minlength=64).cumsum(0)])
    A = csr(64, 64, pos, at[:, 1], dense[at[:, 0], at[:, 1]])
    B = torch.randn(64, R, generator=gen, device="cuda", dtype=torch.bfloat16)
    edges = [0, 65_535 * 64, 65_535 * 128, 65_535 * 256, R]
    cols = torch.cat([torch.arange(max(0, e - 300), min(R, e + 300), device="cuda") for e in edges if e <= R]).unique()
    want, N = dense.double() @ B[:, cols].double(), dense.double().abs() @ B[:, cols].double().abs()
    out = comet.spmm_epilogue(A, B, act=comet.ACT_NONE)
    within(out[:, cols], want, N, 64)
    out = comet.spmm_epilogue(A, B, act=comet.ACT_RELU, out=out)
    within(out[:, cols], want.relu(), N, 64)
    del out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [134_215_616, 134_215_617, 134_300_000])
def test_columns_of_a(cuda_device, monkeypatch, cols):
    """Two rows with an entry in every 50th column, 8 columns of B (2.1 GB)."""
    monkeypatch.setenv("COMET_LAYER_TILE_WORK", "0")       # tiles as long as the lists can count them
    n, R = cols // 50, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    crd = torch.cat([torch.arange(n, device="cuda") * 50 + (cols - 1 - 50 * (n - 1)), torch.arange(n, device="cuda") * 50])
    val = (torch.randn(2 * n, generator=gen, device="cuda") / n ** 0.5).bfloat16()
    A = csr(2, cols, torch.tensor([0, n, 2 * n], device="cuda"), crd, val)
    B = torch.randn(cols, R, generator=gen, device="cuda", dtype=torch.bfloat16)
    got = comet.spmm_epilogue(A, B)
    terms = val.double()[:, None] * B[crd].double()
    want, N = terms.view(2, n, R).sum(1), terms.abs().view(2, n, R).sum(1)
    within(got, want, N, n)
    torch.cuda.empty_cache()
