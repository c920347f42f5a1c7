"""Waits of the tensor-core kernels that run out: the kernel returns, the next call of a layer operator on the handle reports it once, whatever form that
call takes, and the ones after it give the results of before. COMET_LAYER_WAIT_CYCLES shortens the waits: with 0 none is granted, with a few hundred or thousand cycles
some run out while copies and products are in flight, or none does and the result is whole."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import Matrix, random_mask  # noqa: E402

KINDS = {  # rows, cols, density, columns of B: one CTA per tile, unaligned rows, the blocks of k split over a cluster, many tiles
    "tile": (200, 1000, 0.3, 64), "unaligned": (200, 1000, 0.3, 61), "split": (130, 8300, 0.1, 256), "split, unaligned": (130, 4200, 0.3, 121), "many": (4096, 2048, 0.2, 520),
}


@pytest.fixture
def any_work(monkeypatch):
    monkeypatch.setenv("COMET_LAYER_TILE_WORK", "0")


def calls_of(rows, cols, density, R, dt):
    rng = np.random.default_rng(rows)
    m, u = (Matrix(random_mask(rows, cols, density, rng), dt, rng, scale=0.1) for _ in range(2))
    B, dC = (torch.randn(n, R, device="cuda").to(dt) for n in (cols, rows))
    At = comet.transpose_symbolic(m.t)
    return [lambda: comet.spmm_epilogue(m.t, B, act=comet.ACT_GELU, residual=dC), lambda: comet.spmm_gated(m.t, u.t, B), lambda: comet.sddmm(m.t, dC, B).val,
            lambda: comet.spmm_epilogue_backward(m.t, At, None, dC, need_val=False)[1]]


def reported(e):
    assert e.value.status == -7
    assert comet.load_library().comet_last_cuda_error(comet.default_handle()._h) == 702          # a launch that took too long


@pytest.mark.parametrize("kind", list(KINDS))
def test_no_wait_is_granted(cuda_device, any_work, monkeypatch, kind):
    calls = calls_of(*KINDS[kind], torch.bfloat16)
    rng = np.random.default_rng(0)
    other = Matrix(random_mask(20, 30, 0.3, rng), torch.float32, rng)
    x = torch.randn(30, 4, device="cuda")
    others = [lambda: comet.spmm_epilogue(other.t, x), lambda: comet.transpose_symbolic(other.t), lambda: comet.sddmm(other.t, torch.randn(20, 4, device="cuda"), x),
              lambda: comet.spmm_gated(other.t, other.t, x)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    for n, call in enumerate(calls):
        with monkeypatch.context() as m:
            m.setenv("COMET_LAYER_WAIT_CYCLES", "0")
            call()                                         # returns COMET_OK: the kernel has not run yet
        torch.cuda.synchronize()
        before = comet.default_handle().kernel_launches()
        with pytest.raises(comet.CometError) as e:
            others[n]()                                    # other forms, other operators
        reported(e)
        assert comet.default_handle().kernel_launches() == before
        others[n]()
        assert all(torch.equal(c(), w) for c, w in zip(calls, want))
        torch.cuda.synchronize()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("cycles", [1, 100, 400, 1000, 2500, 6000, 15_000, 40_000])
def test_waits_run_out_on_the_way(cuda_device, any_work, monkeypatch, kind, cycles):
    calls = calls_of(*KINDS[kind], torch.float16)
    want = [c() for c in calls]
    torch.cuda.synchronize()
    for call, w in zip(calls, want):
        for _ in range(3):
            with monkeypatch.context() as m:
                m.setenv("COMET_LAYER_WAIT_CYCLES", str(cycles))
                got = call()
            torch.cuda.synchronize()
            try:
                again = call()
            except comet.CometError as e:
                assert e.status == -7
                again = call()
            else:
                assert torch.equal(got, w), "nothing was reported"
            assert torch.equal(again, w)


def test_a_replayed_graph_reports_to_the_next_call(cuda_device, any_work, monkeypatch):
    call = calls_of(*KINDS["tile"], torch.bfloat16)[0]
    want = call()
    graph = torch.cuda.CUDAGraph()
    with monkeypatch.context() as m:
        m.setenv("COMET_LAYER_WAIT_CYCLES", "0")
        with torch.cuda.graph(graph):
            call()
    assert torch.equal(call(), want)                       # nothing has run out yet
    graph.replay()
    torch.cuda.synchronize()
    with pytest.raises(comet.CometError) as e:
        call()
    reported(e)
    assert torch.equal(call(), want)
