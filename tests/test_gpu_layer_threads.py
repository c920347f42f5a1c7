"""Calls from host threads of their own: native ones (a small C program of the test), which have made no CUDA call before and are inside the library at the
same time, as Python's hardly ever are."""
import ctypes as C
import subprocess

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

comet = pytest.importorskip("paper_2102_05187_b200")
from layer_util import Matrix, random_mask  # noqa: E402

SOURCE = r"""
#include <pthread.h>
#include <stdint.h>
typedef int (*sddmm_t)(void *, const void *, const void *, int64_t, const void *, int64_t, int64_t, void *, void *);
struct job { sddmm_t call; void *handle; const void *a, *p, *q; int64_t r; void *out, *stream; int64_t times, refused; };
static void *run(void *arg) {
  struct job *j = arg;
  for (int64_t k = 0; k < j->times; ++k) j->refused += j->call(j->handle, j->a, j->p, j->r, j->q, j->r, j->r, j->out, j->stream) != 0;
  return 0;
}
typedef int (*spmv_t)(void *, const void *, const void *, void *, void *);
static void *run_spmv(void *arg) {
  struct job *j = arg;
  for (int64_t k = 0; k < j->times; ++k) j->refused += ((spmv_t)j->call)(j->handle, j->a, j->p, j->out, j->stream) != 0;
  return 0;
}
int hammer(struct job *jobs, int n, int spmv) {
  pthread_t t[16];
  int started = 0;
  for (; started < n && started < 16; ++started)
    if (pthread_create(t + started, 0, spmv ? run_spmv : run, jobs + started)) break;
  for (int i = 0; i < started; ++i) pthread_join(t[i], 0);
  return started;
}
"""


class Job(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("call", "handle", "a", "p", "q")] + [("r", C.c_int64), ("out", C.c_void_p), ("stream", C.c_void_p),
                                                                               ("times", C.c_int64), ("refused", C.c_int64)]


class Threads:
    """A thread for each of some sampled products of 64 columns, or products with a vector, each with a handle (without an allocator: nothing goes through Python) and a stream of its own."""

    def __init__(self, tmp_path, widths, times, spmv=False):
        self.spmv = spmv
        (tmp_path / "hammer.c").write_text(SOURCE)
        subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-pthread", "-o", str(tmp_path / "hammer.so"), str(tmp_path / "hammer.c")], check=True)
        self.hammer = C.CDLL(str(tmp_path / "hammer.so")).hammer
        self.lib, self.keep, self.jobs = comet.load_library(), [], (Job * len(widths))()
        rng = np.random.default_rng(0)
        for job, cols in zip(self.jobs, widths):
            m = Matrix(random_mask(256, cols, 0.3, rng), torch.float64 if spmv else torch.bfloat16, rng)
            handle, stream = C.c_void_p(), torch.cuda.Stream()
            assert self.lib.comet_create(C.byref(handle), None) == 0
            if spmv:
                x, out = torch.randn(cols, dtype=torch.float64, device="cuda"), torch.zeros(256, dtype=torch.float64, device="cuda")
                want = comet.spmv(m.t, x).clone()
                job.call, job.handle, job.a, job.p = C.cast(self.lib.comet_spmv, C.c_void_p), handle, C.addressof(m.t.c), x.data_ptr()
                job.out, job.stream, job.times = out.data_ptr(), stream.cuda_stream, times
                self.keep.append((m, handle, stream, x, out, want))
                continue
            P, Q = torch.randn(256, 64, device="cuda").bfloat16(), torch.randn(cols, 64, device="cuda").bfloat16()
            out = torch.zeros(m.t.nnz, dtype=torch.bfloat16, device="cuda")
            want = comet.sddmm(m.t, P, Q).val.clone()
            job.call = C.cast(self.lib.comet_sddmm, C.c_void_p)
            job.handle, job.a, job.p, job.q, job.r = handle, C.addressof(m.t.c), P.data_ptr(), Q.data_ptr(), 64
            job.out, job.stream, job.times = out.data_ptr(), stream.cuda_stream, times
            self.keep.append((m, handle, stream, P, Q, out, want))
        torch.cuda.synchronize()

    def run(self):
        assert self.hammer(self.jobs, len(self.jobs), self.spmv) == len(self.jobs)
        torch.cuda.synchronize()
        assert [j.refused for j in self.jobs] == [0] * len(self.jobs)
        for m, handle, *_, out, want in self.keep:
            assert torch.equal(out, want)
            self.lib.comet_destroy(handle)


def test_the_first_call_of_a_thread(cuda_device, tmp_path):
    Threads(tmp_path, (256,), 1).run()


def test_widths_beside_each_other(cuda_device, tmp_path):
    """What a kernel may take of shared memory belongs to the device, not to a call: narrow blocks must not take it from the wide ones beside them."""
    Threads(tmp_path, (64, 256, 128, 256, 192, 64), 20_000).run()


@pytest.mark.parametrize("kernel", ["stream", "stream2", "resident"])
def test_spmv_of_different_lengths(cuda_device, tmp_path, monkeypatch, kernel):
    """The same of comet_spmv, whose vectors lie in shared memory: 128 KB of it, or next to none."""
    monkeypatch.setenv("COMET_SEG_DOT_KERNEL", kernel)
    Threads(tmp_path, (64, 16_000, 300, 15_000, 9000, 64), 10_000, spmv=True).run()
