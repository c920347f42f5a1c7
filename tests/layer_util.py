"""Helpers of the layer operators' tests: random matrices in the three formats, the operators in 64 bits on the CPU (dense, from
their definitions), and the tolerances.

Tolerances, per element. u = 2^-53 for fp64 and 2^-24 otherwise (the width the kernels compute in), n = the longest row,
N = sum |a||b| + |bias|.
  z:        fp64 (n + 8) u N; fp32: at most 128 terms added in fp32, the rest in double, so 130 u N + u |z| for narrowing the sum; 16-bit: n + 8
            additions in fp32, (n + 8) u N.
  f(z):     |f'| <= 1.13 for every activation here, and evaluating f costs at most 16 u |z| (erf, tanh and exp are good to a few
            units in the last place and 1 + erf, 1 + tanh, 1 + exp cancel to an absolute error of that order).
  stored:   half a step of the type, eps / 2 of the value, plus half of the smallest subnormal step (fp16).
"""
import numpy as np
import torch

import paper_2102_05187_b200 as comet
from paper_2102_05187_b200 import CN, CU, D, S

TYPES = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = {"none": comet.ACT_NONE, "relu": comet.ACT_RELU, "gelu": comet.ACT_GELU, "gelu_tanh": comet.ACT_GELU_TANH, "silu": comet.ACT_SILU}
TINY = {torch.float64: 0.0, torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def half_step(t):
    return torch.finfo(t).eps / 2


def u_of(t):
    return 2.0 ** -53 if t == torch.float64 else 2.0 ** -24


def values(shape, dt, rng, scale=1.0):
    """Random values of a type, and the same in 64 bits."""
    t = torch.as_tensor(rng.standard_normal(shape) * scale).to(dt)
    return t, t.double()


class Matrix:
    """mask (rows x cols, bool) -> the tensor on the device in a format, and its dense values in 64 bits."""

    def __init__(self, mask, dt, rng, fmt="csr", scale=1.0):
        self.mask = mask = np.asarray(mask, dtype=bool)
        rows, cols = mask.shape
        r, c = np.nonzero(mask)
        self.val, v64 = values(r.size, dt, rng, scale)
        self.dense = torch.zeros(rows, cols, dtype=torch.float64)
        self.dense[r, c] = v64
        self.rc = (torch.as_tensor(r), torch.as_tensor(c))
        self.longest = int(mask.sum(1).max()) if rows and cols else 0
        self.tallest = int(mask.sum(0).max()) if rows and cols else 0
        i32 = lambda a: torch.as_tensor(np.asarray(a)).to(torch.int32).cuda()  # noqa: E731
        pos = np.concatenate([[0], np.cumsum(mask.sum(1))])
        val = self.val.cuda()
        if fmt == "csr":
            self.t = comet.SpTensor.from_arrays((rows, cols), (0, 1), (D, CU), [i32([rows]), i32(pos)], [None, i32(c)], val)
        elif fmt == "dcsr":
            full = np.nonzero(mask.any(1))[0] if cols else np.zeros(0, int)
            self.t = comet.SpTensor.from_arrays((rows, cols), (0, 1), (CU, CU), [i32([0, full.size]), i32(np.concatenate([pos[:-1][full], [r.size]]))],
                                                [i32(full), i32(c)], val)
        elif fmt == "coo":
            self.t = comet.SpTensor.from_arrays((rows, cols), (0, 1), (CN, S), [i32([0, r.size]), None], [i32(r), i32(c)], val)
        else:                                              # stored with the modes the other way round: rows are mode 1
            assert fmt == "csr10"
            self.t = comet.SpTensor.from_arrays((cols, rows), (1, 0), (D, CU), [i32([rows]), i32(pos)], [None, i32(c)], val)


def random_mask(rows, cols, density, rng, empty=()):
    m = rng.random((rows, cols)) < density
    for i in empty:
        m[i % max(rows, 1)] = False
    return m


def place(t, pad, off=0, fill=float("nan")):
    """t on the device as a view with `pad` more columns per row and `off` elements in front, all of them `fill`."""
    t = t.cuda()
    rows, R = t.shape
    flat = torch.full((off + rows * (R + pad),), fill, dtype=t.dtype, device="cuda")
    view = flat[off:].view(rows, R + pad)[:, :R]
    view.copy_(t)
    return view


def act64(name, z):
    f = torch.nn.functional
    return {"none": lambda x: x * 1.0, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda x: f.gelu(x, approximate="tanh"), "silu": f.silu}[name](z)


def slope64(name, z):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(act64(name, z).sum(), z)[0]


def z_bound(dt, n, N, z):
    u = u_of(dt)
    if dt == torch.float32:
        return 130 * u * N + 2 * u * z.abs()
    return (n + 8) * u * N


def act_bound(dt, dz, z):
    return 1.13 * dz + 16 * u_of(dt) * z.abs()


def stored(dt, want, bound):
    return bound + half_step(dt) * (want.abs() + bound) + TINY[dt]


def assert_within(got, want, bound, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, tuple(got.shape), tuple(want.shape))
    err = (got - want).abs()
    bad = ~(err <= bound)
    if bad.any():
        at = int(torch.argmax(torch.where(bad, (err - bound).nan_to_num(float("inf")), torch.full_like(err, -1.0))))
        raise AssertionError(f"{what}: {int(bad.sum())} of {err.numel()} off; at {np.unravel_index(at, tuple(err.shape))}: got {got.flatten()[at]:.9g}, "
                             f"want {want.flatten()[at]:.9g}, bound {bound.flatten()[at]:.3g}")
