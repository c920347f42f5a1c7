"""The layer operators' part of the boundary that can be checked without a GPU: enumerations and the epilogue struct agree with the header, and
the binding refuses operands before it calls the library."""
import ctypes
import os
import re

import pytest
import torch

import paper_2102_05187_b200 as comet
from paper_2102_05187_b200 import binding

HEADER = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "comet.h")).read()


def value(name):
    return int(re.search(r"\b%s = (-?\d+)" % name, HEADER).group(1))


def test_enumerations_match_the_header():
    for name in ("ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_GELU_TANH", "ACT_SILU", "BIAS_ROWS", "BIAS_COLS"):
        assert getattr(comet, name) == value("COMET_" + name)
    for name in ("F64", "F32", "BF16", "F16", "I32"):
        assert getattr(binding, name) == value("COMET_" + name)


def test_epilogue_struct_matches_the_header():
    e = binding.EpilogueStruct
    assert ctypes.sizeof(e) == 48
    assert [(n, getattr(e, n).offset) for n, _ in e._fields_] == [("act", 0), ("bias_along", 4), ("bias", 8), ("residual", 16), ("ldr", 24), ("preact", 32),
                                                                  ("ldz", 40)]
    body = re.search(r"typedef struct \{([^}]*)\} comet_epilogue_t;", HEADER).group(1)
    assert re.findall(r"(\w+);", re.sub(r"/\*.*?\*/", "", body)) == [n for n, _ in e._fields_]


def _matrix(dtype):
    s = binding.SpTensorStruct()
    s.order, s.dtype = 2, dtype
    s.dims[0], s.dims[1] = 3, 4
    s.mode_order[0], s.mode_order[1] = 0, 1
    return comet.SpTensor(None, s)


def test_operands_are_checked_before_the_call():
    A = _matrix(binding.F32)
    with pytest.raises(ValueError):                        # no host path
        comet.spmm_epilogue(A, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        comet.sddmm(A, torch.zeros(3, 2), torch.zeros(4, 2))
    with pytest.raises(TypeError):                         # the structure of a transpose is no matrix of values
        comet.spmm_epilogue(_matrix(binding.I32), torch.zeros(4, 2))
    three = _matrix(binding.F32)
    three.c.order = 3
    with pytest.raises(ValueError):
        comet.spmm_gated(three, three, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        comet.spmm_gated(A, _matrix(binding.F64), torch.zeros(4, 2))
    with pytest.raises(ValueError):
        A.with_values(torch.zeros(1))
