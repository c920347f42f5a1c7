"""Thin ctypes binding of libcomet.so (include/comet.h): argument marshalling only.

PyTorch is used for device memory and streams: operands are torch CUDA tensors whose `data_ptr()` is
passed through, the library allocates its data-dependent outputs through a callback that hands out
torch tensors (so they live in torch's caching allocator), and every call runs on torch's current
stream. Every step of the contractions and of the packing runs in the library's CUDA kernels; there is
no fallback: importing this module without a built libcomet.so, or calling it without a GPU, raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

D, CU, CN, S = 0, 1, 2, 3
F64 = 0
F32 = 1
BF16, F16, I32 = 2, 3, 4             # values of the layer operators; the entry numbers of transpose_symbolic
_TORCH_DTYPE = {F64: torch.float64, F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16, I32: torch.int32}
_VALUE_CODE = {t: c for c, t in _TORCH_DTYPE.items() if c != I32}
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = range(5)
BIAS_ROWS, BIAS_COLS = 0, 1


def _dtype_code(t: torch.Tensor) -> int:
    """comet_dtype_t of a value tensor (fp64 or fp32; anything else is refused here)."""
    if t.dtype == torch.float64:
        return F64
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"values must be float64 or float32, got {t.dtype}")


def _same_dtype(A, *tensors):
    want = _TORCH_DTYPE[A.c.dtype]
    for t in tensors:
        if t is not None and t.dtype != want:
            raise TypeError(f"dense operand is {t.dtype}, the sparse tensor's values are {want}")
    return want
MAX_ORDER = 4

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcomet.so")

STATUS_NAMES = {
    0: "COMET_OK", -1: "COMET_ERR_INVALID_ARG", -2: "COMET_ERR_UNSUPPORTED_FORMAT",
    -3: "COMET_ERR_COORD_OUT_OF_RANGE", -4: "COMET_ERR_DUPLICATE_COORD", -5: "COMET_ERR_INDEX_OVERFLOW",
    -6: "COMET_ERR_ALLOC", -7: "COMET_ERR_CUDA", -8: "COMET_ERR_WORKSPACE", -9: "COMET_ERR_MISALIGNED",
    -10: "COMET_ERR_INVALID_TENSOR",
}

EXPORTS = [
    "comet_create", "comet_destroy", "comet_status_string", "comet_last_cuda_error", "comet_kernel_launches",
    "comet_pack",
    "comet_sptensor_free", "comet_validate", "comet_spmv", "comet_spmm", "comet_ttv_symbolic", "comet_ttv",
    "comet_ttm_symbolic", "comet_ttm", "comet_mttkrp", "comet_spmv_static", "comet_pack_ex", "comet_ttm_symbolic_ex", "comet_reorder",
    "comet_elementwise_mul", "comet_spmm_from_host", "comet_spmm_epilogue", "comet_spmm_epilogue_backward", "comet_spmm_gated",
    "comet_spmm_gated_backward", "comet_sddmm", "comet_transpose_symbolic",
]


class CometError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str = ""):
        name = STATUS_NAMES.get(status, str(status))
        super().__init__(f"{what}: {name}{(' (' + detail + ')') if detail else ''}")
        self.status = status


class SpTensorStruct(C.Structure):
    _fields_ = [
        ("order", C.c_int32), ("dtype", C.c_int32),
        ("dims", C.c_int64 * MAX_ORDER),
        ("mode_order", C.c_int32 * MAX_ORDER),
        ("attr", C.c_int32 * MAX_ORDER),
        ("pos", C.c_void_p * MAX_ORDER), ("pos_len", C.c_int64 * MAX_ORDER),
        ("crd", C.c_void_p * MAX_ORDER), ("crd_len", C.c_int64 * MAX_ORDER),
        ("val", C.c_void_p), ("nnz", C.c_int64),
        ("owner", C.c_void_p),
    ]


class EpilogueStruct(C.Structure):
    _fields_ = [("act", C.c_int32), ("bias_along", C.c_int32), ("bias", C.c_void_p), ("residual", C.c_void_p), ("ldr", C.c_int64),
                ("preact", C.c_void_p), ("ldz", C.c_int64)]


_ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p)
_FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p, C.c_void_p)


class AllocatorStruct(C.Structure):
    _fields_ = [("alloc", _ALLOC_FN), ("free", _FREE_FN), ("ctx", C.c_void_p)]


_lib = None


def load_library():
    """Loads libcomet.so; raises if it has not been built (python -m paper_2102_05187_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2102_05187_b200.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    for name in EXPORTS:
        if not hasattr(lib, name):
            raise ImportError(f"libcomet.so does not export {name}")
    lib.comet_status_string.restype = C.c_char_p
    lib.comet_status_string.argtypes = [C.c_int]
    lib.comet_kernel_launches.restype = C.c_int64
    lib.comet_kernel_launches.argtypes = [C.c_void_p]
    for name in EXPORTS:
        if name not in ("comet_status_string", "comet_kernel_launches"):
            getattr(lib, name).restype = C.c_int
    # Declared argument types let the calls below pass plain integers (device addresses among them), which costs a
    # fraction of wrapping each one in a ctypes object: a call on a small tensor is bound by the host.
    t, i32, i64, p = C.POINTER(SpTensorStruct), C.c_int32, C.c_int64, C.c_void_p
    lib.comet_spmv.argtypes = [p, t, p, p, p]
    lib.comet_spmm.argtypes = [p, t, p, i64, i64, p, i64, p]
    lib.comet_ttv.argtypes = [p, t, i32, p, t, p]
    lib.comet_ttm.argtypes = [p, t, i32, p, i64, i64, t, p]
    lib.comet_ttv_symbolic.argtypes = [p, t, i32, p, p, t]
    lib.comet_ttm_symbolic_ex.argtypes = [p, t, i32, i64, p, p, t]
    lib.comet_mttkrp.argtypes = [p, t, i32, p, p, i64, p, i64, p]
    lib.comet_pack_ex.argtypes = [p, i32, p, i64, p, p, C.c_int, p, p, C.c_uint32, p, t]
    lib.comet_sptensor_free.argtypes = [p, t, p]
    lib.comet_spmm_epilogue.argtypes = [p, t, p, i64, i64, C.POINTER(EpilogueStruct), p, i64, p]
    lib.comet_spmm_epilogue_backward.argtypes = [p, t, t, p, i64, i64, i32, p, i64, p, i64, i32, p, p, p, i64, p]
    lib.comet_spmm_gated.argtypes = [p, t, t, p, i64, i64, i32, p, p, p, p, i64, p, i64, p]
    lib.comet_spmm_gated_backward.argtypes = [p, t, t, t, t, p, i64, i64, i32, p, p, i64, p, i64, p, p, p, p, p, i64, p]
    lib.comet_sddmm.argtypes = [p, t, p, i64, p, i64, i64, p, p]
    lib.comet_transpose_symbolic.argtypes = [p, t, p, t]
    _lib = lib
    return lib


def _stream_ptr():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream() -> int:
    """The current stream's address, without building a torch.cuda.Stream around it."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _require_cuda(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("operands must be CUDA tensors: the library has no host path")


class Handle:
    """A library handle whose allocator takes its blocks from torch's caching allocator (addresses: no tensor is built
    around a block that only the library sees)."""

    def __init__(self):
        if not torch.cuda.is_available():
            raise RuntimeError("libcomet needs a CUDA device: there is no CPU fallback")
        self.lib = load_library()
        self._live = {}

        torch.cuda.init()
        live = self._live
        raw_alloc, raw_delete = torch._C._cuda_cudaCachingAllocator_raw_alloc, torch._C._cuda_cudaCachingAllocator_raw_delete

        def _alloc(_ctx, nbytes, stream):
            try:
                ptr = raw_alloc(nbytes or 1, stream or 0)
            except Exception:
                return None
            live[ptr] = nbytes
            return ptr

        def _free(_ctx, ptr, _stream):
            if live.pop(ptr, None) is not None:
                raw_delete(ptr)

        self._give_back = raw_delete
        self._alloc_cb = _ALLOC_FN(_alloc)
        self._free_cb = _FREE_FN(_free)
        self._allocator = AllocatorStruct(self._alloc_cb, self._free_cb, None)
        self._h = C.c_void_p()
        st = self.lib.comet_create(C.byref(self._h), C.byref(self._allocator))
        if st:
            raise CometError(st, "comet_create")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self.lib.comet_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        # Tensors hold their handle, and views hold their tensors: nothing refers to a block any more. Blocks of tensors that
        # were alive when the handle was closed are still here (a closed handle frees none).
        try:
            self.close()
            while self._live:
                self._give_back(self._live.popitem()[0])
        except Exception:
            pass

    def kernel_launches(self) -> int:
        """Kernels launched through this handle so far."""
        return int(self.lib.comet_kernel_launches(self._h))

    def check(self, st: int, what: str):
        if st:
            detail = ""
            if st == -7:
                detail = f"cudaError {self.lib.comet_last_cuda_error(self._h)}"
            raise CometError(st, what, detail)


_default_handle = None


def default_handle() -> Handle:
    global _default_handle
    if _default_handle is None:
        _default_handle = Handle()
    return _default_handle


class SpTensor:
    """A sparse tensor descriptor plus whatever keeps its device arrays alive.

    Library-owned tensors (from pack / *_symbolic) are released on `free()` or garbage collection;
    caller-built ones (from `from_arrays`) borrow the torch tensors they were given.
    """

    def __init__(self, handle: Handle, struct: SpTensorStruct, keep=None):
        self.handle = handle
        self.c = struct
        self._ref = C.byref(struct)          # what the calls pass: made once
        self._keep = keep

    @property
    def order(self):
        return self.c.order

    @property
    def nnz(self):
        return self.c.nnz

    @property
    def dims(self):
        return tuple(self.c.dims[m] for m in range(self.c.order))

    @property
    def attr(self):
        return tuple(self.c.attr[l] for l in range(self.c.order))

    @property
    def mode_order(self):
        return tuple(self.c.mode_order[l] for l in range(self.c.order))

    def pos(self, l):
        return _from_ptr(self.c.pos[l], self.c.pos_len[l], torch.int32, self)

    def crd(self, l):
        return _from_ptr(self.c.crd[l], self.c.crd_len[l], torch.int32, self)

    @property
    def val(self):
        return _from_ptr(self.c.val, self.c.nnz, _TORCH_DTYPE[self.c.dtype], self)

    def free(self):
        if self.c.owner:
            self.handle.lib.comet_sptensor_free(self.handle._h, C.byref(self.c), _raw_stream())
        self._keep = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def with_values(self, val: torch.Tensor) -> "SpTensor":
        """The tensor of this one's structure (shared, and kept alive) and other values: nnz of them, float64, float32, bfloat16 or float16."""
        _require_cuda(val)
        if val.dtype not in _VALUE_CODE:
            raise TypeError(f"values must be float64, float32, bfloat16 or float16, got {val.dtype}")
        if val.numel() != self.c.nnz or not val.is_contiguous():
            raise ValueError(f"{self.c.nnz} contiguous values are needed")
        s = SpTensorStruct.from_buffer_copy(self.c)
        s.val = val.data_ptr() if val.numel() else 0
        s.dtype = _VALUE_CODE[val.dtype]
        s.owner = None
        return SpTensor(self.handle, s, keep=[self, val])

    @staticmethod
    def from_arrays(dims, mode_order, attr, pos, crd, val, handle: Handle | None = None) -> "SpTensor":
        """Describe caller-built level arrays (torch CUDA int32 tensors, float64 or float32 values, or bfloat16 / float16 ones for the
        layer operators; None where a level has none)."""
        handle = handle or default_handle()
        s = SpTensorStruct()
        order = len(dims)
        s.order, s.dtype = order, _VALUE_CODE[val.dtype] if val.dtype in _VALUE_CODE else _dtype_code(val)
        keep = []
        for m in range(order):
            s.dims[m] = int(dims[m])
            s.mode_order[m] = int(mode_order[m])
            s.attr[m] = int(attr[m])
            p = pos[m] if pos[m] is not None and pos[m].numel() else None
            c = crd[m] if crd[m] is not None and crd[m].numel() else None
            for t in (p, c):
                if t is not None:
                    _require_cuda(t)
                    assert t.dtype == torch.int32 and t.is_contiguous()
                    keep.append(t)
            s.pos[m] = 0 if p is None else p.data_ptr()
            s.pos_len[m] = 0 if p is None else p.numel()
            s.crd[m] = 0 if c is None else c.data_ptr()
            s.crd_len[m] = 0 if c is None else c.numel()
        _require_cuda(val)
        assert val.is_contiguous()
        keep.append(val)
        s.val = val.data_ptr() if val.numel() else 0
        s.nnz = val.numel()
        s.owner = None
        return SpTensor(handle, s, keep)


class _CudaArray:
    """n elements of device memory at an address, in the form torch takes; keeps the memory's owner alive."""
    __slots__ = ("__cuda_array_interface__", "_owner")


_TYPESTR = {torch.int32: ("<i4", 4), torch.float64: ("<f8", 8), torch.float32: ("<f4", 4), torch.uint8: ("|u1", 1),
            torch.int16: ("<i2", 2)}


def _from_ptr(ptr, n, dtype, owner):
    """A torch tensor aliasing n elements of device memory at ptr (kept alive by `owner`)."""
    if not ptr or n == 0:
        return torch.zeros(0, dtype=dtype, device="cuda")
    if dtype in (torch.bfloat16, torch.float16):
        return _from_ptr(ptr, n, torch.int16, owner).view(dtype)
    typestr, itemsize = _TYPESTR[dtype]
    array = _CudaArray()
    array.__cuda_array_interface__ = {"shape": (int(n),), "typestr": typestr, "data": (int(ptr), False),
                                      "version": 3, "strides": (itemsize,)}
    array._owner = owner
    return torch.as_tensor(array, device="cuda")


# ------------------------------------------------------------------------------------------- entry points

PACK_SUM_DUPLICATES = 1
PACK_CSR_HISTOGRAM = 2


def pack(coords, val, dims, mode_order, attr, handle: Handle | None = None, sum_duplicates: bool = False,
         csr_histogram: bool = False) -> SpTensor:
    """comet_pack / comet_pack_ex: COO (one int32 CUDA tensor per mode, any order) -> packed levels. Cells must be
    distinct unless `sum_duplicates`, which merges equal cells (values added in input order). `csr_histogram`:
    for [D,CU] matrices with rows of similar length, build the rows as a histogram instead of a full sort."""
    handle = handle or default_handle()
    order = len(dims)
    _require_cuda(val, *coords)
    coords = [c.contiguous() for c in coords]
    val = val.contiguous()
    assert all(c.dtype == torch.int32 for c in coords)
    h_dims = (C.c_int64 * order)(*[int(d) for d in dims])
    h_crd = (C.c_void_p * order)(*[c.data_ptr() for c in coords])
    h_mo = (C.c_int32 * order)(*[int(m) for m in mode_order])
    h_at = (C.c_int32 * order)(*[int(a) for a in attr])
    out = SpTensorStruct()
    st = handle.lib.comet_pack_ex(handle._h, order, h_dims, val.numel(), h_crd, val.data_ptr(), _dtype_code(val), h_mo, h_at,
                                  (PACK_SUM_DUPLICATES if sum_duplicates else 0) | (PACK_CSR_HISTOGRAM if csr_histogram else 0),
                                  _raw_stream(), C.byref(out))
    handle.check(st, "comet_pack")
    return SpTensor(handle, out)


def validate(t: SpTensor):
    t.handle.check(t.handle.lib.comet_validate(t.handle._h, C.byref(t.c), _stream_ptr()), "comet_validate")


def spmv(A: SpTensor, x: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
    _require_cuda(x)
    _same_dtype(A, x, y)
    if y is None:
        y = x.new_empty(A.c.dims[A.c.mode_order[0]])
    h = A.handle
    st = h.lib.comet_spmv(h._h, A._ref, x.data_ptr(), y.data_ptr(), _raw_stream())
    if st:
        h.check(st, "comet_spmv")
    return y


def spmm(A: SpTensor, B: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    _require_cuda(B)
    ldb, step = B.stride()
    assert step == 1
    R = B.shape[1]
    _same_dtype(A, B, out)
    if out is None:
        out = B.new_empty((A.c.dims[A.c.mode_order[0]], R))
    h = A.handle
    st = h.lib.comet_spmm(h._h, A._ref, B.data_ptr(), R, ldb, out.data_ptr(), out.stride(0), _raw_stream())
    if st:
        h.check(st, "comet_spmm")
    return out


def elementwise_mul(A: SpTensor, B: torch.Tensor, out_val: torch.Tensor | None = None) -> SpTensor:
    """C = A .* B for a dense B over A's modes (any strides): a tensor that shares A's level arrays (A must
    outlive it) and owns its values."""
    _require_cuda(B)
    dt = _same_dtype(A, B, out_val)
    modes = 2 if A.attr == (D, D, S) else A.c.order
    assert B.dim() == modes
    if out_val is None:
        out_val = torch.empty(A.c.nnz, dtype=dt, device=B.device)
    strides = (C.c_int64 * MAX_ORDER)(*[int(x) for x in B.stride()], *([0] * (MAX_ORDER - modes)))
    st = A.handle.lib.comet_elementwise_mul(A.handle._h, C.byref(A.c), _ptr(B), strides, _ptr(out_val), _stream_ptr())
    A.handle.check(st, "comet_elementwise_mul")
    s = SpTensorStruct.from_buffer_copy(A.c)
    s.val = out_val.data_ptr() if out_val.numel() else 0
    s.owner = None
    return SpTensor(A.handle, s, keep=[A, out_val])


# ---- layer operators: any of the four value types, every dense operand of A's own

def _rows_of(A):
    return A.c.dims[A.c.mode_order[0]]


def _cols_of(A):
    return A.c.dims[A.c.mode_order[1]]


def _operand(A, t, rows, R, what):
    """Checks a dense operand (rows x R, or rows values where R is None) and returns its address and leading dimension."""
    if t is None:
        return 0, 0
    if not t.is_cuda:
        raise ValueError("operands must be CUDA tensors: the library has no host path")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{what} is on device {t.get_device()}, the current device is another one")
    if t.dtype != _TORCH_DTYPE[A.c.dtype]:
        raise TypeError(f"{what} is {t.dtype}, the sparse tensor's values are {_TORCH_DTYPE[A.c.dtype]}")
    if R is None:
        if t.dim() != 1 or t.shape[0] != rows or (rows > 1 and t.stride(0) != 1):
            raise ValueError(f"{what} must be a contiguous vector of {rows} values")
        return t.data_ptr(), 0
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != R:
        raise ValueError(f"{what} must be {rows} x {R}, got {tuple(t.shape)}")
    ld, step = t.stride()
    if (step != 1 and R > 1) or (ld < R and rows > 1):
        raise ValueError(f"{what} must be row-major")
    return t.data_ptr(), max(ld, R)


def _layer_matrix(*matrices):
    for A in matrices:
        if A.c.order != 2:
            raise ValueError("the layer operators take matrices")
        if A.c.dtype == I32:
            raise TypeError("the structure of a transpose has no values")


def transpose_symbolic(A: SpTensor) -> SpTensor:
    """Structure of A stored column by column, for the backward passes: its `val` holds the int32 number in A of each entry."""
    _layer_matrix(A)
    out = SpTensorStruct()
    st = A.handle.lib.comet_transpose_symbolic(A.handle._h, A._ref, _raw_stream(), C.byref(out))
    A.handle.check(st, "comet_transpose_symbolic")
    return SpTensor(A.handle, out)


def spmm_epilogue(A: SpTensor, B: torch.Tensor, act: int = ACT_NONE, bias: torch.Tensor | None = None, bias_along: int | None = BIAS_ROWS,
                  residual: torch.Tensor | None = None, preact: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """act(A @ B + bias) + residual in one pass; `preact` (rows x R) receives A @ B + bias for the backward pass. The bias has a value
    per row of A (BIAS_ROWS) or per column of B (BIAS_COLS). `residual` may be `out`."""
    _layer_matrix(A)
    rows, R = _rows_of(A), B.shape[1]
    b, ldb = _operand(A, B, _cols_of(A), R, "B")
    along = BIAS_ROWS if bias is None or bias_along is None else bias_along
    if bias is not None and bias_along is None:
        raise ValueError("a bias needs bias_along")
    if out is None:
        out = B.new_empty((rows, R))
    c, ldc = _operand(A, out, rows, R, "out")
    e = EpilogueStruct(act, along, _operand(A, bias, rows if along == BIAS_ROWS else R, None, "bias")[0], *_operand(A, residual, rows, R, "residual"),
                       *_operand(A, preact, rows, R, "preact"))
    h = A.handle
    if rows == 0:
        return out
    st = h.lib.comet_spmm_epilogue(h._h, A._ref, b or out.data_ptr(), R, ldb, C.byref(e), c, ldc, _raw_stream())
    if st:
        h.check(st, "comet_spmm_epilogue")
    return out


def spmm_epilogue_backward(A: SpTensor, At: SpTensor | None, B: torch.Tensor | None, dC: torch.Tensor, act: int = ACT_NONE,
                           preact: torch.Tensor | None = None, bias_along: int | None = None, need_val: bool = True, need_dense: bool = True):
    """Gradients (dval, dB, dbias) of spmm_epilogue; None for what is not wanted (dbias: unless `bias_along` is given). At:
    transpose_symbolic(A), needed for dB; B is needed for dval. The residual's gradient is dC."""
    _layer_matrix(A)
    rows, cols, R = _rows_of(A), _cols_of(A), dC.shape[1]
    g, lddc = _operand(A, dC, rows, R, "dC")
    if act != ACT_NONE and preact is None:
        raise ValueError("the activation's gradient needs preact")
    if (need_val and B is None) or (need_dense and At is None):
        raise ValueError("dval needs B, dB needs At")
    z, ldz = _operand(A, preact, rows, R, "preact") if act != ACT_NONE else (0, 0)
    b, ldb = _operand(A, B, cols, R, "B") if need_val else (0, 0)
    dval = dC.new_empty(A.c.nnz) if need_val else None
    dB = dC.new_empty((cols, R)) if need_dense else None
    dbias = None if bias_along is None else dC.new_empty(rows if bias_along == BIAS_ROWS else R)
    if rows == 0 or cols == 0:                # nothing is stored: empty or zero gradients, but for the sums of dZ
        if rows == 0 or dbias is None:
            return dval, None if dB is None else dB.zero_(), None if dbias is None else dbias.zero_()
    h = A.handle
    st = h.lib.comet_spmm_epilogue_backward(h._h, A._ref, At._ref if need_dense and cols else None, b, R, ldb, act, z, ldz, g, lddc,
                                            0 if bias_along is None else bias_along, 0 if dbias is None else dbias.data_ptr(),
                                            dval.data_ptr() if dval is not None and A.c.nnz else 0, 0 if dB is None or not cols else dB.data_ptr(), R,
                                            _raw_stream())
    if st:
        h.check(st, "comet_spmm_epilogue_backward")
    return dval, dB, dbias


def _same_extents(G, U):
    if _rows_of(G) != _rows_of(U) or _cols_of(G) != _cols_of(U) or G.c.dtype != U.c.dtype or G.handle is not U.handle:
        raise ValueError("the two matrices must have the same extents, value type and handle")


def spmm_gated(G: SpTensor, U: SpTensor, B: torch.Tensor, act: int = ACT_SILU, bias_g: torch.Tensor | None = None,
               bias_u: torch.Tensor | None = None, preact=None, out: torch.Tensor | None = None) -> torch.Tensor:
    """act(G @ B + bias_g) * (U @ B + bias_u) in one pass; `preact`: a pair of rows x R tensors of one leading dimension that receive the
    two pre-activations for the backward pass."""
    _layer_matrix(G, U)
    _same_extents(G, U)
    rows, R = _rows_of(G), B.shape[1]
    b, ldb = _operand(G, B, _cols_of(G), R, "B")
    if out is None:
        out = B.new_empty((rows, R))
    c, ldc = _operand(G, out, rows, R, "out")
    (zg, ldz), (zu, ldu) = [_operand(G, z, rows, R, "preact") for z in (preact if preact is not None else (None, None))]
    if ldz != ldu:
        raise ValueError("the two pre-activations need one leading dimension")
    h = G.handle
    if rows == 0:
        return out
    st = h.lib.comet_spmm_gated(h._h, G._ref, U._ref, b or out.data_ptr(), R, ldb, act, _operand(G, bias_g, rows, None, "bias_g")[0],
                                _operand(G, bias_u, rows, None, "bias_u")[0], zg, zu, ldz, c, ldc, _raw_stream())
    if st:
        h.check(st, "comet_spmm_gated")
    return out


def spmm_gated_backward(G: SpTensor, Gt: SpTensor | None, U: SpTensor, Ut: SpTensor | None, B: torch.Tensor | None, dC: torch.Tensor, preact,
                        act: int = ACT_SILU, need_val: bool = True, need_dense: bool = True, need_bias: bool = False):
    """Gradients (dval_g, dval_u, dB, dbias_g, dbias_u) of spmm_gated; None for what is not wanted. Gt, Ut: transpose_symbolic of the two,
    needed for dB; B is needed for the values' gradients; `preact`: the pair that the forward pass kept."""
    _layer_matrix(G, U)
    _same_extents(G, U)
    rows, cols, R = _rows_of(G), _cols_of(G), dC.shape[1]
    g, lddc = _operand(G, dC, rows, R, "dC")
    (zg, ldz), (zu, ldu) = [_operand(G, z, rows, R, "preact") for z in preact]
    if ldz != ldu:
        raise ValueError("the two pre-activations need one leading dimension")
    if (need_val and B is None) or (need_dense and (Gt is None or Ut is None)):
        raise ValueError("the values' gradients need B, dB needs Gt and Ut")
    b, ldb = _operand(G, B, cols, R, "B") if need_val else (0, 0)
    dvals = [dC.new_empty(A.c.nnz) if need_val else None for A in (G, U)]
    dB = dC.new_empty((cols, R)) if need_dense else None
    dbias = [dC.new_empty(rows) if need_bias else None for _ in (G, U)]
    if rows == 0:
        return (*dvals, None if dB is None else dB.zero_(), *dbias)
    h = G.handle
    dense = dB is not None and cols > 0
    st = h.lib.comet_spmm_gated_backward(h._h, G._ref, Gt._ref if dense else None, U._ref, Ut._ref if dense else None, b, R, ldb, act, zg, zu, ldz, g,
                                         lddc, *[0 if t is None else t.data_ptr() for t in dbias],
                                         *[t.data_ptr() if t is not None and t.numel() else 0 for t in dvals], dB.data_ptr() if dense else 0, R,
                                         _raw_stream())
    if st:
        h.check(st, "comet_spmm_gated_backward")
    return (*dvals, dB, *dbias)


def sddmm(A: SpTensor, P: torch.Tensor, Q: torch.Tensor, out_val: torch.Tensor | None = None) -> SpTensor:
    """P @ Q.T at A's stored cells: a tensor that shares A's level arrays (A must outlive it) and owns its values. A's values are not read."""
    _layer_matrix(A)
    R = P.shape[1]
    p, ldp = _operand(A, P, _rows_of(A), R, "P")
    q, ldq = _operand(A, Q, _cols_of(A), R, "Q")
    if out_val is None:
        out_val = P.new_empty(A.c.nnz)
    o = _operand(A, out_val, A.c.nnz, None, "out_val")[0]
    h = A.handle
    st = h.lib.comet_sddmm(h._h, A._ref, p, ldp, q, ldq, R, o, _raw_stream())
    if st:
        h.check(st, "comet_sddmm")
    return A.with_values(out_val)


def ttv_symbolic(X: SpTensor, mode: int, out_attr=None) -> SpTensor:
    """Structure of X x_mode v: one level fewer than X. Default format: CSR [D,CU] for a 3-order X,
    CSF [CU,CU,CU] for a 4-order X."""
    out = SpTensorStruct()
    n = X.c.order - 1
    if out_attr is None:
        out_attr = (D, CU) if n == 2 else (CU,) * n
    assert len(out_attr) == n
    h_at = (C.c_int32 * n)(*out_attr)
    st = X.handle.lib.comet_ttv_symbolic(X.handle._h, C.byref(X.c), mode, h_at, _raw_stream(), C.byref(out))
    X.handle.check(st, "comet_ttv_symbolic")
    return SpTensor(X.handle, out)


def ttv(X: SpTensor, mode: int, v: torch.Tensor, Y: SpTensor | None = None) -> SpTensor:
    _require_cuda(v)
    _same_dtype(X, v)
    if Y is None:
        Y = ttv_symbolic(X, mode)
    st = X.handle.lib.comet_ttv(X.handle._h, X._ref, mode, v.data_ptr(), Y._ref, _raw_stream())
    X.handle.check(st, "comet_ttv")
    return Y


def ttm_symbolic(X: SpTensor, mode: int, R: int, out_attr=None) -> SpTensor:
    """Structure of X x_mode U. out_attr: None (compressed levels + dense last level) or, for a 3-order X,
    (CN, S, D): the mode-generic form with one coordinate pair per stored fiber."""
    out = SpTensorStruct()
    h_at = None if out_attr is None else (C.c_int32 * X.c.order)(*out_attr)
    st = X.handle.lib.comet_ttm_symbolic_ex(X.handle._h, C.byref(X.c), mode, R, h_at, _raw_stream(), C.byref(out))
    X.handle.check(st, "comet_ttm_symbolic")
    return SpTensor(X.handle, out)


def ttm(X: SpTensor, mode: int, U: torch.Tensor, Y: SpTensor | None = None) -> SpTensor:
    _require_cuda(U)
    assert U.dim() == 2 and U.stride(1) == 1
    R = U.shape[1]
    _same_dtype(X, U)
    if Y is None:
        Y = ttm_symbolic(X, mode, R)
    st = X.handle.lib.comet_ttm(X.handle._h, X._ref, mode, U.data_ptr(), R, U.stride(0), Y._ref, _raw_stream())
    X.handle.check(st, "comet_ttm")
    return Y


def mttkrp(X: SpTensor, mode: int, factors, out: torch.Tensor | None = None) -> torch.Tensor:
    """factors: one (dims[m] x R) CUDA tensor per mode; the entry at `mode` may be None."""
    live = [f for m, f in enumerate(factors) if m != mode and f is not None]
    _require_cuda(*live)
    R = live[0].shape[1]
    assert all(f.dim() == 2 and f.stride(1) == 1 and f.shape[1] == R for f in live)
    rows = X.c.dims[mode]
    dt = _same_dtype(X, out, *live)
    if out is None:
        out = torch.empty((rows, R), dtype=dt, device=live[0].device)
    order = X.c.order
    assert len(factors) == order
    h_f = (C.c_void_p * order)(*[0 if (m == mode or f is None) else f.data_ptr() for m, f in enumerate(factors)])
    h_ld = (C.c_int64 * order)(*[0 if (m == mode or f is None) else f.stride(0) for m, f in enumerate(factors)])
    st = X.handle.lib.comet_mttkrp(X.handle._h, X._ref, mode, h_f, h_ld, R, out.data_ptr(), out.stride(0), _raw_stream())
    X.handle.check(st, "comet_mttkrp")
    return out


def reorder(coords, dims, iterations: int = 5, handle: Handle | None = None):
    """comet_reorder: new numbers for the indices of every mode (one int32 CUDA tensor per mode) that gather
    the entries around the diagonal. Apply with `label[m][coords[m].long()]`; dense operands and results
    indexed by mode m move their rows accordingly."""
    handle = handle or default_handle()
    order = len(dims)
    _require_cuda(*coords)
    coords = [c.contiguous() for c in coords]
    assert all(c.dtype == torch.int32 for c in coords)
    labels = [torch.empty(int(d), dtype=torch.int32, device=coords[0].device) for d in dims]
    h_dims = (C.c_int64 * order)(*[int(d) for d in dims])
    h_crd = (C.c_void_p * order)(*[c.data_ptr() for c in coords])
    h_lab = (C.c_void_p * order)(*[l.data_ptr() for l in labels])
    st = handle.lib.comet_reorder(handle._h, C.c_int32(order), h_dims, C.c_int64(coords[0].numel()), h_crd,
                                  C.c_int32(iterations), h_lab, _stream_ptr())
    handle.check(st, "comet_reorder")
    return labels


def spmm_from_host(h_coords, h_val, dims, h_B, h_out, handle: Handle | None = None):
    """comet_spmm_from_host: the whole SpMM path from HOST buffers (pinned host tensors make the copies
    asynchronous): COO entries and B in, CSR packing, multiplication, C back into `h_out`, with B and C
    travelling in column chunks so that the two directions of the bus overlap. Returns after the result has
    landed in `h_out`."""
    handle = handle or default_handle()
    tensors = list(h_coords) + [h_val, h_B, h_out]
    if any(t.is_cuda for t in tensors):
        raise ValueError("spmm_from_host takes host tensors")
    assert len(h_coords) == 2 and all(c.dtype == torch.int32 and c.is_contiguous() for c in h_coords)
    assert h_val.is_contiguous() and h_B.dim() == 2 and h_out.dim() == 2 and h_B.stride(1) == 1 and h_out.stride(1) == 1
    assert h_B.dtype == h_val.dtype == h_out.dtype
    R = int(h_B.shape[1])
    assert tuple(h_out.shape) == (int(dims[0]), R) and int(h_B.shape[0]) == int(dims[1])
    h_dims = (C.c_int64 * 2)(int(dims[0]), int(dims[1]))
    st = handle.lib.comet_spmm_from_host(handle._h, h_dims, C.c_int64(h_val.numel()), _ptr(h_coords[0]), _ptr(h_coords[1]),
                                         _ptr(h_val), C.c_int32(_dtype_code(h_val)), _ptr(h_B), C.c_int64(h_B.stride(0)),
                                         C.c_int64(R), _ptr(h_out), C.c_int64(h_out.stride(0)), _stream_ptr())
    handle.check(st, "comet_spmm_from_host")
    return h_out
