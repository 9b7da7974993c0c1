"""Thin Python binding of the feed-forward operators of libozimmu (C ABI declared in include/ozimmu_layers.h).

Argument marshalling only, as in `ozimmu`: PyTorch provides device memory and the current stream.  Matrices are torch
tensors with a token (or an output feature of a weight) per row, stride(1) == 1 and any row stride.
"""
import ctypes

import torch

from . import ozimmu
from .ozimmu import BAD_ARG, OK, OzimmuError

BF16, F16, F32, E4M3 = 0, 1, 2, 3
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
ACTIVATIONS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}

_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}

_c = ctypes
_int, _ptr, _size = _c.c_int, _c.c_void_p, _c.c_size_t
_SIGNATURES = {
    "ozimmu_linear_workspace_bytes": (_size, [_int] * 4),
    "ozimmu_linear": (_int, [_int] * 4 + [_ptr, _int, _ptr, _int, _ptr, _ptr, _int, _int, _ptr, _int, _ptr, _int, _ptr, _size, _ptr]),
    "ozimmu_linear_grad_workspace_bytes": (_size, [_int] * 5),
    "ozimmu_linear_grad": (_int, [_int] * 4 + [_ptr, _int] * 4 + [_int] + [_ptr, _int] * 2 + [_ptr, _ptr, _size, _ptr]),
}

_lib = None


def lib():
    """The loaded shared library.  Raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        handle = ozimmu.lib()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _type_of(x, what):
    kind = _TYPES.get(x.dtype)
    if kind is None or not x.is_cuda:
        raise ValueError(f"{what}: bfloat16, float16 or float32 CUDA tensor expected")
    return kind


def _ld(x, rows, cols, like, what):
    """Row stride of a [rows, cols] device tensor of `like`'s type, on its device, whose rows are contiguous."""
    if x.dim() != 2 or x.shape[0] != rows or x.shape[1] != cols:
        raise ValueError(f"{what}: [{rows}, {cols}] expected, got {list(x.shape)}")
    if x.dtype != like.dtype or x.device != like.device:
        raise ValueError(f"{what}: {like.dtype} on {like.device} expected")
    if cols > 1 and x.stride(1) != 1:
        raise ValueError(f"{what}: contiguous rows expected (stride(1) == 1)")
    ld = x.stride(0) if rows > 1 else max(1, cols)
    if ld < max(1, cols):
        raise ValueError(f"{what}: row stride {ld} smaller than {cols}")
    return ld


def _vector(x, n, like, what):
    if x.dim() != 1 or x.shape[0] != n or x.dtype != like.dtype or x.device != like.device or (n > 1 and x.stride(0) != 1):
        raise ValueError(f"{what}: contiguous [{n}] of {like.dtype} on {like.device} expected")
    return x.data_ptr()


def _workspace(given, nbytes, device):
    """(pointer, bytes) of the caller's workspace or of a new one, which has to live until the call has returned."""
    if given is None:
        given = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    return given, (given.data_ptr() if given is not None else None), (given.numel() * given.element_size() if given is not None else 0)


def linear_workspace_bytes(tokens, n_in, n_out, dtype):
    return lib().ozimmu_linear_workspace_bytes(tokens, n_in, n_out, _TYPES[dtype])


def linear(x, w, bias=None, residual=None, activation=ACT_NONE, pre=None, out=None, workspace=None):
    """y = act(x @ w.T + bias) + residual.  x [tokens, n_in], w [n_out, n_in], bias [n_out], residual [tokens, n_out].

    `pre`, a [tokens, n_out] tensor, receives x @ w.T + bias for linear_grad.  `out` may be `residual` itself.
    Asynchronous on the current stream."""
    kind = _type_of(x, "x")
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x and w: matrices expected")
    tokens, n_in = x.shape
    n_out = w.shape[0]
    ldx, ldw = _ld(x, tokens, n_in, x, "x"), _ld(w, n_out, n_in, x, "w")
    if out is None:
        out = torch.empty((tokens, n_out), dtype=x.dtype, device=x.device)
    ldy = _ld(out, tokens, n_out, x, "out")
    pbias = None if bias is None else _vector(bias, n_out, x, "bias")
    ldr = 0 if residual is None else _ld(residual, tokens, n_out, x, "residual")
    ldp = 0 if pre is None else _ld(pre, tokens, n_out, x, "pre")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, L.ozimmu_linear_workspace_bytes(tokens, n_in, n_out, kind) if workspace is None else 0, x.device)
    rc = L.ozimmu_linear(tokens, n_in, n_out, kind, x.data_ptr(), ldx, w.data_ptr(), ldw, pbias,
                         None if residual is None else residual.data_ptr(), ldr, activation,
                         None if pre is None else pre.data_ptr(), ldp, out.data_ptr(), ldy, ws, nbytes, ozimmu._stream())
    if rc != OK:
        raise OzimmuError(rc, "linear")
    return out


def linear_grad_workspace_bytes(tokens, n_in, n_out, dtype, activation=ACT_NONE):
    return lib().ozimmu_linear_grad_workspace_bytes(tokens, n_in, n_out, _TYPES[dtype], activation)


def linear_grad(dy, x, w, pre=None, activation=ACT_NONE, bias=True, dx=None, dw=None, db=None, want=("dx", "dw"), workspace=None):
    """Gradients (dx, dw, db) of linear from dy [tokens, n_out], its x, w and `pre` (not needed for ACT_NONE).

    db is None with bias=False; of dx and dw those in `want` are formed, the others are None.  Given tensors receive
    the results.  The gradient of linear's residual is dy itself."""
    kind = _type_of(dy, "dy")
    if dy.dim() != 2 or x.dim() != 2 or w.dim() != 2:
        raise ValueError("dy, x and w: matrices expected")
    tokens, n_out = dy.shape
    n_in = x.shape[1]
    lddy, ldx, ldw = _ld(dy, tokens, n_out, dy, "dy"), _ld(x, tokens, n_in, dy, "x"), _ld(w, n_out, n_in, dy, "w")
    if activation != ACT_NONE and pre is None:
        raise ValueError("pre: the values before the activation are needed")
    ldp = _ld(pre, tokens, n_out, dy, "pre") if activation != ACT_NONE else 0

    def result(given, name, shape):
        if name not in want:
            return None
        return torch.empty(shape, dtype=dy.dtype, device=dy.device) if given is None else given

    dx, dw = result(dx, "dx", (tokens, n_in)), result(dw, "dw", (n_out, n_in))
    db = (torch.empty(n_out, dtype=dy.dtype, device=dy.device) if db is None else db) if bias else None
    lddx = 0 if dx is None else _ld(dx, tokens, n_in, dy, "dx")
    lddw = 0 if dw is None else _ld(dw, n_out, n_in, dy, "dw")
    pdb = None if db is None else _vector(db, n_out, dy, "db")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, L.ozimmu_linear_grad_workspace_bytes(tokens, n_in, n_out, kind, activation)
                                  if workspace is None else 0, dy.device)
    rc = L.ozimmu_linear_grad(tokens, n_in, n_out, kind, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw,
                              pre.data_ptr() if activation != ACT_NONE else None, ldp, activation,
                              None if dx is None else dx.data_ptr(), lddx, None if dw is None else dw.data_ptr(), lddw, pdb,
                              ws, nbytes, ozimmu._stream())
    if rc != OK:
        raise OzimmuError(rc, "linear_grad")
    return dx, dw, db
