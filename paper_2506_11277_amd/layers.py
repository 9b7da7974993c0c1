"""Thin Python binding of the feed-forward operators of libozimmu (C ABI declared in include/ozimmu_layers.h).

Argument marshalling only, as in `ozimmu`: PyTorch provides device memory and the current stream.  Matrices are torch
tensors with a token (or an output feature of a weight) per row, stride(1) == 1 and any row stride.

Nothing here is recorded by autograd: results do not require gradients whatever the operands do (linear_grad forms linear's;
to use them under autograd, call both from a torch.autograd.Function), and a given output is overwritten without a trace in its
version counter.  AdamW.step does raise the counters of what it writes, so that autograd notices a saved weight that changed.
"""
import ctypes
from array import array
from functools import lru_cache
from operator import attrgetter

import torch
from torch.autograd.graph import increment_version

from . import ozimmu
from .ozimmu import BAD_ARG, OK, OzimmuError

BF16, F16, F32, E4M3 = 0, 1, 2, 3
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
ACTIVATIONS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}

_dtype, _shape = attrgetter("dtype"), attrgetter("shape")

BLOCK = 256          # values that share a scale where AdamW's moments are held in 8 bits

_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}

_c = ctypes
_int, _ptr, _size = _c.c_int, _c.c_void_p, _c.c_size_t
_SIGNATURES = {
    "ozimmu_linear_workspace_bytes": (_size, [_int] * 5),
    "ozimmu_linear": (_int, [_int] * 4 + [_ptr, _int, _ptr, _int, _ptr, _ptr, _int, _int, _ptr, _int, _ptr, _int, _ptr, _size, _ptr]),
    "ozimmu_linear_grad_workspace_bytes": (_size, [_int] * 6),
    "ozimmu_linear_grad": (_int, [_int] * 4 + [_ptr, _int] * 4 + [_int] + [_ptr, _int] * 2 + [_ptr, _ptr, _size, _ptr]),
    "ozimmu_moe_workspace_bytes": (_size, [_int] * 6),
    "ozimmu_linear8_workspace_bytes": (_size, [_int] * 4),
    "ozimmu_linear8": (_int, [_int] * 4 + [_ptr, _int, _ptr] * 2 + [_ptr, _ptr, _int, _int, _ptr, _int, _ptr, _int, _ptr, _size, _ptr]),
    "ozimmu_linear8_grad_workspace_bytes": (_size, [_int] * 8),
    "ozimmu_linear8_grad": (_int, [_int] * 4 + [_ptr, _int] + [_ptr, _int, _ptr] * 3 + [_int] + [_ptr, _int] * 2 + [_ptr, _ptr, _size, _ptr]),
    "ozimmu_quantise": (_int, [_int] * 3 + [_ptr, _int, _ptr, _int, _ptr, _ptr]),
    "ozimmu_rms_norm": (_int, [_int] * 3 + [_ptr, _int, _ptr, _int, _ptr, _c.c_double, _ptr, _int, _ptr, _int, _ptr, _int, _ptr, _ptr]),
    "ozimmu_rms_norm_grad_workspace_bytes": (_size, [_int] * 2),
    "ozimmu_rms_norm_grad": (_int, [_int] * 3 + [_ptr, _int, _ptr, _int, _ptr, _c.c_double] + [_ptr, _int] * 2 + [_ptr, _ptr, _size, _ptr]),
    "ozimmu_moe": (_int, [_int] * 7 + [_ptr, _int] + [_ptr] * 6 + [_int, _ptr, _size, _ptr]),
}


class _AdamWTensor(ctypes.Structure):
    _fields_ = [("param", _ptr), ("grad", _ptr), ("m", _ptr), ("v", _ptr), ("m_scale", _ptr), ("v_scale", _ptr), ("copy", _ptr),
                ("count", _c.c_int64), ("param_type", _int), ("grad_type", _int), ("state_type", _int), ("copy_type", _int)]


_SIGNATURES["ozimmu_adamw"] = (_int, [_int, _c.POINTER(_AdamWTensor), _ptr] + [_c.c_double] * 5 +
                               [_c.c_longlong, _c.c_uint32, _ptr])

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


def _sizes(*sizes):
    """The sizes, which the library takes as ints (larger ones would arrive there as others)."""
    for n in sizes:
        if not -1 << 31 <= n < 1 << 31:
            raise ValueError(f"sizes: {n} is more than the library takes")
    return sizes


def _ld(x, rows, cols, like, what):
    """Row stride of a [rows, cols] device tensor of `like`'s type, on its device, whose rows are contiguous."""
    if x.shape != (rows, cols):
        raise ValueError(f"{what}: [{rows}, {cols}] expected, got {list(x.shape)}")
    if x.dtype is not like.dtype or x.get_device() != like.get_device():
        raise ValueError(f"{what}: {like.dtype} on {like.device} expected")
    ld, step = x.stride()
    if (rows | cols) >> 30:
        raise ValueError(f"{what}: sizes below 2^30 expected, got {list(x.shape)}")
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: contiguous rows expected (stride(1) == 1)")
    if rows <= 1:
        return cols or 1
    if ld < cols or ld < 1 or ld >> 31:
        raise ValueError(f"{what}: row stride {ld} smaller than {cols} or not below 2^31")
    return ld


def _vector(x, n, like, what):
    if x.shape != (n,) or x.dtype is not like.dtype or x.get_device() != like.get_device() or (n > 1 and x.stride(0) != 1):
        raise ValueError(f"{what}: contiguous [{n}] of {like.dtype} on {like.device} expected")
    return x.data_ptr()


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = ozimmu._raw_stream


def _stream(index, what):
    """The current stream of the current device, on which the tensors have to be."""
    if index != _get_device():
        raise ValueError(f"{what}: tensors on cuda:{index}, which is not the current device")
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _workspace(given, nbytes, device):
    """(tensor, pointer, bytes) of the caller's workspace or of a new one, which has to live until the call has returned."""
    if given is None:
        given = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    elif given.device != device or not given.is_contiguous():
        raise ValueError(f"workspace: contiguous tensor on {device} expected")
    return given, (given.data_ptr() if given is not None else None), (given.numel() * given.element_size() if given is not None else 0)


def _aligned(x, ldx, *rest):
    """Whether every row of the matrices (tensor, row stride, ...) starts on 16 bytes."""
    bits, size = x.data_ptr() | ldx * x.element_size(), x.element_size()
    for w, ld in zip(rest[::2], rest[1::2]):
        bits |= w.data_ptr() | ld * size
    return 0 if bits & 15 else 1


def linear_workspace_bytes(tokens, n_in, n_out, dtype, aligned=True):
    """Bytes of workspace for linear; aligned: every row of x and w starts on 16 bytes (with less a slower way is taken)."""
    return lib().ozimmu_linear_workspace_bytes(*_sizes(tokens, n_in, n_out), _TYPES[dtype], int(aligned))


def linear(x, w, bias=None, residual=None, activation=ACT_NONE, pre=None, out=None, workspace=None):
    """y = act(x @ w.T + bias) + residual.  x [tokens, n_in], w [n_out, n_in], bias [n_out], residual [tokens, n_out].

    `pre`, a [tokens, n_out] tensor, receives x @ w.T + bias for linear_grad.  `out` may be `residual` itself.
    Asynchronous on the current stream."""
    kind = _type_of(x, "x")
    try:
        (tokens, n_in), (n_out, _) = x.shape, w.shape
    except ValueError:
        raise ValueError("x and w: matrices expected") from None
    ldx, ldw = _ld(x, tokens, n_in, x, "x"), _ld(w, n_out, n_in, x, "w")
    if out is None:
        out = torch.empty((tokens, n_out), dtype=x.dtype, device=x.device)
    ldy = _ld(out, tokens, n_out, x, "out")
    pbias = None if bias is None else _vector(bias, n_out, x, "bias")
    ldr = 0 if residual is None else _ld(residual, tokens, n_out, x, "residual")
    ldp = 0 if pre is None else _ld(pre, tokens, n_out, x, "pre")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, L.ozimmu_linear_workspace_bytes(tokens, n_in, n_out, kind, _aligned(x, ldx, w, ldw))
                                  if workspace is None else 0, x.device)
    rc = L.ozimmu_linear(tokens, n_in, n_out, kind, x.data_ptr(), ldx, w.data_ptr(), ldw, pbias,
                         None if residual is None else residual.data_ptr(), ldr, activation,
                         None if pre is None else pre.data_ptr(), ldp, out.data_ptr(), ldy, ws, nbytes,
                         _stream(x.get_device(), "linear"))
    if rc != OK:
        raise OzimmuError(rc, "linear")
    return out


def linear_grad_workspace_bytes(tokens, n_in, n_out, dtype, activation=ACT_NONE, aligned=True):
    """Bytes of workspace for linear_grad; aligned: every row of dy, x and w starts on 16 bytes."""
    return lib().ozimmu_linear_grad_workspace_bytes(*_sizes(tokens, n_in, n_out), _TYPES[dtype], activation, int(aligned))


def linear_grad(dy, x, w, pre=None, activation=ACT_NONE, bias=True, dx=None, dw=None, db=None, want=("dx", "dw"), workspace=None):
    """Gradients (dx, dw, db) of linear from dy [tokens, n_out], its x, w and `pre` (not needed for ACT_NONE).

    db is None with bias=False; of dx and dw those in `want` are formed, the others are None (what is formed together may be summed in
    another order than alone).  Given tensors receive the results.  The gradient of linear's residual is dy itself."""
    kind = _type_of(dy, "dy")
    try:
        (tokens, n_out), (_, n_in) = dy.shape, x.shape
    except ValueError:
        raise ValueError("dy and x: matrices expected") from None
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
    keep, ws, nbytes = _workspace(workspace, L.ozimmu_linear_grad_workspace_bytes(tokens, n_in, n_out, kind, activation,
                                                                       _aligned(dy, lddy, x, ldx, w, ldw))
                                  if workspace is None else 0, dy.device)
    rc = L.ozimmu_linear_grad(tokens, n_in, n_out, kind, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw,
                              pre.data_ptr() if activation != ACT_NONE else None, ldp, activation,
                              None if dx is None else dx.data_ptr(), lddx, None if dw is None else dw.data_ptr(), lddw, pdb,
                              ws, nbytes, _stream(dy.get_device(), "linear_grad"))
    if rc != OK:
        raise OzimmuError(rc, "linear_grad")
    return dx, dw, db


def adamw_state(params, bits=32):
    """Moments of new parameters for AdamW: (m, v, m_scale, v_scale), lists with a tensor per parameter.  bits=32: float32,
    the scales None; bits=8: float8_e4m3fn values of m and of the root of v, one float32 scale of each per BLOCK values."""
    if bits not in (8, 32):
        raise ValueError("bits: 8 or 32 expected")
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn

    def zeros():
        return [torch.zeros(p.numel(), dtype=torch.float32 if bits == 32 else torch.uint8, device=p.device).view(kind).view(p.shape) for p in params]

    def scales():
        return None if bits == 32 else [torch.zeros(-(-p.numel() // BLOCK), dtype=torch.float32, device=p.device) for p in params]

    return zeros(), zeros(), scales(), scales()


class AdamW:
    """AdamW over many tensors at once: a plan for parameters and moments that stay where they are.

    params: float32, bfloat16 or float16; m, v and their scales as adamw_state gives them (float32 moments, or float8_e4m3fn
    ones with scales); copies: None, or a bfloat16 or float16 tensor per parameter that receives it with every step.
    The plan holds the tensors, which may not overlap; one that is replaced or resized needs a new plan."""

    def __init__(self, params, m, v, m_scale=None, v_scale=None, copies=None):
        n = len(params)
        given = [params, m, v] + [x for x in (m_scale, v_scale, copies) if x is not None]
        if any(len(x) != n for x in given):
            raise ValueError("AdamW: lists of one length expected")
        self._held = [list(x) for x in given]              # (the tensors: their addresses are what every step uses)
        self._weights = self._held[0] + (self._held[-1] if copies is not None else [])
        self._list = (_AdamWTensor * n)()
        self._shapes = [p.shape for p in params]
        self._device = params[0].device if n else None
        self._devices = [p.get_device() for p in params]
        spans = []                                         # what a step writes: addresses and bytes
        for i, (t, p) in enumerate(zip(self._list, params)):
            kind = _type_of(p, f"params[{i}]")
            eight = m[i].dtype == torch.float8_e4m3fn
            expected = torch.float8_e4m3fn if eight else torch.float32
            for x, what, dtypes in ((p, "params", (p.dtype,)), (m[i], "m", (expected,)), (v[i], "v", (expected,)),
                                    (None if copies is None else copies[i], "copies", (torch.bfloat16, torch.float16))):
                if x is not None and (x.dtype not in dtypes or x.shape != p.shape or x.device != self._device or not x.is_contiguous()):
                    raise ValueError(f"{what}[{i}]: contiguous {list(p.shape)} of {dtypes[0]} on {self._device} expected")
            t.param, t.m, t.v, t.count, t.param_type, t.grad_type = p.data_ptr(), m[i].data_ptr(), v[i].data_ptr(), p.numel(), kind, -1
            t.state_type = E4M3 if eight else F32
            if eight:
                for x, what in ((m_scale, "m_scale"), (v_scale, "v_scale")):
                    if x is None or x[i].dtype != torch.float32 or x[i].numel() != -(-p.numel() // BLOCK) or x[i].device != self._device or not x[i].is_contiguous():
                        raise ValueError(f"{what}[{i}]: contiguous [{-(-p.numel() // BLOCK)}] of float32 on {self._device} expected")
                t.m_scale, t.v_scale = m_scale[i].data_ptr(), v_scale[i].data_ptr()
            if copies is not None:
                t.copy, t.copy_type = copies[i].data_ptr(), _TYPES[copies[i].dtype]
            count = t.count
            if count:
                spans += [(t.param, count * (4 if kind == F32 else 2)), (t.m, count * (1 if eight else 4)), (t.v, count * (1 if eight else 4))]
                if eight:
                    spans += [(t.m_scale, 4 * -(-count // BLOCK)), (t.v_scale, 4 * -(-count // BLOCK))]
                if copies is not None:
                    spans.append((t.copy, 2 * count))
        spans.sort()
        if any(start + size > after for (start, size), (after, _) in zip(spans, spans[1:])):
            raise ValueError("AdamW: tensors that overlap (each may be in the lists once)")
        self._grad_types = None

    def step(self, grads, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, seed=0):
        """One step with the gradients `grads`, contiguous tensors of the parameters' shapes; `step` counts from 1; `seed`
        makes the random words that 8-bit moments are rounded with.  Asynchronous on the current stream."""
        # (map() over the methods: half the time of comprehensions, and 90 small tensors are host time before all else)
        kinds = list(map(_dtype, grads))
        if (list(map(_shape, grads)) != self._shapes or not all(map(torch.Tensor.is_contiguous, grads)) or
                list(map(torch.Tensor.get_device, grads)) != self._devices):
            raise ValueError("grads: contiguous tensors of the parameters' shapes and device expected")
        if kinds != self._grad_types:
            if not all(kind in _TYPES for kind in kinds):           # (before any of them is noted)
                raise ValueError("grads: bfloat16, float16 or float32 expected")
            for t, kind in zip(self._list, kinds):
                t.grad_type = _TYPES[kind]
            self._grad_types = kinds
        pointers = array("Q", map(torch.Tensor.data_ptr, grads))
        rc = (_lib or lib()).ozimmu_adamw(len(self._list), self._list, pointers.buffer_info()[0], lr, beta1, beta2, eps, weight_decay, step,
                                          seed & 0xffffffff, _stream(self._devices[0] if self._devices else _get_device(), "AdamW"))
        if rc != OK:
            raise OzimmuError(rc, "adamw")
        increment_version(self._weights)


MOE_TOKENS, MOE_EXPERTS, MOE_TOP_K = 64, 512, 16       # at most


def moe_workspace_bytes(tokens, width, hidden, experts, top_k, dtype):
    return lib().ozimmu_moe_workspace_bytes(*_sizes(tokens, width, hidden, experts, top_k), _TYPES[dtype])


def moe(x, router, w_in, w_out, top_k, normalise=True, out=None, chosen=None, gates=None, workspace=None):
    """A mixture-of-experts layer on at most MOE_TOKENS tokens; returns (y, chosen, gates).

    x [tokens, width], router [experts, width], w_in [experts, 2 * hidden, width] (gate rows, then up rows), w_out [experts,
    width, hidden], the weights contiguous.  Every token takes the top_k experts of its largest logits x @ router.T
    (ties to the lowest index) with the softmax over all experts, or over the chosen ones (normalise), as their gates.
    chosen [tokens, top_k], int32, lists them in ascending order, gates, float32, has theirs."""
    kind = _type_of(x, "x")
    try:
        (tokens, width), (experts, _, hidden) = x.shape, w_out.shape
    except ValueError:
        raise ValueError("x: a matrix, w_out: three dimensions expected") from None
    if (experts | hidden | top_k) >> 30:
        raise ValueError(f"moe: sizes below 2^30 expected, got {experts} experts of {hidden}, {top_k} chosen")
    index = x.get_device()
    for w, shape, what in ((router, (experts, width), "router"), (w_in, (experts, 2 * hidden, width), "w_in"),
                           (w_out, (experts, width, hidden), "w_out")):
        if w.shape != shape or w.dtype is not x.dtype or w.get_device() != index or not w.is_contiguous():
            raise ValueError(f"{what}: contiguous {list(shape)} of {x.dtype} on {x.device} expected")
    ldx = _ld(x, tokens, width, x, "x")
    if out is None:
        out = torch.empty((tokens, width), dtype=x.dtype, device=x.device)
    ldy = _ld(out, tokens, width, x, "out")
    def small(t, dtype, what):
        if t is None:
            return torch.empty((tokens, top_k), dtype=dtype, device=x.device)
        if t.shape != (tokens, top_k) or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"{what}: contiguous [{tokens}, {top_k}] of {dtype} on {x.device} expected")
        return t

    chosen, gates = small(chosen, torch.int32, "chosen"), small(gates, torch.float32, "gates")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, L.ozimmu_moe_workspace_bytes(tokens, width, hidden, experts, top_k, kind)
                                  if workspace is None else 0, x.device)
    rc = L.ozimmu_moe(tokens, width, hidden, experts, top_k, kind, int(normalise), x.data_ptr(), ldx, router.data_ptr(), w_in.data_ptr(),
                      w_out.data_ptr(), chosen.data_ptr(), gates.data_ptr(), out.data_ptr(), ldy, ws, nbytes,
                      _stream(index, "moe"))
    if rc != OK:
        raise OzimmuError(rc, "moe")
    return out, chosen, gates


def _first(x, what):
    """(type, shape, device, row stride) of the matrix that the others of a call go by."""
    kind, shape = _type_of(x, what), x.shape
    if len(shape) != 2:
        raise ValueError(f"{what}: a matrix expected")
    return kind, shape, x.get_device(), _ld(x, shape[0], shape[1], x, what)


def _like(x, shape, dtype, index, what):
    """Row stride of a [rows, cols] device tensor of this type, as _ld; the plain case first (a third of the time)."""
    if x is not None and x.dtype is dtype and x.shape == shape and x.get_device() == index:
        return (shape[1] or 1) if x.is_contiguous() and not (shape[0] | shape[1]) >> 30 else _ld(x, shape[0], shape[1], x, what)
    raise ValueError(f"{what}: {list(shape)} of {dtype} on cuda:{index} expected")


def _line(x, n, dtype, index, what):
    """Address of a contiguous vector."""
    if x is not None and x.dtype is dtype and x.shape == (n,) and x.get_device() == index and x.is_contiguous():
        return x.data_ptr()
    raise ValueError(f"{what}: contiguous [{n}] of {dtype} on cuda:{index} expected")


_int8, _float32 = torch.int8, torch.float32


# (sizes of workspaces follow from the sizes of a call: asked for once, where the library would take 1 us of every call)
@lru_cache(maxsize=4096)
def _norm_grad_bytes(*sizes):
    return lib().ozimmu_rms_norm_grad_workspace_bytes(*sizes)


@lru_cache(maxsize=4096)
def _linear8_bytes(*sizes):
    return lib().ozimmu_linear8_workspace_bytes(*sizes)


@lru_cache(maxsize=4096)
def _linear8_grad_bytes(*sizes):
    return lib().ozimmu_linear8_grad_workspace_bytes(*sizes)


def quantise(x, out=None, scale=None):
    """x [rows, cols] in 8 bits: (codes, scale), int8 [rows, cols] and float32 [rows], that stand for codes * scale[:, None].

    scale is the row's largest magnitude / 127, codes are rounded to nearest; a row with a value that is not finite has
    a scale of NaN.  Asynchronous on the current stream."""
    kind, shape, index, ldx = _first(x, "x")
    rows, cols = shape
    if out is None:
        out = torch.empty(shape, dtype=_int8, device=x.device)
    if scale is None:
        scale = torch.empty(rows, dtype=_float32, device=x.device)
    rc = (_lib or lib()).ozimmu_quantise(rows, cols, kind, x.data_ptr(), ldx, out.data_ptr(), _like(out, shape, _int8, index, "out"),
                                         _line(scale, rows, _float32, index, "scale"), _stream(index, "quantise"))
    if rc != OK:
        raise OzimmuError(rc, "quantise")
    return out, scale


def _norm(x, weight, residual, eps, total, y, codes, scale, what):
    """The norm's call: (tensors that it made or was given)."""
    kind, shape, index, ldx = _first(x, "x")
    (tokens, width), dtype = shape, x.dtype
    pw = None if weight is None else _line(weight, width, dtype, index, "weight")
    ldr = ldt = ldy = ldc = 0
    py = pc = ps = pt = pr = None
    if residual is not None:
        ldr, pr = _like(residual, shape, dtype, index, "residual"), residual.data_ptr()
        if total is None:
            total = torch.empty(shape, dtype=dtype, device=x.device)
    if total is not None:
        ldt, pt = _like(total, shape, dtype, index, "total"), total.data_ptr()
    if what == "rms_norm":
        if y is None:
            y = torch.empty(shape, dtype=dtype, device=x.device)
        ldy, py = _like(y, shape, dtype, index, "out"), y.data_ptr()
    else:
        if codes is None:
            codes = torch.empty(shape, dtype=_int8, device=x.device)
        if scale is None:
            scale = torch.empty(tokens, dtype=_float32, device=x.device)
        ldc, pc, ps = _like(codes, shape, _int8, index, "out"), codes.data_ptr(), _line(scale, tokens, _float32, index, "scale")
    rc = (_lib or lib()).ozimmu_rms_norm(tokens, width, kind, x.data_ptr(), ldx, pr, ldr, pw, eps, pt, ldt, py, ldy, pc, ldc, ps,
                                         _stream(index, what))
    if rc != OK:
        raise OzimmuError(rc, what)
    return y, codes, scale, x if total is None else total


def rms_norm(x, weight=None, residual=None, eps=1e-6, total=None, out=None):
    """Root-mean-square norm of each row of h = x + residual: (y, total), y = h * (mean(h^2) + eps)^-1/2 * weight, total = h.

    x, residual [tokens, width], weight [width] (None: ones).  `total` receives h, rounded (y goes by the unrounded h), and may be
    x or residual itself; without a residual it is x unless a tensor is given.  Asynchronous on the current stream."""
    y, _, _, total = _norm(x, weight, residual, eps, total, out, None, None, "rms_norm")
    return y, total


def rms_norm8(x, weight=None, residual=None, eps=1e-6, total=None, out=None, scale=None):
    """rms_norm with its result in 8 bits, as linear8 takes it: (codes, scale, total)."""
    return _norm(x, weight, residual, eps, total, None, out, scale, "rms_norm8")[1:]


def rms_norm_grad_workspace_bytes(tokens, width):
    return lib().ozimmu_rms_norm_grad_workspace_bytes(*_sizes(tokens, width))


def rms_norm_grad(dy, total, weight=None, eps=1e-6, add=None, dx=None, dw=None, want=("dx", "dw"), workspace=None):
    """Gradients (dx, dw) of rms_norm, or of the values that rms_norm8's results stand for, from dy [tokens, width] and its `total`.

    dx is the gradient of x and of the residual; `add` [tokens, width], the gradient that reaches `total` from elsewhere, is added to
    it, and dx may be dy, total or add itself.  Of dx and dw those in `want` are formed, the others are None."""
    kind, shape, index, lddy = _first(dy, "dy")
    (tokens, width), dtype = shape, dy.dtype
    ldh = _like(total, shape, dtype, index, "total")
    pw = None if weight is None else _line(weight, width, dtype, index, "weight")
    lda = 0 if add is None else _like(add, shape, dtype, index, "add")
    dx = None if "dx" not in want else torch.empty(shape, dtype=dtype, device=dy.device) if dx is None else dx
    dw = None if "dw" not in want else torch.empty(width, dtype=dtype, device=dy.device) if dw is None else dw
    lddx = 0 if dx is None else _like(dx, shape, dtype, index, "dx")
    pdw = None if dw is None else _line(dw, width, dtype, index, "dw")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, _norm_grad_bytes(tokens, width) if workspace is None and dw is not None else 0, dy.device)
    rc = L.ozimmu_rms_norm_grad(tokens, width, kind, dy.data_ptr(), lddy, total.data_ptr(), ldh, pw, eps, None if add is None else add.data_ptr(), lda,
                                None if dx is None else dx.data_ptr(), lddx, pdw, ws, nbytes, _stream(index, "rms_norm_grad"))
    if rc != OK:
        raise OzimmuError(rc, "rms_norm_grad")
    return dx, dw


LINEAR8_IN = 131071          # at most: sums of products of codes are exact in 32 bits


def linear8_workspace_bytes(tokens, n_in, n_out, aligned=True):
    """Bytes of workspace for linear8; aligned: every row of x and w starts on 16 bytes."""
    return lib().ozimmu_linear8_workspace_bytes(*_sizes(tokens, n_in, n_out), int(aligned))


def linear8(x, x_scale, w, w_scale, bias=None, residual=None, activation=ACT_NONE, dtype=None, pre=None, out=None, workspace=None):
    """linear with x [tokens, n_in] and w [n_out, n_in] in 8 bits: act((x * x_scale[:, None]) @ (w * w_scale[:, None]).T + bias) + residual.

    x and w: int8, with float32 scales for their rows, as quantise and rms_norm8 give them.  Everything else is of one type: that of
    `out`, `residual`, `bias` or `pre` where given, else `dtype` (bfloat16 by default)."""
    given = out if out is not None else residual if residual is not None else bias if bias is not None else pre
    if given is None:
        dtype = torch.bfloat16 if dtype is None else dtype
    elif dtype is None:
        dtype = given.dtype
    elif dtype != given.dtype:
        raise ValueError(f"dtype: {given.dtype} or None expected")
    kind, index = _TYPES.get(dtype), x.get_device()
    if kind is None or not x.is_cuda:
        raise ValueError("linear8: CUDA tensors and a result in bfloat16, float16 or float32 expected")
    try:
        (tokens, n_in), (n_out, _) = x.shape, w.shape
    except ValueError:
        raise ValueError("x and w: matrices expected") from None
    if n_in > LINEAR8_IN:
        raise ValueError(f"linear8: at most {LINEAR8_IN} input features expected, got {n_in}")
    ldx, ldw = _like(x, x.shape, _int8, index, "x"), _like(w, (n_out, n_in), _int8, index, "w")
    px, pw = _line(x_scale, tokens, _float32, index, "x_scale"), _line(w_scale, n_out, _float32, index, "w_scale")
    shape = (tokens, n_out)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=x.device)
    ldy = _like(out, shape, dtype, index, "out")
    pbias = None if bias is None else _line(bias, n_out, dtype, index, "bias")
    ldr = 0 if residual is None else _like(residual, shape, dtype, index, "residual")
    ldp = 0 if pre is None else _like(pre, shape, dtype, index, "pre")
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, _linear8_bytes(tokens, n_in, n_out, _aligned(x, ldx, w, ldw)) if workspace is None else 0, x.device)
    rc = L.ozimmu_linear8(tokens, n_in, n_out, kind, x.data_ptr(), ldx, px, w.data_ptr(), ldw, pw, pbias,
                          None if residual is None else residual.data_ptr(), ldr, activation,
                          None if pre is None else pre.data_ptr(), ldp, out.data_ptr(), ldy, ws, nbytes, _stream(index, "linear8"))
    if rc != OK:
        raise OzimmuError(rc, "linear8")
    return out


def linear8_grad_workspace_bytes(tokens, n_in, n_out, dtype, activation=ACT_NONE, aligned=True, x8=True, w8=False):
    """Bytes of workspace for linear8_grad; x8, w8: which of x and w are in 8 bits; aligned: every row of dy, and of x and w that are
    not, starts on 16 bytes."""
    return lib().ozimmu_linear8_grad_workspace_bytes(*_sizes(tokens, n_in, n_out), _TYPES[dtype], activation, int(aligned), int(x8), int(w8))


def linear8_grad(dy, x, w, pre=None, activation=ACT_NONE, x_scale=None, w_scale=None, pre_scale=None, bias=True, dx=None, dw=None, db=None,
                 want=("dx", "dw"), workspace=None):
    """Gradients (dx, dw, db) of linear8, or of linear with operands kept in 8 bits for them, from dy [tokens, n_out].

    x [tokens, n_in], w [n_out, n_in] and pre [tokens, n_out] each are of dy's type, or int8 with a float32 scale for every row,
    as quantise and rms_norm8 give them.  The rest is linear_grad's."""
    kind, index = _type_of(dy, "dy"), dy.get_device()
    try:
        (tokens, n_out), (_, n_in) = dy.shape, x.shape
    except ValueError:
        raise ValueError("dy and x: matrices expected") from None

    dtype = dy.dtype

    def held(t, scale, rows, cols, what):
        """(row stride, scales) of an operand of either kind."""
        if scale is None:
            return _like(t, (rows, cols), dtype, index, what), None
        return _like(t, (rows, cols), _int8, index, what), _line(scale, rows, _float32, index, what + "_scale")

    lddy = _like(dy, (tokens, n_out), dtype, index, "dy")
    ldx, pxs = held(x, x_scale, tokens, n_in, "x")
    ldw, pws = held(w, w_scale, n_out, n_in, "w")
    if activation != ACT_NONE and pre is None:
        raise ValueError("pre: the values before the activation are needed")
    ldp, pps = held(pre, pre_scale, tokens, n_out, "pre") if activation != ACT_NONE else (0, None)

    def result(given, name, shape):
        if name not in want:
            return None
        return torch.empty(shape, dtype=dtype, device=dy.device) if given is None else given

    dx, dw = result(dx, "dx", (tokens, n_in)), result(dw, "dw", (n_out, n_in))
    db = (torch.empty(n_out, dtype=dtype, device=dy.device) if db is None else db) if bias else None
    lddx = 0 if dx is None else _like(dx, (tokens, n_in), dtype, index, "dx")
    lddw = 0 if dw is None else _like(dw, (n_out, n_in), dtype, index, "dw")
    pdb = None if db is None else _line(db, n_out, dtype, index, "db")
    plain = [v for t, ld, scale in ((x, ldx, pxs), (w, ldw, pws)) if scale is None for v in (t, ld)]
    L = _lib or lib()
    keep, ws, nbytes = _workspace(workspace, _linear8_grad_bytes(tokens, n_in, n_out, kind, activation, _aligned(dy, lddy, *plain),
                                                                       pxs is not None, pws is not None) if workspace is None else 0, dy.device)
    rc = L.ozimmu_linear8_grad(tokens, n_in, n_out, kind, dy.data_ptr(), lddy, x.data_ptr(), ldx, pxs, w.data_ptr(), ldw, pws,
                               pre.data_ptr() if activation != ACT_NONE else None, ldp, pps, activation,
                               None if dx is None else dx.data_ptr(), lddx, None if dw is None else dw.data_ptr(), lddw, pdb,
                               ws, nbytes, _stream(index, "linear8_grad"))
    if rc != OK:
        raise OzimmuError(rc, "linear8_grad")
    return dx, dw, db
