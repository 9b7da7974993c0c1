"""Plain 64-bit forms of the feed-forward operators, and the error bounds their tests use."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}    # unit roundoff
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half the least subnormal
U32 = 2.0 ** -24


def act(name, z):
    if name == "relu":
        return torch.clamp_min(z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "none":
        return torch.ones_like(z)
    with torch.enable_grad():
        z = z.detach().requires_grad_(True)
        return torch.autograd.grad(act(name, z).sum(), z)[0]


def sum_bound(terms):
    """Error of a sum of `terms` products in 32 bits, relative to the sum of their magnitudes (any order)."""
    return (terms + 8) * U32


def product_bound(x, w, extra=0.0):
    """Error of x @ w.T with operands off by `extra` (relative), against the magnitudes' product."""
    k = x.shape[1]
    return torch.matmul(x.abs(), w.abs().t()) * (sum_bound(k) + extra)


def rounded(y, dtype):
    """Error of rounding to `dtype` once."""
    return ROUND[dtype] * y.abs() + LEAST[dtype]


def guarded(rows, cols, ld, dtype, values=None):
    """A [rows, cols] view of a NaN-filled buffer with row stride ld, rows in front and behind; and the buffer."""
    buf = torch.full(((rows + 2) * ld + 8,), float("nan"), dtype=dtype, device="cuda")
    view = buf[ld:ld + rows * ld].view(rows, ld)[:, :cols] if rows else buf[ld:ld].view(0, ld)[:, :cols]
    if values is not None:
        view.copy_(values)
    return view, buf


def untouched(view, buf):
    """Whether everything of a guarded buffer outside its view still is NaN."""
    rows, cols = view.shape
    ld = (buf.numel() - 8) // (rows + 2)
    outside = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    if rows:
        outside[ld:ld + rows * ld].view(rows, ld)[:, :cols] = False
    return bool(torch.isnan(buf[outside].float()).all())


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float(off[bad].max()), float((off / bound.clamp_min(1e-300))[bad].max()))
