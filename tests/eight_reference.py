"""Plain forms of the layers' operators on rows in 8 bits: the codes in 32 bits, operation by operation, the rest in 64."""
import torch

from tests.layers_reference import U32

MOST = 127.0
NAN = float("nan")


def codes_of(t):
    """(codes, scales) of the rows of t, float32 values, as the header defines them."""
    t = t.cpu()
    assert t.dtype is torch.float32
    if t.shape[1] == 0:
        return torch.zeros(t.shape, dtype=torch.int8), torch.zeros(t.shape[0])
    top = t.abs().amax(1)                                    # (a NaN is the largest)
    held = torch.isfinite(top) & (top >= 2.0 ** -100)
    inverse = torch.where(held, torch.div(torch.full_like(top, MOST), torch.where(held, top, 1.0)), 0.0)   # (MOST / top would be MOST * (1 / top))
    codes = torch.where(held[:, None], torch.round(t * inverse[:, None]), 0.0).to(torch.int8)
    scale = torch.where(held, top.double() / MOST, 0.0)
    return codes, torch.where(torch.isfinite(top), scale, NAN)


def guarded_codes(rows, cols, ld, values=None):
    """A [rows, cols] int8 view of a buffer of 99s with row stride ld, rows in front and behind; and the buffer."""
    buf = torch.full(((rows + 2) * ld + 8,), 99, dtype=torch.int8, device="cuda")
    view = buf[ld:ld + rows * ld].view(rows, ld)[:, :cols] if rows else buf[ld:ld].view(0, ld)[:, :cols]
    if values is not None:
        view.copy_(values)
    return view, buf


def codes_untouched(view, buf):
    rows, cols = view.shape
    ld = (buf.numel() - 8) // (rows + 2)
    outside = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    if rows:
        outside[ld:ld + rows * ld].view(rows, ld)[:, :cols] = False
    return bool((buf[outside] == 99).all())


def depth(width):
    """Additions that a value of a row passes on its way into the row's sum: at most 64 of a thread (of a longer row less than width /
    1024, and a group of 8), 6 among lanes, 16 among wavefronts."""
    return max(64, width // 1024 + 8) + 22


def root_error(width):
    """Relative error of 1 / sqrt(mean of h^2 + eps): half that of the sum, whose h are rounded (2 in the square), of the quotient
    and of the addition of eps; the root and the reciprocal (the library's, two units each)."""
    return ((depth(width) + 2 + 2) / 2 + 4) * U32


def norm(h, weight, eps):
    """(r, y) in 64 bits."""
    h = h.double()
    r = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    return r, h * r * (1.0 if weight is None else weight.double())
