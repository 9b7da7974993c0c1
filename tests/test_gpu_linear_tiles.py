"""ozimmu_linear and ozimmu_linear_grad in their larger tiles: each tile and order of operands, its edges, parts and epilogues."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers, ozimmu
from tests.layers_reference import ROUND, TYPES, U32, guarded, product_bound, rounded, slope, sum_bound, untouched, within
from tests.test_gpu_linear import ACTS, check_linear, operands


def tile(which, shape, kind, aligned=1):
    """(edge, whether the contraction is divided) for operands on 16 bytes, or off them and not copied."""
    parts = ctypes.c_int()
    edge = ozimmu.lib().ozimmu_debug_linear_tile(which, *shape, {"bf16": 0, "f16": 1, "f32": 2}[kind], aligned, ctypes.byref(parts))
    return edge, parts.value > 1


# (kinds, shape, tile, divided): whole tiles and tiles that end anywhere, contractions that end within a step and are shorter than the ring
LINEAR = [("16", (3000, 72, 4096), 256, False), ("16", (4096, 328, 4096), 256, False), ("16", (3000, 1000, 4099), 256, False),
          ("16", (4097, 2056, 2300), 256, False), ("16", (777, 8192, 2560), 256, True), ("16", (2561, 8192, 779), 256, True),
          ("16", (1777, 64, 1777), 128, False), ("16", (1790, 200, 1784), 128, False), ("16", (1280, 1000, 1921), 128, False),
          ("16", (300, 8192, 777), 128, True), ("16", (777, 8192, 304), 128, True), ("f32", (1777, 776, 1777), 128, False),
          ("f32", (1921, 2048, 1800), 128, False), ("f32", (1800, 1032, 4099), 128, False)]


def kinds(cases):
    return [(kind, *case[1:]) for case in cases for kind in (("bf16", "f16") if case[0] == "16" else ("f32",))]


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("kind,shape,edge,divided", kinds(LINEAR))
def test_linear_in_the_larger_tiles(kind, shape, edge, divided, extra):
    tokens, n_in, n_out = shape
    assert tile(0, shape, kind) == (edge, divided)
    x, w, bias, residual, _ = operands(tokens, n_in, n_out, kind, extra, 400 + n_in)
    name = ACTS[(tokens + n_out + extra) % 5]
    (y, ybuf), (pre, pbuf) = (guarded(tokens, n_out, n_out + extra, x.dtype) for _ in range(2))
    print(kind, shape, extra, name, flush=True)
    layers.linear(x, w, bias, residual, layers.ACTIVATIONS[name], pre=pre, out=y)
    torch.cuda.synchronize()
    check_linear(x, w, bias, residual, name, y, pre)
    assert untouched(y, ybuf) and untouched(pre, pbuf)
    check_linear(x, w, None, None, name, layers.linear(x, w, activation=layers.ACTIVATIONS[name]), None)
    stream = residual.clone(memory_format=torch.preserve_format)
    layers.linear(x, w, bias, stream, layers.ACTIVATIONS[name], out=stream)          # added to in place
    assert torch.equal(stream, y)


# (kinds, shape, tile of dx and whether it is divided, of dw, of both in one launch or 0; None: not what the case is for)
GRAD = [("16", (3000, 4096, 264), (256, False), None, None), ("16", (264, 4096, 3000), None, (256, False), None),
        ("16", (4096, 1400, 4096), (256, True), (256, True), None), ("16", (3001, 4096, 3003), (256, False), (256, False), 0),
        ("16", (4096, 776, 300), (128, False), None, None), ("16", (300, 776, 4096), None, (128, False), None),
        ("16", (1280, 776, 4096), (128, True), (128, False), None), ("16", (4096, 776, 1280), (128, False), (128, True), None),
        ("16", (500, 8192, 384), None, None, 128), ("16", (640, 4096, 640), None, None, 128), ("16", (1777, 1024, 2304), None, None, 128),
        ("f32", (4096, 776, 640), (128, False), None, None), ("f32", (640, 776, 4096), None, (128, False), None),
        ("f32", (1777, 2048, 777), (128, False), None, None), ("f32", (1536, 183121, 1629), None, None, 128)]


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("kind,shape,of_dx,of_dw,of_both", kinds(GRAD))
def test_gradients_in_the_larger_tiles(kind, shape, of_dx, of_dw, of_both, extra):
    tokens, n_in, n_out = shape
    assert of_dx is None or tile(1, shape, kind) == of_dx
    assert of_dw is None or tile(2, shape, kind) == of_dw
    assert of_both is None or tile(3, shape, kind)[0] == of_both
    x, w, _, dy, z = operands(tokens, n_in, n_out, kind, extra, 500 + n_in)
    name = ACTS[(tokens + n_in + extra) % 5]
    dtype, u = x.dtype, ROUND[x.dtype]
    out = [guarded(tokens, n_in, n_in + extra, dtype), guarded(n_out, n_in, n_in + extra, dtype)]
    print(kind, shape, extra, name, flush=True)
    dx, dw, db = layers.linear_grad(dy, x, w, None if name == "none" else z, layers.ACTIVATIONS[name], dx=out[0][0], dw=out[1][0])
    torch.cuda.synchronize()
    G, Z = dy.double(), z.double()
    dz = G * slope(name, Z)
    # the slope in 32 bits, then one rounding of dz for the products
    sb = 0 * G if name in ("none", "relu") else 32 * U32 * G.abs() * (1 + Z.abs()) ** 2
    zb = sb + (0 if name == "none" else rounded(dz, dtype))
    X, W = x.double(), w.double()
    for got, P, Q, PB, what in ((dx, dz, W.t(), zb, "dx"), (dw, dz.t(), X.t(), zb.t(), "dw")):
        want = torch.matmul(P, Q.t())
        bound = product_bound(P, Q, 2 * U32) + torch.matmul(PB, Q.abs().t())
        within(got, want, bound + rounded(want, dtype) + u * bound, what)
    want, bound = dz.sum(0), dz.abs().sum(0) * sum_bound(tokens) + sb.sum(0)
    within(db, want, bound + rounded(want, dtype) + u * bound, "db")
    assert untouched(dx, out[0][1]) and untouched(dw, out[1][1])
    # each alone, in tiles of its own and parts of the contraction
    for what, at, P, Q, PB in (("dx", 0, dz, W.t(), zb), ("dw", 1, dz.t(), X.t(), zb.t())):
        got = layers.linear_grad(dy, x, w, None if name == "none" else z, layers.ACTIVATIONS[name], want=(what,), bias=False)[at]
        want = torch.matmul(P, Q.t())
        bound = product_bound(P, Q, 2 * U32) + torch.matmul(PB, Q.abs().t())
        within(got, want, bound + rounded(want, dtype) + u * bound, what + " alone")


@pytest.mark.parametrize("kind,shape,edges", [("bf16", (4096, 1000, 2056), (128, 128)), ("f16", (4097, 1000, 2064), (128, 64)), ("f16", (1000, 520, 2056), (128, 64)),
                                              ("f32", (4096, 1000, 2056), (64, 128)), ("f32", (1800, 1032, 4096), (128, 64)), ("f32", (1001, 136, 2064), (64, 64))])
def test_operands_that_are_not_aligned_without_room_for_copies(kind, shape, edges):
    tokens, n_in, n_out = shape
    assert tuple(tile(which, shape, kind, aligned=0)[0] for which in (0, 1)) == edges
    x, w, bias, residual, dy = operands(tokens, n_in, n_out, kind, 3, 600)
    room = layers.linear_workspace_bytes(*shape, x.dtype, True)
    print(kind, shape, flush=True)
    y = layers.linear(x, w, bias, residual, layers.ACT_SILU, workspace=torch.empty(room + 256, dtype=torch.uint8, device="cuda"))
    check_linear(x, w, bias, residual, "silu", y, None)
    room = layers.linear_grad_workspace_bytes(*shape, x.dtype, layers.ACT_NONE, True)
    dx, dw, db = layers.linear_grad(dy, x, w, workspace=torch.empty(room + 256, dtype=torch.uint8, device="cuda"))
    G, X, W, u = dy.double(), x.double(), w.double(), ROUND[x.dtype]
    for got, P, Q, what in ((dx, G, W.t(), "dx"), (dw, G.t(), X.t(), "dw")):
        want, bound = torch.matmul(P, Q.t()), product_bound(P, Q, 2 * U32)
        within(got, want, bound + rounded(want, x.dtype) + u * bound, what)
    want, bound = G.sum(0), G.abs().sum(0) * sum_bound(tokens)
    within(db, want, bound + rounded(want, x.dtype) + u * bound, "db")
