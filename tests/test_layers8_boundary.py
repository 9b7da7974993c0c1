"""CPU-side checks of the operators on rows in 8 bits: refused arguments, sizes of workspaces, what the binding refuses."""
import ctypes
import itertools
import os

import pytest

torch = pytest.importorskip("torch")

BAD, OK = 1, 0
F = ctypes.c_void_p(1 << 20)           # never read: every call below is refused, or has nothing to do, before a kernel starts
ODD = ctypes.c_void_p((1 << 20) + 1)
MOST = (1 << 30) - 1


@pytest.fixture(scope="module")
def handle():
    from paper_2506_11277_amd import build, layers, ozimmu
    if not os.path.exists(ozimmu.LIB_PATH):
        build.build_lib()
    return layers.lib()


def norm(h, tokens=4, width=8, type=0, x=F, ldx=8, residual=None, ldr=8, weight=F, eps=1e-6, total=None, ldt=8, y=F, ldy=8, codes=None, ldc=8, scale=None):
    return h.ozimmu_rms_norm(tokens, width, type, x, ldx, residual, ldr, weight, eps, total, ldt, y, ldy, codes, ldc, scale, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(width=-1), dict(tokens=1 << 30), dict(width=1 << 30, ldx=1 << 30, ldy=1 << 30), dict(type=3), dict(type=-1),
                                   dict(x=None), dict(x=ODD), dict(ldx=7), dict(residual=F, ldr=7), dict(residual=ODD), dict(weight=ODD), dict(eps=0.0),
                                   dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-60), dict(eps=1e60), dict(total=F, ldt=7), dict(total=ODD), dict(y=ODD), dict(ldy=7),
                                   dict(codes=F, scale=None), dict(codes=F, scale=F, ldc=7), dict(codes=F, scale=ODD), dict(codes=None, scale=F),
                                   dict(type=2, x=ctypes.c_void_p((1 << 20) + 2))])
def test_norm_refuses(handle, wrong):
    assert norm(handle, **wrong) == BAD


def test_norm_of_nothing(handle):
    assert norm(handle, tokens=0, x=None, y=None) == OK and norm(handle, y=None) == OK


def quantise(h, rows=4, cols=8, type=0, x=F, ldx=8, codes=F, ldc=8, scale=F):
    return h.ozimmu_quantise(rows, cols, type, x, ldx, codes, ldc, scale, None)


@pytest.mark.parametrize("wrong", [dict(rows=-1), dict(cols=-1), dict(rows=1 << 30), dict(cols=1 << 30, ldx=1 << 30, ldc=1 << 30), dict(type=4), dict(type=-1), dict(x=None),
                                   dict(x=ODD), dict(ldx=7), dict(codes=None), dict(ldc=7), dict(scale=None), dict(scale=ODD)])
def test_quantise_refuses(handle, wrong):
    assert quantise(handle, **wrong) == BAD


def norm_grad(h, tokens=4, width=8, type=0, dy=F, lddy=8, x=F, ldh=8, weight=F, eps=1e-6, add=None, ldadd=8, dx=F, lddx=8, dw=F, ws=F, nbytes=1 << 40):
    return h.ozimmu_rms_norm_grad(tokens, width, type, dy, lddy, x, ldh, weight, eps, add, ldadd, dx, lddx, dw, ws, nbytes, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(width=-1), dict(tokens=1 << 30), dict(width=1 << 30, lddy=1 << 30, ldh=1 << 30, lddx=1 << 30), dict(type=3), dict(dy=None),
                                   dict(dy=ODD), dict(lddy=7), dict(x=None), dict(x=ODD), dict(ldh=7), dict(weight=ODD), dict(eps=0.0), dict(eps=float("nan")),
                                   dict(add=F, ldadd=7), dict(add=ODD), dict(dx=ODD), dict(lddx=7), dict(dw=ODD), dict(ws=None), dict(nbytes=0),
                                   dict(ws=ctypes.c_void_p((1 << 20) + 128))])
def test_norm_grad_refuses(handle, wrong):
    assert norm_grad(handle, **wrong) == BAD


def test_norm_grad_workspace(handle):
    need = handle.ozimmu_rms_norm_grad_workspace_bytes
    assert need(-1, 8) == 0 and need(8, 1 << 30) == 0 and need(0, 8) == 0 and need(8, 0) == 0
    for tokens in (1, 5, 1000, 1 << 20, MOST):
        for width in (1, 1001, 4096, 16384, 16385, 1 << 20):
            # 512 parts, or one of every 1024 rows; and two numbers a row
            assert 4 * width <= need(tokens, width) <= 4 * width * max(512, tokens // 1024 + 1) + 8 * tokens + 1024
            assert norm_grad(handle, tokens, width, lddy=width, ldh=width, lddx=width, nbytes=need(tokens, width) - 1) == BAD
    assert norm_grad(handle, width=0) == OK and norm_grad(handle, dx=None, dw=None, ws=None, nbytes=0) == OK


def bf16(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_the_binding_refuses(monkeypatch):
    from paper_2506_11277_amd import layers
    with pytest.raises(ValueError):
        layers.quantise(bf16(2, 8))                       # not a CUDA tensor
    monkeypatch.setattr(layers, "_type_of", lambda x, what: layers._TYPES[x.dtype])
    monkeypatch.setattr(layers, "_stream", lambda index, what: None)
    x, w, f32 = bf16(2, 8), bf16(8), torch.float32
    for call in (lambda: layers.quantise(bf16(8)), lambda: layers.quantise(x, out=bf16(2, 8)), lambda: layers.quantise(x, out=bf16(2, 7, dtype=torch.int8)),
                 lambda: layers.quantise(x, scale=bf16(2)), lambda: layers.quantise(x, scale=bf16(3, dtype=f32)), lambda: layers.quantise(bf16(8, 2).t()),
                 lambda: layers.quantise(x, scale=bf16(4, dtype=f32)[::2]),
                 lambda: layers.rms_norm(x, bf16(7)), lambda: layers.rms_norm(x, bf16(8, dtype=f32)), lambda: layers.rms_norm(x, w, bf16(3, 8)),
                 lambda: layers.rms_norm(x, w, bf16(2, 8, dtype=f32)), lambda: layers.rms_norm(x, w, out=bf16(2, 7)), lambda: layers.rms_norm(bf16(1, 2, 8), w),
                 lambda: layers.rms_norm(x, w, x, total=bf16(2, 7)), lambda: layers.rms_norm8(x, w, out=x), lambda: layers.rms_norm8(x, w, scale=bf16(2)),
                 lambda: layers.rms_norm_grad(x, bf16(3, 8), w), lambda: layers.rms_norm_grad(x, x, bf16(9)), lambda: layers.rms_norm_grad(x, x, w, add=bf16(2, 9)),
                 lambda: layers.rms_norm_grad(x, x, w, dx=bf16(2, 8, dtype=f32)), lambda: layers.rms_norm_grad(x, x, w, dw=bf16(7)),
                 lambda: layers.rms_norm_grad_workspace_bytes(1 << 32, 8)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(layers.OzimmuError):
        layers.rms_norm(x, w, eps=0.0)


def linear8(h, tokens=4, n_in=8, n_out=8, type=0, x=F, ldx=8, xs=F, w=F, ldw=8, ws=F, bias=None, residual=None, ldr=8, act=0, pre=None, ldpre=8, y=F, ldy=8,
            room=None, nbytes=0):
    return h.ozimmu_linear8(tokens, n_in, n_out, type, x, ldx, xs, w, ldw, ws, bias, residual, ldr, act, pre, ldpre, y, ldy, room, nbytes, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(n_in=-1), dict(n_out=-1), dict(tokens=1 << 30), dict(n_in=131072, ldx=1 << 20, ldw=1 << 20), dict(type=3), dict(type=8),
                                   dict(act=5), dict(act=-1), dict(x=None), dict(w=None), dict(y=None), dict(xs=None), dict(ws=None), dict(xs=ODD), dict(ws=ODD), dict(ldx=7), dict(ldw=7),
                                   dict(ldy=7), dict(y=ODD), dict(bias=ODD), dict(residual=F, ldr=7), dict(residual=ODD), dict(pre=F, ldpre=7), dict(pre=ODD)])
def test_linear8_refuses(handle, wrong):
    assert linear8(handle, **wrong) == BAD


def test_linear8_workspace(handle):
    need = handle.ozimmu_linear8_workspace_bytes
    assert need(-1, 1, 1, 1) == 0 and need(1, 131072, 1, 1) == 0 and need(0, 0, 0, 1) == 0 and need(1 << 30, 1, 1, 1) == 0
    sizes = [(t, i, o) for t in (1, 64, 65, 300, 1531, 8192) for i in (1, 1001, 8192, 65536) for o in (1, 777, 2048, 8192)]
    some = [s for s in sizes if need(*s, 1) > 0 and s[1] % 16 == 0]
    assert some
    t, i, o = some[0]
    assert linear8(handle, t, i, o, ldx=i, ldw=i, ldy=o) == BAD
    assert linear8(handle, t, i, o, ldx=i, ldw=i, ldy=o, room=F, nbytes=need(t, i, o, 1) - 1) == BAD
    assert linear8(handle, t, i, o, ldx=i, ldw=i, ldy=o, room=ctypes.c_void_p((1 << 20) + 128), nbytes=1 << 40) == BAD
    assert need(4096, 4096, 4096, 0) >= need(4096, 4096, 4096, 1) + 2 * 4096 * 4096        # room for copies of x and w
    assert linear8(handle, tokens=0, x=None, xs=None, y=None) == OK and linear8(handle, n_out=0, w=None, ws=None, y=None) == OK


def test_the_binding_refuses_operands_of_linear8(monkeypatch):
    from paper_2506_11277_amd import layers
    x, s = bf16(4, 8, dtype=torch.int8), bf16(4, dtype=torch.float32)
    with pytest.raises(ValueError):
        layers.linear8(x, s, x, s)                         # not CUDA tensors
    with pytest.raises(ValueError):
        layers.linear8_workspace_bytes(1 << 32, 8, 8)
    for dtype in (torch.float64, torch.int8):
        with pytest.raises(ValueError):
            layers.linear8(x, s, x, s, dtype=dtype)


def linear8_grad(h, tokens=4, n_in=8, n_out=8, type=0, dy=F, lddy=8, x=F, ldx=8, xs=F, w=F, ldw=8, ws=None, pre=F, ldpre=8, ps=F, act=2, dx=F, lddx=8, dw=F, lddw=8,
                 db=F, room=F, nbytes=1 << 40):
    return h.ozimmu_linear8_grad(tokens, n_in, n_out, type, dy, lddy, x, ldx, xs, w, ldw, ws, pre, ldpre, ps, act, dx, lddx, dw, lddw, db, room, nbytes, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(n_in=-1), dict(n_out=1 << 30), dict(type=3), dict(type=8), dict(act=5), dict(dy=None), dict(dy=ODD), dict(lddy=7), dict(x=None),
                                   dict(x=ODD, xs=None), dict(ldx=7), dict(xs=ODD), dict(w=None), dict(w=ODD), dict(ldw=7), dict(ws=ODD), dict(pre=None), dict(pre=ODD, ps=None), dict(ldpre=7),
                                   dict(ps=ODD), dict(dx=ODD), dict(lddx=7), dict(dw=ODD), dict(lddw=7), dict(db=ODD), dict(room=None), dict(nbytes=0),
                                   dict(room=ctypes.c_void_p((1 << 20) + 128))])
def test_linear8_grad_refuses(handle, wrong):
    assert linear8_grad(handle, **wrong) == BAD


def test_linear8_grad_workspace(handle):
    need, plain = handle.ozimmu_linear8_grad_workspace_bytes, handle.ozimmu_linear_grad_workspace_bytes
    assert need(-1, 1, 1, 0, 0, 1, 1, 1) == 0 and need(1, 1, 1, 9, 0, 1, 1, 1) == 0 and need(1, 1, 1, 0, 7, 1, 1, 1) == 0
    for tokens, n_in, n_out in itertools.product((1, 65, 1531), (8, 1001, 4096), (8, 777, 2048)):
        for kind, size in ((0, 2), (1, 2), (2, 4)):
            for act, aligned in itertools.product((0, 2), (0, 1)):
                base = plain(tokens, n_in, n_out, kind, act, aligned)
                assert need(tokens, n_in, n_out, kind, act, aligned, 0, 0) == base
                both = need(tokens, n_in, n_out, kind, act, aligned, 1, 1)
                assert both >= base and both >= size * n_in * (tokens + n_out)
                assert base <= need(tokens, n_in, n_out, kind, act, aligned, 1, 0) <= both
                given = dict(tokens=tokens, n_in=n_in, n_out=n_out, type=kind, act=act, lddy=n_out, ldx=n_in, ldw=n_in, ldpre=n_out, lddx=n_in, lddw=n_in, ws=F)
                assert linear8_grad(handle, **given, nbytes=need(tokens, n_in, n_out, kind, act, 1, 1, 1) - 1) == BAD


def test_the_binding_refuses_operands_of_linear8_grad(monkeypatch):
    from paper_2506_11277_amd import layers
    monkeypatch.setattr(layers, "_type_of", lambda x, what: layers._TYPES[x.dtype])
    monkeypatch.setattr(layers, "_stream", lambda index, what: None)
    dy, w, x = bf16(4, 6), bf16(6, 8), bf16(4, 8)
    x8, s, p8 = bf16(4, 8, dtype=torch.int8), bf16(4, dtype=torch.float32), bf16(4, 6, dtype=torch.int8)
    for call in (lambda: layers.linear8_grad(dy, x8, w), lambda: layers.linear8_grad(dy, x, w, x_scale=s), lambda: layers.linear8_grad(dy, x8, w, x_scale=s[:3]),
                 lambda: layers.linear8_grad(dy, x8, w, x_scale=s.double()), lambda: layers.linear8_grad(dy, x8, w, w_scale=s, x_scale=s),
                 lambda: layers.linear8_grad(dy, x8, w, None, layers.ACT_GELU, x_scale=s), lambda: layers.linear8_grad(dy, x8, w, p8, layers.ACT_GELU, x_scale=s),
                 lambda: layers.linear8_grad(dy, x8, w, dy, layers.ACT_GELU, x_scale=s, pre_scale=s), lambda: layers.linear8_grad(dy, x8, w, p8[:, :5], layers.ACT_GELU, x_scale=s, pre_scale=s),
                 lambda: layers.linear8_grad(dy, x8, w[:, :7], x_scale=s), lambda: layers.linear8_grad(dy, x8, w, x_scale=s, dx=bf16(4, 7)),
                 lambda: layers.linear8_grad_workspace_bytes(8, 1 << 32, 8, torch.bfloat16)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows,cols,ld", [(2, 8, (1 << 32) + 8), (2, 8, 1 << 31), (2, (1 << 32) + 8, (1 << 32) + 8), ((1 << 32) + 2, 8, 8), (1, 1 << 30, 1 << 30), (1 << 30, 1, 1)])
def test_sizes_that_an_int_cannot_hold_are_refused(rows, cols, ld):
    from paper_2506_11277_amd import layers
    x = torch.empty_strided((rows, cols), (ld, 1), dtype=torch.int8, device="meta")
    with pytest.raises(ValueError):
        layers._like(x, x.shape, torch.int8, x.get_device(), "x")


def test_sizes_up_to_the_largest_are_taken():
    from paper_2506_11277_amd import layers
    for rows, cols, ld in ((2, MOST, (1 << 31) - 1), (MOST, 1, 1), (0, MOST, MOST), (1, 8, 1 << 40), (5, 7, 7), (5, 7, 9)):
        x = torch.empty_strided((rows, cols), (ld, 1), dtype=torch.int8, device="meta")
        assert layers._like(x, x.shape, torch.int8, x.get_device(), "x") == (ld if rows > 1 else cols)


def test_tiles_of_both_gradients(handle):
    # 32 bits: 32 x 64 where tiles of 64 would leave half of the compute units without one
    tile = handle.ozimmu_debug_linear_tile
    assert [tile(3, *shape, 2, 1, None) for shape in ((500, 512, 384), (1000, 512, 384), (512, 512, 512), (512, 576, 512), (1536, 183121, 1629))] == [32, 64, 32, 64, 128]
    assert tile(3, 500, 512, 384, 0, 1, None) == 64


def test_what_is_not_given_is_refused():
    from paper_2506_11277_amd import layers
    with pytest.raises(ValueError):
        layers._line(None, 4, torch.float32, 0, "x_scale")
    with pytest.raises(ValueError):
        layers._like(None, (4, 8), torch.int8, 0, "w")
