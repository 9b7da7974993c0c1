"""CPU-side checks of the feed-forward operators' boundary: declared symbols, sizes of workspaces, refused arguments."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ozimmu_layers.h")
BAD = 1


@pytest.fixture(scope="module")
def handle():
    from paper_2506_11277_amd import build, layers, ozimmu
    if not os.path.exists(ozimmu.LIB_PATH):
        build.build_lib()
    return layers.lib()


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(ozimmu_\w+)\s*\(", text)))


def test_binding_and_library_cover_every_declared_symbol(handle):
    from paper_2506_11277_amd import layers
    assert sorted(layers._SIGNATURES) == declared()
    raw = ctypes.CDLL(handle._name)
    for name in declared():
        assert hasattr(raw, name), name


def test_constants_match_the_header():
    from paper_2506_11277_amd import layers
    defines = dict(re.findall(r"#define OZIMMU_(\w+) (\d+)", open(HEADER).read()))
    for name in ("BF16", "F16", "F32", "E4M3", "ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_GELU_TANH", "ACT_SILU", "MOE_TOKENS",
                 "MOE_EXPERTS", "MOE_TOP_K"):
        assert getattr(layers, name) == int(defines[name]), name


F = ctypes.c_void_p(1 << 20)           # never read: every call below is refused before a kernel starts
ODD = ctypes.c_void_p((1 << 20) + 1)


def linear(h, tokens=4, n_in=8, n_out=8, type=0, x=F, ldx=8, w=F, ldw=8, bias=None, residual=None, ldr=8, act=0, pre=None, ldpre=8, y=F,
           ldy=8, ws=None, nbytes=0):
    return h.ozimmu_linear(tokens, n_in, n_out, type, x, ldx, w, ldw, bias, residual, ldr, act, pre, ldpre, y, ldy, ws, nbytes, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(n_in=-1), dict(n_out=-1), dict(tokens=1 << 30), dict(n_in=1 << 30, ldx=1 << 30, ldw=1 << 30), dict(type=3), dict(type=-1), dict(act=5), dict(act=-1),
                                   dict(x=None), dict(w=None), dict(y=None), dict(ldx=7), dict(ldw=7), dict(ldy=7), dict(x=ODD), dict(w=ODD),
                                   dict(y=ODD), dict(bias=ODD), dict(residual=F, ldr=7), dict(residual=ODD), dict(pre=F, ldpre=7), dict(pre=ODD),
                                   dict(type=2, x=ctypes.c_void_p((1 << 20) + 2))])
def test_linear_refuses(handle, wrong):
    assert linear(handle, **wrong) == BAD


def test_linear_workspace(handle):
    need = handle.ozimmu_linear_workspace_bytes
    assert need(-1, 1, 1, 0, 1) == 0 and need(1, 1, 1, 9, 1) == 0 and need(0, 0, 0, 0, 1) == 0 and need(1 << 30, 1, 1, 0, 1) == 0
    sizes = [(t, i, o) for t in (1, 64, 65, 300, 1531, 8192) for i in (1, 1001, 8192) for o in (1, 777, 2048, 8192)]
    some = [s for s in sizes if need(*s, 0, 1) > 0 and s[1] % 8 == 0]
    assert some
    t, i, o = some[0]
    assert linear(handle, t, i, o, ldx=i, ldw=i, ldy=o, ws=None) == BAD
    assert linear(handle, t, i, o, ldx=i, ldw=i, ldy=o, ws=F, nbytes=need(t, i, o, 0, 1) - 1) == BAD
    assert linear(handle, t, i, o, ldx=i, ldw=i, ldy=o, ws=ctypes.c_void_p((1 << 20) + 128), nbytes=1 << 40) == BAD
    for s in sizes:
        aligned, other = need(*s, 0, 1), need(*s, 0, 0)
        copies = 2 * (s[0] + s[2]) * (s[1] + 7) + 1024
        assert other >= aligned and aligned <= 16 * 4 * s[0] * (s[2] + 7) + 512 + copies and other <= aligned + copies
    assert need(4096, 4096, 4096, 0, 0) >= need(4096, 4096, 4096, 0, 1) + 2 * 2 * 4096 * 4096       # room for copies of x and w
    assert need(1, 4096, 4096, 0, 0) == need(1, 4096, 4096, 0, 1)                                   # which few tokens do not want


def grad(h, tokens=4, n_in=8, n_out=8, type=0, dy=F, lddy=8, x=F, ldx=8, w=F, ldw=8, pre=F, ldpre=8, act=2, dx=F, lddx=8, dw=F, lddw=8,
         db=F, ws=F, nbytes=1 << 40):
    return h.ozimmu_linear_grad(tokens, n_in, n_out, type, dy, lddy, x, ldx, w, ldw, pre, ldpre, act, dx, lddx, dw, lddw, db, ws, nbytes,
                                None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(n_in=-1), dict(n_out=-1), dict(type=7), dict(act=9), dict(dy=None), dict(lddy=7),
                                   dict(pre=None), dict(ldpre=7), dict(x=None), dict(ldx=7), dict(w=None), dict(ldw=7), dict(lddx=7),
                                   dict(lddw=7), dict(db=ODD), dict(dx=ODD), dict(dw=ODD), dict(dy=ODD), dict(ws=None), dict(nbytes=16)])
def test_linear_grad_refuses(handle, wrong):
    assert grad(handle, **wrong) == BAD


def test_linear_grad_workspace(handle):
    need = handle.ozimmu_linear_grad_workspace_bytes
    assert need(-1, 1, 1, 0, 0, 1) == 0 and need(1, 1, 1, 0, 5, 1) == 0 and need(1, 1, 1, 3, 0, 1) == 0
    assert need(1000, 512, 704, 0, 2, 1) >= need(1000, 512, 704, 0, 0, 1) + 1000 * 704 * 2       # dz
    assert need(1000, 512, 700, 2, 2, 1) >= 1000 * 704 * 4
    assert need(1000, 512, 704, 0, 2, 0) >= need(1000, 512, 704, 0, 2, 1) + (1000 + 704) * 512 * 2  # copies of x and w


def test_adamw_refuses(handle):
    from paper_2506_11277_amd import layers

    def one(**changed):
        t = layers._AdamWTensor(1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, None, 5, 2, 2, 2, 0)
        for name, value in changed.items():
            setattr(t, name, value)
        return (layers._AdamWTensor * 1)(t)

    def call(list, n=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, decay=0.0, step=1):
        return handle.ozimmu_adamw(n, list, None, lr, b1, b2, eps, decay, step, 0, None)

    for wrong in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(count=-1), dict(param_type=3), dict(grad_type=3),
                  dict(state_type=0), dict(state_type=3, m_scale=None), dict(state_type=3, v_scale=None), dict(copy=1 << 20, copy_type=2),
                  dict(param=(1 << 20) + 2), dict(grad=(1 << 20) + 2), dict(m=(1 << 20) + 2), dict(copy=(1 << 20) + 1),
                  dict(state_type=3, m_scale=(1 << 20) + 2)):
        assert call(one(**wrong)) == BAD, wrong
    nan = float("nan")
    for wrong in (dict(n=-1), dict(step=0), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0), dict(b2=nan), dict(eps=-1.0), dict(eps=nan),
                  dict(lr=nan), dict(decay=nan)):
        assert call(one(), **wrong) == BAD, wrong
    assert handle.ozimmu_adamw(1, None, None, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, None) == BAD
    assert call(one(count=0, param=None)) == 0 and call(one(), n=0) == 0


def moe(h, tokens=4, width=8, hidden=8, experts=4, top_k=2, type=0, x=F, ldx=8, router=F, w_in=F, w_out=F, chosen=F, gates=F, y=F, ldy=8,
        ws=F, nbytes=1 << 40):
    return h.ozimmu_moe(tokens, width, hidden, experts, top_k, type, 1, x, ldx, router, w_in, w_out, chosen, gates, y, ldy, ws, nbytes, None)


@pytest.mark.parametrize("wrong", [dict(tokens=-1), dict(tokens=65), dict(width=-1), dict(hidden=-1), dict(experts=0), dict(experts=513), dict(top_k=0),
                                   dict(top_k=5), dict(hidden=(1 << 24) + 1), dict(width=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), dict(experts=64, top_k=17), dict(type=3), dict(x=None), dict(ldx=7), dict(router=None),
                                   dict(w_in=None), dict(w_out=None), dict(chosen=None), dict(gates=None), dict(y=None), dict(ldy=7), dict(x=ODD),
                                   dict(router=ODD), dict(w_in=ODD), dict(w_out=ODD), dict(y=ODD), dict(ws=None), dict(nbytes=8),
                                   dict(chosen=ctypes.c_void_p((1 << 20) + 2)), dict(gates=ctypes.c_void_p((1 << 20) + 2))])
def test_moe_refuses(handle, wrong):
    assert moe(handle, **wrong) == BAD


def test_moe_of_no_tokens_and_its_workspace(handle):
    assert moe(handle, tokens=0, chosen=None, gates=None, x=None, y=None, ws=None, nbytes=0) == 0
    need = handle.ozimmu_moe_workspace_bytes
    assert need(4, 8, 100, 4, 2, 0) >= 4 * 2 * 100 * 2
    assert need(65, 8, 8, 4, 2, 0) == 0 and need(4, 8, 8, 4, 5, 0) == 0 and need(4, 8, 8, 4, 2, 3) == 0


def test_the_binding_refuses_what_it_can_see():
    import torch
    from paper_2506_11277_amd import layers
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        layers.linear(x, w)                       # not on a GPU
    with pytest.raises(ValueError):
        layers.adamw_state([x], bits=4)
    with pytest.raises(ValueError):
        layers.AdamW([x], [x], [x])
