"""The layers' binding on the CPU, with a stand-in for the library that notes what it is called with."""
import gc
import weakref

import pytest

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers


class Library:
    """Notes the types that each AdamW step sends for its gradients."""

    def __init__(self):
        self.grad_types = []

    def ozimmu_adamw(self, n, tensors, *rest):
        self.grad_types.append([t.grad_type for t in tensors])
        return layers.OK


@pytest.fixture
def library(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(layers, "_lib", stand_in)
    monkeypatch.setattr(layers, "_type_of", lambda x, what: layers._TYPES[x.dtype])
    monkeypatch.setattr(layers, "_stream", lambda index, what: None)
    return stand_in


def plan_of(sizes):
    params = [torch.ones(n) for n in sizes]
    m, v, _, _ = layers.adamw_state(params)
    return layers.AdamW(params, m, v)


@pytest.mark.parametrize("first", [torch.bfloat16, torch.float32])
def test_a_refused_step_leaves_the_plan_as_it_was(library, first):
    plan = plan_of([5, 6])
    plan.step([torch.ones(n, dtype=first) for n in (5, 6)], 1)
    other = torch.float32 if first is torch.bfloat16 else torch.bfloat16
    with pytest.raises(ValueError):
        plan.step([torch.ones(5, dtype=other), torch.ones(6, dtype=torch.float64)], 2)
    plan.step([torch.ones(n, dtype=first) for n in (5, 6)], 2)
    assert library.grad_types == [[layers._TYPES[first]] * 2] * 2
    plan.step([torch.ones(5, dtype=other), torch.ones(6, dtype=first)], 3)
    assert library.grad_types[-1] == [layers._TYPES[other], layers._TYPES[first]]


def test_a_plan_keeps_its_tensors_whatever_becomes_of_the_lists(library):
    params = [torch.ones(300), torch.ones(7)]
    lists = [params, *layers.adamw_state(params, bits=8), [p.bfloat16() for p in params]]
    kept = [weakref.ref(t) for x in lists for t in x]
    plan = layers.AdamW(lists[0], *lists[1:5], copies=lists[5])
    del params
    for x in lists:
        x[0] = torch.zeros(1)
        x.clear()
    gc.collect()
    assert all(r() is not None for r in kept)
    plan.step([torch.ones(300), torch.ones(7)], 1)
    del plan
    gc.collect()
    assert all(r() is None for r in kept)


@pytest.mark.parametrize("rows,cols,ld", [(2, 8, (1 << 32) + 8), (2, 8, 1 << 31), (2, (1 << 32) + 8, (1 << 32) + 8), ((1 << 32) + 2, 8, 8), (1, 1 << 30, 1 << 30)])
def test_sizes_that_an_int_cannot_hold_are_refused(rows, cols, ld):
    # (the library takes ints: 2^32 + 8 would arrive there as 8)
    x = torch.empty_strided((rows, cols), (ld, 1), dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError):
        layers._ld(x, rows, cols, x, "x")


def test_sizes_up_to_the_largest_are_taken():
    most = (1 << 30) - 1
    for rows, cols, ld in ((2, most, (1 << 31) - 1), (most, 1, 1), (0, most, most), (1, 8, 1 << 40)):
        x = torch.empty_strided((rows, cols), (ld, 1), dtype=torch.bfloat16, device="meta")
        assert layers._ld(x, rows, cols, x, "x") == (ld if rows > 1 else cols)


def test_workspaces_of_sizes_that_an_int_cannot_hold():
    big = (1 << 32) + 300
    for call in (lambda: layers.linear_workspace_bytes(big, 8, 8, torch.bfloat16), lambda: layers.linear_grad_workspace_bytes(8, big, 8, torch.bfloat16),
                 lambda: layers.moe_workspace_bytes(4, 8, big, 8, 2, torch.bfloat16), lambda: layers.moe_workspace_bytes(4, 8, 8, 8, big, torch.bfloat16)):
        with pytest.raises(ValueError):
            call()


def test_experts_that_an_int_cannot_hold_are_refused(library):
    # (two experts too many would arrive as two)
    def meta(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="meta")

    for experts, hidden in (((1 << 32) + 2, 8), (2, (1 << 32) + 8)):
        with pytest.raises(ValueError, match="sizes"):
            layers.moe(meta(1, 8), meta(experts, 8), meta(experts, 2 * hidden, 8), meta(experts, 8, hidden), 1)


def test_autograd_notices_weights_that_a_step_changed(library):
    weight = torch.ones(3, requires_grad=True)
    m, v, _, _ = layers.adamw_state([weight])
    half = weight.detach().bfloat16()
    plan = layers.AdamW([weight], m, v, copies=[half])
    x = torch.ones(3, requires_grad=True)
    loss, rounded = (x * weight).sum(), (x.bfloat16() * half).sum()
    plan.step([torch.ones(3)], 1)
    for saved in (loss, rounded):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            saved.backward()


def test_tensors_of_a_plan_that_overlap_are_refused(library):
    # (two work-groups would update the shared values at once)
    whole, other = torch.ones(600), torch.ones(300)
    m, v, _, _ = layers.adamw_state([whole, other])
    for params in ([whole, whole], [whole[:300], whole[299:599]]):
        state = layers.adamw_state(params)[:2]
        with pytest.raises(ValueError, match="overlap"):
            layers.AdamW(params, *state)
    with pytest.raises(ValueError, match="overlap"):
        layers.AdamW([other, torch.ones(300)], [m[1], torch.zeros(300)], [v[1], m[1]])
    half = whole[:300].bfloat16()
    with pytest.raises(ValueError, match="overlap"):
        layers.AdamW([other, whole[300:]], *layers.adamw_state([other, other])[:2], copies=[half, half])
    layers.AdamW([whole[:300], whole[300:], torch.ones(0), torch.ones(0)], *layers.adamw_state([other, other, whole[:0], whole[:0]])[:2])
    # (scales that float moments do not use are nobody's)
    layers.AdamW([whole[:300], whole[300:]], *layers.adamw_state([other, other])[:2], m_scale=[other, other], v_scale=[other, other])
