"""Slopes of the activations where the value before them is large: 0 or 1, as the formulas have it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.layers_reference import TYPES

SIZES = [20.0, 1e3, 6e4, 1e10, 2e19, 1e25, 3e38]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("name", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_of_large_values(name, kind):
    dtype = TYPES[kind]
    sizes = [s for s in SIZES if s <= torch.finfo(dtype).max]
    z = torch.tensor([[s, -s] for s in sizes], device="cuda").repeat(1, 4).to(dtype)
    w = torch.eye(8, device="cuda").to(dtype)
    dy = torch.full_like(z, 3.0)
    dx, dw, db = layers.linear_grad(dy, torch.ones(len(sizes), 8, device="cuda").to(dtype), w, z, layers.ACTIVATIONS[name])
    # at 20 an activation's slope is 1 or 0 to 20 exp(-20), 4e-8
    want = torch.tensor([3.0, 0.0], device="cuda").repeat(len(sizes), 4)
    assert bool(((dx.float() - want).abs() <= 3e-7).all()), dx
    assert bool(((db.float() - want.sum(0)).abs() <= 3e-6).all()), db
    y = layers.linear(z, w, activation=layers.ACTIVATIONS[name])
    assert bool(((y.double() - z.double().clamp_min(0)).abs() <= 1e-7 * z.double().abs()).all()), y
