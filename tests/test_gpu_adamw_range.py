"""AdamW's moments in 8 bits over the range of float32: every size of gradient is held as well as any other."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.layers_reference import TYPES


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-12, 1.0, 2e5, 1e6, 1e10, 1e13, 1e18])
def test_moments_in_8_bits_of_any_size(size, kind):
    # the first step from nothing: m = 0.1 g and a root of v of sqrt(0.001) |g|
    n = 1 << 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    g = torch.randn(n, device="cuda", generator=gen).mul_(size).to(TYPES[kind])
    p = [torch.zeros(n, device="cuda")]
    m, v, m_scale, v_scale = layers.adamw_state(p, bits=8)
    print(size, kind, flush=True)
    layers.AdamW(p, m, v, m_scale, v_scale).step([g], 1, seed=1)
    torch.cuda.synchronize()
    G = g.double()
    for what, x, codes, scale in (("m", G * (1 - 0.9), m[0], m_scale[0]), ("root", (G * G * (1 - 0.999)).sqrt(), v[0], v_scale[0])):
        x = x.view(-1, 256)
        top = x.abs().amax(1, keepdim=True)
        # (in 32 bits a moment is off by a few of its units: 1e-6 of it)
        assert bool(((scale.double()[:, None] * 448 - top).abs() <= 1e-6 * top).all()), what
        y, held = x * 448 / top, codes.double().view(-1, 256)
        unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
        off = (held - y) / unit
        # one of the two codes beside the value, up or down by its distance from them: a block's largest value is the largest
        # code, and over 65536 values, each off by half a unit at most in the root mean square, the mean stays within 6 / 256 / 2
        # (of m; a root that is not 0 does not become 0, so that the smallest are off to one side: they are left out)
        assert bool((off.abs() <= 1 + 1e-4).all()), what
        assert bool((held.abs().amax(1) == 448).all()), what
        towards = (off * torch.sign(y))[y.abs() >= 2.0 ** -6]
        assert towards.numel() > 60000 and abs(float(towards.mean())) <= 6 * 0.5 / 244, what
