"""ozimmu_linear with workspaces that it does not need but could use: wherever they are."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.layers_reference import TYPES


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("behind", [1, 2, 4, 8, 24, 64, 128, 256])
def test_room_for_copies_that_is_not_aligned(behind, kind):
    tokens, n_in, n_out = 700, 1000, 776
    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    x, w = (torch.randn(rows, n_in + 3, device="cuda", generator=gen).to(TYPES[kind])[:, :n_in] for rows in (tokens, n_out))
    without = layers.linear_workspace_bytes(tokens, n_in, n_out, x.dtype, True)
    room = layers.linear_workspace_bytes(tokens, n_in, n_out, x.dtype, False)
    assert without == 0 < room
    buffer = torch.full((room + 1024,), 255, dtype=torch.uint8, device="cuda")
    print(behind, kind, flush=True)
    y = layers.linear(x, w, workspace=buffer[behind:])
    plain = layers.linear(x, w, workspace=buffer[:0])
    copied = layers.linear(x, w)
    torch.cuda.synchronize()
    # without room the operands go another way, in the same order of sums of a contraction that is not divided
    for other in (plain, copied):
        assert bool(((y.double() - other.double()).abs() <= 2.0 ** -7 * y.double().abs() + 1e-3).all())
    if behind % 256:
        assert torch.equal(y, plain) and bool((buffer == 255).all())
