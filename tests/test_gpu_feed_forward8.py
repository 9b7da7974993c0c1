"""The example's block in 8 bits: it runs, runs again the same, and its gradients are those of the formulas."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.test_gpu_feed_forward import example  # noqa: F401


def test_training_runs(example):  # noqa: F811
    losses = example.train(20, block=example.FeedForward8)
    assert len(losses) == 20 and all(0 < loss < float("inf") for loss in losses)
    assert losses == example.train(20, block=example.FeedForward8)


def test_its_gradients(example):  # noqa: F811
    # in 64 bits, from what the forward pass kept, by differentiation: the slopes are those at the kept values, roundings to 8 bits the identity
    torch.manual_seed(2)
    tokens, width, hidden = 200, 64, 96
    block = example.FeedForward8(width, hidden)
    x, dy = (torch.randn(tokens, width, device="cuda").bfloat16() for _ in range(2))
    y = block.forward(x)
    dx, got = block.backward(dy)
    _, n, n_scale, pre, pre_scale, h, h_scale = block.kept
    N, P, H = (c.double() * s.double()[:, None] for c, s in ((n, n_scale), (pre, pre_scale), (h, h_scale)))
    gain, w1, b1, w2, b2 = (w.double().requires_grad_(True) for w in block.weights)
    X, D = x.double().requires_grad_(True), dy.double()

    def held(value, through):                # the value that is held, with the gradient of what it was made of
        return value + through - through.detach()

    norm = X * (X.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain
    before = held(P, held(N, norm) @ w1.t() + b1)
    after = held(H, before * torch.special.ndtr(before))
    out = X + after @ w2.t() + b2
    want = torch.autograd.grad((out * D).sum(), (X, gain, w1, b1, w2, b2))
    # y: both weights in 8 bits, half a code of 127 each way, and 16-bit results
    assert float((y.double() - out.detach()).abs().max()) <= 0.05 * float(out.detach().abs().max())
    # a few roundings to bfloat16, of sums of products of rounded values
    for a, b, what in zip((dx, *got), want, ("x", "gain", "w1", "b1", "w2", "b2")):
        off = float((a.double() - b).norm() / b.norm())
        assert off <= 4 * 2.0 ** -8, (what, off)
