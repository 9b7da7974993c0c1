"""The layers' largest sizes: thin matrices of up to 2^30 - 1 rows, whose tiles are more than one row of a launch's grid."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers

MOST = (1 << 30) - 1


def values(*shape):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(31)
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def same(got, want, rows=1 << 27):
    """Equality in parts (want: a function of a range of rows)."""
    return all(torch.equal(got[i:i + rows], want(i, min(i + rows, got.shape[0]))) for i in range(0, got.shape[0], rows))


@pytest.mark.parametrize("n_out", [(1 << 26) + 5, (1 << 27) + 5, MOST])
def test_one_token_of_many_features(n_out):
    # (a product of two bfloat16 numbers is exact in 32 bits)
    x, w = values(1, 1), values(n_out, 1)
    print(n_out, flush=True)
    y = layers.linear(x, w)
    torch.cuda.synchronize()
    assert same(y[0], lambda i, j: (w[i:j, 0].float() * x.float()[0, 0]).bfloat16())


@pytest.mark.parametrize("n_in", [1, 9])
def test_many_tokens(n_in):
    x, w = values(MOST, n_in), values(1, n_in)
    x[:, 1:] = 0                                       # (one product a sum: exact again)
    print(n_in, flush=True)
    y = layers.linear(x, w)
    torch.cuda.synchronize()
    assert same(y[:, 0], lambda i, j: (x[i:j, 0].float() * w.float()[0, 0]).bfloat16())


def test_gradients_of_many_features():
    dy, x, w = values(1, MOST), values(1, 1), values(MOST, 1)
    dx, dw, db = layers.linear_grad(dy, x, w, want=("dw",))
    torch.cuda.synchronize()
    assert dx is None and torch.equal(db, dy[0])
    assert same(dw[:, 0], lambda i, j: (dy[0, i:j].float() * x.float()[0, 0]).bfloat16())


def test_gradients_of_many_tokens():
    # the sums over the tokens are of ones and zeros, below 2^24
    dy, x, w = torch.zeros(MOST, 1, dtype=torch.bfloat16, device="cuda"), torch.zeros(MOST, 1, dtype=torch.bfloat16, device="cuda"), values(1, 1)
    dy[::1 << 10], x[::1 << 12] = 1.0, 1.0
    dx, dw, db = layers.linear_grad(dy, x, w)
    torch.cuda.synchronize()
    assert float(db) == 1 << 20 and float(dw) == 1 << 18
    assert same(dx[:, 0], lambda i, j: dy[i:j, 0] * w[0, 0])
