"""The operators on rows in 8 bits at their largest sizes: more rows than one line of a launch's grid holds, and rows of up to 2^30 - 1 values."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.eight_reference import codes_of, norm, root_error
from tests.layers_reference import ROUND, U32, rounded, within

MOST = (1 << 30) - 1
BF16 = torch.bfloat16


def values(*shape, seed=41):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(generator=gen)


def parts(n, size=1 << 27):
    return [(i, min(i + size, n)) for i in range(0, n, size)]


def test_many_rows_of_one_value():
    # (a row's only value is its largest: code 127 or -127; the norm is the sign, nearly)
    x = values(MOST, 1)
    codes, scale = layers.quantise(x)
    y, _ = layers.rms_norm(x, eps=1e-5)
    torch.cuda.synchronize()
    for i, j in parts(MOST):
        part = x[i:j, 0].float()
        assert torch.equal(codes[i:j, 0].float(), 127 * part.sign()) and torch.equal(scale[i:j], part.abs() * (1.0 / 127))
        want = (part.double() / (part.double().square() + 1e-5).sqrt())
        assert bool(((y[i:j, 0].double() - want).abs() <= (ROUND[BF16] + 16 * U32) * want.abs()).all())


@pytest.mark.parametrize("cols", [8200, 16392])
def test_more_rows_of_a_work_group_than_one_line_of_the_grid(cols):
    rows = (1 << 21) + 5
    x = values(rows, cols)
    print(cols, flush=True)
    codes, scale = layers.quantise(x)
    torch.cuda.synchronize()
    assert bool((scale > 0).all())
    for i, j in ((0, 8), ((1 << 20) - 3, (1 << 20) + 3), ((1 << 21) - 3, rows)):
        want, top = codes_of(x[i:j].float())
        assert torch.equal(codes[i:j].cpu(), want)
        assert bool(((scale[i:j].double().cpu() - top).abs() <= 2 * U32 * top).all())
    del codes
    # the gradient in place of dy and h, which are one tensor: with eps = 1 it is r^3 x, the difference of r x and r x (1 - r^2)
    kept = {i: x[i:j].clone() for i, j in ((0, 8), ((1 << 21) - 3, rows))}
    layers.rms_norm_grad(x, x, eps=1.0, dx=x, want=("dx",))
    torch.cuda.synchronize()
    for i, h in kept.items():
        r, _ = norm(h, None, 1.0)
        want = r ** 3 * h.double()
        within(x[i:i + h.shape[0]], want, 2 * r * h.double().abs() * (3 * root_error(cols) + 128 * U32) + rounded(want, BF16), "dx")


def test_the_longest_row():
    x, weight = values(1, MOST), values(MOST, seed=42)
    y, _ = layers.rms_norm(x, weight, eps=1e-5)
    codes, scale, _ = layers.rms_norm8(x, weight, eps=1e-5)
    square, top = 0.0, 0.0
    for i, j in parts(MOST):
        square += float(x[0, i:j].double().square().sum())
        top = max(top, float((x[0, i:j].float() * weight[i:j].float()).abs().max()))
    r = (square / MOST + 1e-5) ** -0.5
    # (a thread's sum: 2^30 / 2^13 groups of 8 values; half of it in r)
    error = ((1 << 17) / 2 + 64) * U32
    assert abs(float(scale) - top / 127 * r) <= error * top / 127 * r
    inverse = torch.div(torch.tensor(127.0), torch.tensor(top)).cuda()
    for i, j in parts(MOST):
        t = x[0, i:j].float() * weight[i:j].float()
        assert torch.equal(codes[0, i:j].float(), torch.round(t * inverse))
        within(y[0, i:j], t.double() * r, (error + 4 * U32) * (t * r).abs().double() + rounded(t.double() * r, BF16), "y")
    del codes, y
    dy = weight[None]                       # with h = x and no weight: g = dy
    dx, dw = layers.rms_norm_grad(dy, x, eps=1e-5)
    mean = sum(float((dy[0, i:j].double() * x[0, i:j].double()).sum()) for i, j in parts(MOST)) * r / MOST
    size = sum(float((dy[0, i:j].double() * x[0, i:j].double()).abs().sum()) for i, j in parts(MOST)) * r / MOST
    for i, j in parts(MOST):
        g, n = dy[0, i:j].double(), x[0, i:j].double() * r
        within(dw[i:j], g * n, (error + 8 * U32) * (g * n).abs() + rounded(g * n, BF16), "dw")
        want = r * (g - n * mean)
        within(dx[0, i:j], want, r * (g.abs() + n.abs() * size) * 4 * error + rounded(want, BF16), "dx")


def test_gradients_of_many_rows():
    # dw: 2^20 of the tokens count, each with n = 1 / sqrt(1 + 1 / 4)
    dy, h = torch.zeros(MOST, 1, dtype=BF16, device="cuda"), torch.ones(MOST, 1, dtype=BF16, device="cuda")
    dy[::1 << 10] = 1.0
    dx, dw = layers.rms_norm_grad(dy, h, eps=0.25)
    torch.cuda.synchronize()
    n = 1.25 ** -0.5
    # at most 1024 terms one behind the other in a thread; of the 2^18 parts' sums, 2^13 to a thread, the 1024 that are not 0 meet in one thread, then 32
    assert abs(float(dw) - (1 << 20) * n) <= ((1 << 20) * n) * (ROUND[BF16] + (1024 + 1024 + 64) * U32)
    want = n * (1 - n * n)
    assert all(bool(((dx[i:j, 0].double() - want * dy[i:j, 0].double()).abs() <= want * (2 * ROUND[BF16])).all()) for i, j in parts(MOST))


@pytest.mark.parametrize("n_in", [1, 17])
def test_linear8_of_many_tokens(n_in):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.zeros(MOST, n_in, dtype=torch.int8, device="cuda")
    for i, j in parts(MOST):
        x[i:j, n_in - 1] = torch.randint(-127, 128, (j - i,), dtype=torch.int8, device="cuda", generator=gen)
    xs = torch.ones(MOST, device="cuda")
    xs[::3] = 0.5
    w = torch.full((1, n_in), 3, dtype=torch.int8, device="cuda")
    y = layers.linear8(x, xs, w, torch.ones(1, device="cuda"), dtype=BF16)
    torch.cuda.synchronize()
    for i, j in parts(MOST):
        assert torch.equal(y[i:j, 0], (x[i:j, n_in - 1].float() * 3 * xs[i:j]).to(BF16))


@pytest.mark.parametrize("n_out", [(1 << 26) + 5, MOST])
def test_linear8_of_many_features(n_out):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    w = torch.randint(-127, 128, (n_out, 1), dtype=torch.int8, device="cuda", generator=gen)
    ws = torch.ones(n_out, device="cuda")
    ws[::5] = 0.25
    for tokens in (1, 20):
        if tokens * n_out > 1 << 32:
            continue
        x = torch.full((tokens, 1), 5, dtype=torch.int8, device="cuda")
        y = layers.linear8(x, torch.ones(tokens, device="cuda"), w, ws)
        torch.cuda.synchronize()
        for i, j in parts(n_out):
            assert torch.equal(y[tokens - 1, i:j], (w[i:j, 0].float() * 5 * ws[i:j]).to(BF16))


def test_gradients_from_8_bits_of_many_tokens():
    # sums over the tokens of ones and zeros, below 2^24; scales of 1.5, half of which goes into dz
    dy, x = torch.zeros(MOST, 1, dtype=BF16, device="cuda"), torch.zeros(MOST, 1, dtype=torch.int8, device="cuda")
    dy[::1 << 10], x[::1 << 12] = 1.0, 2
    xs = torch.full((MOST,), 1.5, device="cuda")
    dx, dw, db = layers.linear8_grad(dy, x, torch.ones(1, 1, dtype=BF16, device="cuda"), x_scale=xs)
    torch.cuda.synchronize()
    assert float(db) == 1 << 20 and float(dw) == 3 * (1 << 18)
    assert all(torch.equal(dx[i:j], dy[i:j]) for i, j in parts(MOST))


def test_entries_beyond_32_bit_offsets():
    ld, rows = (1 << 20) + 8, 2200
    buf = torch.zeros(rows * ld, dtype=BF16, device="cuda")
    x = buf.view(rows, ld)[:, :136]
    x.copy_(values(rows, 136))
    plain = x.contiguous()
    out = torch.zeros(rows * ld, dtype=torch.int8, device="cuda").view(rows, ld)[:, :136]
    codes, scale, total = layers.rms_norm8(x, None, x, out=out)
    want = layers.rms_norm8(plain, None, plain)
    assert all(torch.equal(a, b) for a, b in zip((codes, scale, total), want))
    assert torch.equal(layers.rms_norm_grad(x, x)[0], layers.rms_norm_grad(plain, plain)[0])
    dy = values(rows, 8)
    w = values(8, 136, seed=3)
    assert all(torch.equal(a, b) for a, b in zip(layers.linear8_grad(dy, codes, w, x_scale=scale), layers.linear8_grad(dy, want[0], w, x_scale=scale)))


@pytest.mark.parametrize("cols,line", [(1600, 1 << 22), (4104, 1 << 22), (24584, 1 << 21)])
def test_more_rows_than_one_line_of_the_grid_of_every_kernel(cols, line):
    # 256, 512 and 1024 threads a row, rows in registers
    rows = line + 5
    x = values(rows, cols)
    print(cols, flush=True)
    codes, scale = layers.quantise(x)
    torch.cuda.synchronize()
    assert bool((scale > 0).all())
    for i, j in ((0, 8), (line // 2 - 3, line // 2 + 3), (line - 3, rows)):
        want, top = codes_of(x[i:j].float())
        assert torch.equal(codes[i:j].cpu(), want)
        assert bool(((scale[i:j].double().cpu() - top).abs() <= 2 * U32 * top).all())
