"""ozimmu_linear8_grad against 64-bit forms, and the layers in 8 bits together: a block's step, captured, on other streams."""
import itertools
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.eight_reference import guarded_codes
from tests.layers_reference import LEAST, ROUND, TYPES, U32, act, guarded, product_bound, rounded, slope, sum_bound, untouched, within

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
HELD = [(True, False, True), (True, True, True), (True, False, False), (False, True, False), (False, False, True), (False, False, False)]   # x, w, pre
SHAPES = [(1, 1, 1), (1, 1024, 300), (2, 0, 40), (0, 40, 24), (3, 40, 0), (7, 64, 16), (16, 65, 15), (33, 1000, 130), (64, 127, 129), (128, 128, 128), (129, 63, 257),
          (300, 1000, 256), (512, 384, 500), (1531, 1001, 777), (4097, 72, 64)]
# the larger tiles: of dx and dw, alone and in one launch
LARGE = [("16", (3000, 4096, 264)), ("16", (264, 4096, 3000)), ("16", (3001, 4096, 3003)), ("16", (1777, 1024, 2304)), ("16", (640, 4096, 640)),
         ("f32", (1777, 2048, 777)), ("f32", (640, 776, 4096))]


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def held_rows(values, eight, kind, extra):
    """(operand, scale, the values it stands for in 64 bits)."""
    rows, cols = values.shape
    if not eight:
        x = guarded(rows, cols, cols + extra, TYPES[kind], values)[0] if cols + extra else values.to(TYPES[kind])
        return x, None, x.double()
    codes = guarded_codes(rows, cols, cols + extra)[0] if cols + extra else None
    codes, scale = layers.quantise(values, out=codes)
    return codes, scale, codes.double() * scale.double()[:, None]


def check(got, dy, x, w, pre, name, kind, held):
    dtype, u = TYPES[kind], ROUND[TYPES[kind]]
    dx, dw, db = got
    G = dy.double()
    dz = G * slope(name, pre)
    # pre's product with its scale and the slope in 32 bits, then one rounding of dz for the products (behind two products with parts of scales)
    sb = 0 if name in ("none", "relu") else 32 * U32 * G.abs() * (1 + pre.abs()) ** 2
    zb = sb + (0 if name == "none" and (kind == "f32" or not (held[0] or held[1])) else rounded(dz, dtype) + 4 * U32 * dz.abs())
    # what is held in 8 bits: in 32 bits the product with the scale, in 16 nothing but float16's least numbers (times the scale's other part, below 2)
    xb, wb = ((U32 * v.abs() if kind == "f32" else torch.full_like(v, 2 * LEAST[dtype])) if h else None for v, h in ((x, held[0]), (w, held[1])))
    for out, P, Q, PB, QB, what in ((dx, dz, w.t(), zb, None if wb is None else wb.t(), "dx"), (dw, dz.t(), x.t(), zb.t() if torch.is_tensor(zb) else zb, None if xb is None else xb.t(), "dw")):
        if out is None:
            continue
        want = torch.matmul(P, Q.t())
        bound = product_bound(P, Q, 2 * U32) + 4 * U32 * want.abs()
        if torch.is_tensor(PB):
            bound = bound + torch.matmul(PB, Q.abs().t())
        if QB is not None:
            bound = bound + torch.matmul(P.abs() + PB, QB.t())
        within(out, want, bound + rounded(want, dtype) + u * bound, what)
    if db is not None:
        want = dz.sum(0)
        bound = dz.abs().sum(0) * sum_bound(dy.shape[0]) + (sb.sum(0) if torch.is_tensor(sb) else 0)
        within(db, want, bound + rounded(want, dtype) + u * bound, "db")


def run(shape, kind, extra, name, held, want=("dx", "dw")):
    tokens, n_in, n_out = shape
    gen = generator(200 + n_in)
    x, w, z, dy = (torch.randn(*s, device="cuda", generator=gen) * std for s, std in (((tokens, n_in), 1.0), ((n_out, n_in), max(1, n_in) ** -0.5),
                                                                                      ((tokens, n_out), 1.0), ((tokens, n_out), 1.0)))
    (x, xs, X), (w, ws, W), (z, zs, Z) = (held_rows(v, h, kind, extra) for v, h in zip((x, w, z), held))
    dy = guarded(tokens, n_out, n_out + extra, TYPES[kind], dy)[0] if n_out + extra else dy.to(TYPES[kind])
    (dx, xbuf), (dw, wbuf) = (guarded(rows, n_in, n_in + extra, TYPES[kind]) if n_in + extra else (None, None) for rows in (tokens, n_out))
    print(shape, kind, extra, name, held, flush=True)
    given = dict(activation=layers.ACTIVATIONS[name], x_scale=xs, w_scale=ws, pre_scale=zs if name != "none" else None)
    got = layers.linear8_grad(dy, x, w, None if name == "none" else z, dx=dx, dw=dw, **given)
    torch.cuda.synchronize()
    check(got, dy, X, W, Z, name, kind, held)
    if n_in + extra:
        assert untouched(dx, xbuf) and untouched(dw, wbuf)
    return got, (dy, x, w, z), given


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("extra", [0, 16, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients(shape, extra, kind):
    for i, held in enumerate(HELD):
        run(shape, kind, extra, ACTS[(sum(shape) + extra + i) % 5], held)


@pytest.mark.parametrize("kind,shape", [(k, s) for c, s in LARGE for k in (("bf16", "f16") if c == "16" else ("f32",))])
@pytest.mark.parametrize("extra", [0, 3])
def test_gradients_in_the_larger_tiles(kind, shape, extra):
    for held, name in ((HELD[0], "gelu"), (HELD[1], "silu"), (HELD[3], "none")):
        run(shape, kind, extra, name, held)


@pytest.mark.parametrize("shape", [(300, 1000, 256), (129, 63, 257)])
def test_it_forms_what_is_asked_for(shape):
    for held in HELD[:2]:
        all_, operands, given = run(shape, "bf16", 0, "gelu", held)
        for want in (("dx",), ("dw",), ()):
            got = layers.linear8_grad(*operands, want=want, bias="dw" not in want, **given)
            for name, a, b in zip(("dx", "dw", "db"), all_, got):
                if name in want or (name == "db" and "dw" not in want):
                    assert torch.equal(a, b)
                else:
                    assert b is None


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_without_8_bits_it_is_linear_grad(kind):
    got, (dy, x, w, z), given = run((300, 200, 96), kind, 0, "silu", HELD[5])
    assert all(torch.equal(a, b) for a, b in zip(got, layers.linear_grad(dy, x, w, z, layers.ACT_SILU)))


@pytest.mark.parametrize("shape,extra", [((700, 1001, 777), 0), ((700, 1000, 776), 3), ((130, 2048, 4099), 0)])
def test_with_and_without_room_for_copies(shape, extra):
    # dy's rows off 16 bytes: without room for a copy of it, it goes another way
    for held, name in itertools.product(HELD[:4], ("none", "gelu")):
        got, (dy, x, w, z), given = run(shape, "bf16", extra, name, held)
        X, W, Z = (v.double() * s.double()[:, None] if s is not None else v.double() for v, s in ((x, given["x_scale"]), (w, given["w_scale"]), (z, given["pre_scale"] if held[2] and name != "none" else None)))
        if name == "none":
            Z = torch.zeros_like(Z)
        nbytes = layers.linear8_grad_workspace_bytes(*shape, dy.dtype, given["activation"], True, held[0], held[1])
        tight = torch.full((max(256, nbytes),), 255, dtype=torch.uint8, device="cuda")
        check(layers.linear8_grad(dy, x, w, None if name == "none" else z, workspace=tight, **given), dy, X, W, Z, name, "bf16", held)


def test_a_scale_that_is_not_finite():
    # a token whose pre-activations have no scale has no gradient, nor has any weight (dw sums over the tokens); the other tokens' dx stay
    got, (dy, x, w, z), given = run((40, 64, 48), "bf16", 0, "gelu", HELD[0])
    given["pre_scale"][3] = float("nan")
    dx, dw, db = layers.linear8_grad(dy, x, w, z, **given)
    assert bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dw).all()) and bool(torch.isnan(db).all())
    keep = [i for i in range(40) if i != 3]
    assert torch.equal(dx[keep], got[0][keep])


def test_scales_of_any_size():
    # zeros, powers of two, scales below the normal numbers and negative ones stand for what they are; codes of -128 too
    gen = generator(3)
    x8, w8 = (torch.randint(-128, 128, (rows, 40), dtype=torch.int8, device="cuda", generator=gen) for rows in (70, 24))
    xs, ws = torch.rand(70, device="cuda", generator=gen) + 0.5, torch.rand(24, device="cuda", generator=gen) - 0.5
    xs[0], xs[1], xs[2], xs[3], xs[4], xs[5] = 0.0, 1.0, 2.0 ** -30, -3.0, 2.0 ** -140, 1e30
    ws[0], ws[1] = 0.0, 2.0 ** 20
    for kind in ("bf16", "f32"):
        dy = torch.randn(70, 24, device="cuda", generator=gen).to(TYPES[kind])
        X, W = x8.double() * xs.double()[:, None], w8.double() * ws.double()[:, None]
        check(layers.linear8_grad(dy, x8, w8, x_scale=xs, w_scale=ws), dy, X, W, torch.zeros(70, 24, device="cuda").double(), "none", kind, (True, True, False))


def test_no_tokens_and_no_features():
    for kind in TYPES:
        one = torch.ones(24, device="cuda")
        w8 = torch.ones(24, 40, dtype=torch.int8, device="cuda")
        dx, dw, db = layers.linear8_grad(torch.empty(0, 24, dtype=TYPES[kind], device="cuda"), torch.empty(0, 40, dtype=torch.int8, device="cuda"), w8, x_scale=one[:0], w_scale=one)
        assert dx.shape == (0, 40) and bool((dw == 0).all()) and bool((db == 0).all())
        dx, dw, db = layers.linear8_grad(torch.empty(24, 0, dtype=TYPES[kind], device="cuda"), w8, w8[:0], x_scale=one, w_scale=one[:0])
        assert bool((dx == 0).all()) and dw.shape == (0, 40) and db.shape == (0,)


class Block:
    """y = x + W2 gelu(W1 norm(x) + b1) + b2 in 8 bits, as a training step runs it: what the gradients need is kept in 8 bits."""

    def __init__(self, tokens, width, hidden, kind, seed=0):
        gen = generator(seed)
        dtype = TYPES[kind]

        def normal(*shape, std=1.0):
            return (torch.randn(*shape, device="cuda", generator=gen) * std).to(dtype)

        self.x, self.dy = normal(tokens, width), normal(tokens, width)
        self.g = 1 + normal(width, std=0.2)
        self.w1, self.b1, self.w2, self.b2 = normal(hidden, width, std=width ** -0.5), normal(hidden), normal(width, hidden, std=hidden ** -0.5), normal(width)

    def step(self):
        (w1, s1), (w2, s2) = layers.quantise(self.w1), layers.quantise(self.w2)
        n8, ns, x = layers.rms_norm8(self.x, self.g)
        pre = torch.empty(x.shape[0], self.w1.shape[0], dtype=x.dtype, device="cuda")
        h = layers.linear8(n8, ns, w1, s1, self.b1, activation=layers.ACT_GELU, pre=pre)
        h8, hs = layers.quantise(h)
        p8, ps = layers.quantise(pre)
        y = layers.linear8(h8, hs, w2, s2, self.b2, x)
        self.kept = (n8, ns, w1, s1, h8, hs, w2, s2, p8, ps, pre)
        dh, dw2, db2 = layers.linear8_grad(self.dy, h8, self.w2, x_scale=hs)
        dn, dw1, db1 = layers.linear8_grad(dh, n8, self.w1, p8, layers.ACT_GELU, x_scale=ns, pre_scale=ps)
        dx, dg = layers.rms_norm_grad(dn, x, self.g, add=self.dy)
        return y, dx, dg, dw1, db1, dw2, db2


def values_of(codes, scale):
    return codes.double() * scale.double()[:, None]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 64, 96), (300, 256, 520)])
def test_a_block_of_them(shape, kind):
    block = Block(*shape, kind)
    y, dx, dg, dw1, db1, dw2, db2 = block.step()
    n8, ns, w1, s1, h8, hs, w2, s2, p8, ps, pre = block.kept
    # every operator from what it was given, in 64 bits: relative to the largest value, some roundings to the type each
    x, g = block.x.double(), block.g.double()
    r = (x.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    N, W1, H, W2, P = values_of(n8, ns), values_of(w1, s1), values_of(h8, hs), values_of(w2, s2), values_of(p8, ps)

    def near(got, want, steps):
        assert float((got.double() - want).abs().max()) <= steps * ROUND[TYPES[kind]] * float(want.abs().max())

    # 8 bits: half a code, 1/254 of a row's largest value
    for got, want in ((N, x * r * g), (P, pre.double())):
        assert bool(((got - want).abs() <= want.abs().amax(1, keepdim=True) * (0.5 / 127 + 2.0 ** -16)).all())
    near(pre, N @ W1.t() + block.b1.double(), 2)
    near(y, x + H @ W2.t() + block.b2.double(), 2)
    dh = block.dy.double() @ block.w2.double()
    near(dw2, block.dy.double().t() @ H, 2 + shape[0] ** 0.5)           # (a sum over the tokens of products of rounded values)
    near(db2, block.dy.double().sum(0), 2 + shape[0] * U32 / ROUND[TYPES[kind]])
    dz = dh * slope("gelu", P)
    near(db1, dz.sum(0), 4 + 2 * shape[0] ** 0.5)
    near(dw1, dz.t() @ N, 4 + 2 * shape[0] ** 0.5)
    dn = dz @ block.w1.double()
    gg = dn * g
    near(dx, r * (gg - x * r * (gg * x * r).mean(1, keepdim=True)) + block.dy.double(), 16)
    near(dg, (dn * x * r).sum(0), 8 + 4 * shape[0] ** 0.5)


def test_a_block_in_a_graph_beside_eager_ones():
    block, other = Block(70, 96, 200, "bf16"), Block(300, 256, 520, "bf16", 1)
    block.step(), other.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = block.step()
    for turn in range(4):
        block.x.copy_(torch.randn(block.x.shape, device="cuda", generator=generator(30 + turn)))
        for t in results:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        other.step()
        want = block.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_blocks_on_two_streams():
    blocks = [Block(300, 256, 520, "f16", i) for i in range(2)]
    want = [b.step() for b in blocks]
    torch.cuda.synchronize()
    sides, got = [torch.cuda.Stream() for _ in blocks], []
    for _ in range(3):
        for b, side in zip(blocks, sides):
            with torch.cuda.stream(side):
                got.append(b.step())
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for i, g in enumerate(got) for p, q in zip(g, want[i % 2]))


@pytest.mark.parametrize("held", [(True, False, True), (False, True, False), (True, True, False), (True, True, True)])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_gradients_up_to_their_types_range(kind, held):
    # what linear_grad takes stays finite: dz up to 60000 (bfloat16: 3e38), beside scales of every m in [1, 2)
    gen = generator(17)
    tokens, n_in, n_out = 70, 48, 40
    most = 6e4 if kind == "f16" else 3e38
    dy = (torch.empty(tokens, n_out, device="cuda").uniform_(1 / 3, 1.0, generator=gen) * most).to(TYPES[kind])
    dy[1::2] *= -1
    x, w = (torch.empty(rows, n_in, device="cuda").uniform_(-1.0, 1.0, generator=gen) * 2.0 ** -9 for rows in (tokens, n_out))
    x, w = (v * torch.linspace(1.0, 2.0, v.shape[0], device="cuda")[:, None] for v in (x, w))
    (x, xs, X), (w, ws, W) = (held_rows(v, h, kind, 0) for v, h in zip((x, w), held))
    z = torch.empty(tokens, n_out, device="cuda").uniform_(1.0, 2.0, generator=gen)
    z, zs, Z = held_rows(z, held[2], kind, 0)
    check(layers.linear8_grad(dy, x, w, z, layers.ACT_RELU, x_scale=xs, w_scale=ws, pre_scale=zs, bias=False), dy, X, W, Z, "relu", kind, held)


@pytest.mark.parametrize("kind,scales", [("f16", (200.0, 1e5)), ("bf16", (2.0 ** 119, 3e38))])
def test_codes_whose_values_leave_the_range_of_16_bits(kind, scales):
    # the values that they stand for are finite in 64 bits (beyond 65504, or 2^128), and so are the results
    gen = generator(18)
    x8, w8 = (torch.randint(-128, 128, (rows, 40), dtype=torch.int8, device="cuda", generator=gen) for rows in (70, 24))
    x8[0], w8[0] = -128, -128
    xs, ws = (torch.empty(rows, device="cuda").uniform_(0.0, 1.0, generator=gen).mul_(math.log(scales[1] / scales[0])).exp_().mul_(scales[0]) for rows in (70, 24))
    dy = (torch.randn(70, 24, device="cuda", generator=gen) * (2.0 ** -12 if kind == "f16" else 1e-8)).to(TYPES[kind])
    X, W = x8.double() * xs.double()[:, None], w8.double() * ws.double()[:, None]
    Z = torch.zeros(70, 24, device="cuda").double()
    dx, dw, _ = layers.linear8_grad(dy, x8, w8, x_scale=xs, w_scale=ws, bias=False)
    check((dx, dw, None), dy, X, W, Z, "none", kind, (True, True, False))


@pytest.mark.parametrize("kind,shape", [("bf16", (2048, 256, 256)), ("f32", (500, 512, 384))])
@pytest.mark.parametrize("held", HELD[:4])
def test_gradients_asked_for_alone(kind, shape, held):
    # alone, dx or dw may be summed in other parts than in the launch for both: the bounds hold either way, and a call repeats itself
    _, (dy, x, w, z), given = run(shape, kind, 0, "gelu", held)
    X, W, Z = (v.double() * s.double()[:, None] if s is not None else v.double() for v, s in ((x, given["x_scale"]), (w, given["w_scale"]), (z, given["pre_scale"])))
    for want, bias in ((("dx",), True), (("dw",), True), (("dw",), False), (("dx", "dw"), False)):
        got, again = (layers.linear8_grad(dy, x, w, z, want=want, bias=bias, **given) for _ in range(2))
        check(got, dy, X, W, Z, "gelu", kind, held)
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, again))
