"""ozimmu_linear8: sums of products of codes exactly, the epilogue against 64-bit forms; its tiles, edges, parts and routes."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers, ozimmu
from tests.eight_reference import guarded_codes
from tests.layers_reference import ROUND, TYPES, U32, act, guarded, rounded, untouched, within

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
# one token ... many, sizes that fit tiles, miss them by one, and fit nothing; contractions of nothing, less than a step, and long
# enough to be divided among work-groups
SHAPES = [(1, 1, 1), (1, 1024, 4096), (1, 8192, 33), (2, 0, 40), (7, 64, 16), (16, 65, 15), (17, 2048, 64), (33, 1000, 130), (48, 8192, 260), (48, 16384, 600),
          (64, 127, 129), (65, 128, 128), (128, 128, 128), (129, 63, 257), (200, 4100, 72), (257, 256, 255), (300, 1000, 256),
          (512, 384, 500), (1531, 1001, 777), (1300, 72, 1288), (2300, 520, 2200), (3, 131071, 20), (70, 131071, 70)]


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def operands(tokens, n_in, n_out, extra, seed):
    """Codes over their whole range and scales of different sizes: (x, x_scale, w, w_scale)."""
    gen = generator(seed)

    def codes(rows):
        c = torch.randint(-128, 128, (rows, n_in), dtype=torch.int8, device="cuda", generator=gen)
        return guarded_codes(rows, n_in, n_in + extra, c)[0] if n_in + extra else c

    x, w = codes(tokens), codes(n_out)
    scale = [torch.empty(n, device="cuda").uniform_(0.5, 2.0, generator=gen) * s for n, s in ((tokens, 2.0 ** -6), (n_out, 2.0 ** -6 * max(1, n_in) ** -0.5))]
    return x, scale[0], w, scale[1]


def others(tokens, n_out, kind, extra, seed):
    gen = generator(seed)
    return (torch.randn(n_out, device="cuda", generator=gen).to(TYPES[kind]),
            guarded(tokens, n_out, n_out + extra, TYPES[kind], torch.randn(tokens, n_out, device="cuda", generator=gen))[0])


def check(x, xs, w, ws, bias, residual, name, y, pre):
    dtype = y.dtype
    z = torch.matmul(x.double(), w.double().t()) * xs.double()[:, None] * ws.double()
    b = 0.0 if bias is None else bias.double()
    # the sum to a float, two products, the bias: one rounding each
    zb = 3 * U32 * z.abs()
    z = z + b
    zb = zb + U32 * (z.abs() + zb)
    if pre is not None:
        within(pre, z, zb + rounded(z, dtype) + ROUND[dtype] * zb, "pre")
    a = act(name, z)
    # the slope of every activation is below 1.13; evaluated in 32 bits, whose exponential is off by a few units times its argument; gelu in 16 bits
    # by a polynomial: |z| Phi(-|z|) to 4e-6 up to 4 and 1e-5 up to 6, behind which it is below 6e-9
    ab = 1.2 * zb + (0 if name in ("none", "relu") else 16 * U32 * (a.abs() + z.abs() * (1 + z.abs()).clamp_max(8)))
    if name == "gelu" and dtype is not torch.float32:
        ab = ab + torch.where(z.abs() <= 4, 4e-6, 1e-5) * (z.abs() * torch.special.ndtr(-z.abs())) + 6e-9 * (z.abs() > 6)
    Y = a if residual is None else a + residual.double()
    ab = ab + (0 if residual is None else U32 * (Y.abs() + ab))
    within(y, Y, ab + rounded(Y, dtype) + ROUND[dtype] * ab, "y")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("extra", [0, 16, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_linear8(shape, extra, kind):
    tokens, n_in, n_out = shape
    x, xs, w, ws = operands(*shape, extra, 100 + n_in)
    bias, residual = others(tokens, n_out, kind, extra, 7)
    name = ACTS[(tokens + n_out + extra) % 5]
    (y, ybuf), (pre, pbuf) = (guarded(tokens, n_out, n_out + extra, TYPES[kind]) for _ in range(2))
    print(shape, kind, extra, name, flush=True)
    assert layers.linear8(x, xs, w, ws, bias, residual, layers.ACTIVATIONS[name], pre=pre, out=y) is y
    torch.cuda.synchronize()
    check(x, xs, w, ws, bias, residual, name, y, pre)
    assert untouched(y, ybuf) and untouched(pre, pbuf)
    stream = residual.clone(memory_format=torch.preserve_format)
    layers.linear8(x, xs, w, ws, bias, stream, layers.ACTIVATIONS[name], out=stream)          # added to in place
    assert torch.equal(stream, y)
    if kind == "f32":                           # without scales: the sums themselves, to the nearest float
        one = [torch.ones_like(s) for s in (xs, ws)]
        sums = layers.linear8(x, one[0], w, one[1], dtype=torch.float32)
        assert torch.equal(sums, torch.matmul(x.double(), w.double().t()).float())


def tile(shape, aligned=1):
    parts = ctypes.c_int()
    edge = ozimmu.lib().ozimmu_debug_linear_tile(0, *shape, 8, aligned, ctypes.byref(parts))
    return edge, parts.value > 1


# whole tiles and tiles that end anywhere, contractions that end within a step and are shorter than the ring
TILES = [((4096, 144, 4096), 256, False), ((4096, 656, 4096), 256, False), ((3000, 2000, 4099), 256, False), ((4097, 4112, 2300), 256, False),
         ((777, 16384, 2560), 256, True), ((1777, 128, 1777), 128, False), ((1790, 400, 1784), 128, False), ((1280, 2000, 1921), 128, False),
         ((300, 16384, 777), 128, True), ((777, 16384, 304), 128, True)]


@pytest.mark.parametrize("extra", [0, 16, 3])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape,edge,divided", TILES)
def test_linear8_in_the_larger_tiles(shape, edge, divided, kind, extra):
    assert tile(shape) == (edge, divided)
    tokens, n_in, n_out = shape
    x, xs, w, ws = operands(*shape, extra, 400 + n_in)
    bias, residual = others(tokens, n_out, kind, extra, 8)
    name = ACTS[(tokens + n_out + extra) % 5]
    (y, ybuf), (pre, pbuf) = (guarded(tokens, n_out, n_out + extra, TYPES[kind]) for _ in range(2))
    print(shape, kind, extra, name, flush=True)
    layers.linear8(x, xs, w, ws, bias, residual, layers.ACTIVATIONS[name], pre=pre, out=y)
    torch.cuda.synchronize()
    check(x, xs, w, ws, bias, residual, name, y, pre)
    assert untouched(y, ybuf) and untouched(pre, pbuf)
    check(x, xs, w, ws, None, None, name, layers.linear8(x, xs, w, ws, activation=layers.ACTIVATIONS[name], dtype=TYPES[kind]), None)


@pytest.mark.parametrize("tokens", [2, 40, 300])
def test_the_largest_sums(tokens):
    # 131071 products of -128 and -128: 2147467264, the sum that is nearest to 2^31
    x, w = (torch.full((n, layers.LINEAR8_IN), -128, dtype=torch.int8, device="cuda") for n in (tokens, 70))
    w[1] = 127
    y = layers.linear8(x, torch.ones(tokens, device="cuda"), w, torch.ones(70, device="cuda"), dtype=torch.float32)
    assert bool((y[:, 0] == float(128 * 128 * 131071)).all()) and bool((y[:, 1] == torch.tensor(-128.0 * 127 * 131071).float().cuda()).all())
    with pytest.raises(ValueError):
        layers.linear8(torch.zeros(1, layers.LINEAR8_IN + 1, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda"),
                       torch.zeros(1, layers.LINEAR8_IN + 1, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda"))


@pytest.mark.parametrize("shape,extra", [((700, 1001, 777), 0), ((700, 1008, 776), 3), ((1100, 2048, 4099), 1), ((20, 333, 50), 1)])
def test_unaligned_operands_with_and_without_room_for_copies(shape, extra):
    x, xs, w, ws = operands(*shape, extra, 33)
    results = [layers.linear8(x, xs, w, ws, workspace=torch.full((max(256, layers.linear8_workspace_bytes(*shape, aligned)),), 255, dtype=torch.uint8, device="cuda"))
               for aligned in (False, True)]
    check(x, xs, w, ws, None, None, "none", results[0], None)
    assert torch.equal(*results)                # (the sums are exact in any order)


@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_scales_that_are_not_finite_stay_in_their_rows(tokens):
    x, xs, w, ws = operands(tokens, 200, 96, 0, 9)
    want = layers.linear8(x, xs, w, ws)
    xs[1], ws[5] = float("nan"), float("inf")
    y = layers.linear8(x, xs, w, ws)
    assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[:, 5]).any())
    rows, cols = ([i for i in range(n) if i != j] for n, j in ((tokens, 1), (96, 5)))
    assert torch.equal(y[rows][:, cols], want[rows][:, cols])


def test_results_do_not_depend_on_what_else_is_called_with():
    # a token alone, among 16, 17 and 300 gives the same bits: sums are exact, and the epilogue is the same
    x, xs, w, ws = operands(300, 1000, 200, 0, 10)
    bias, residual = others(300, 200, "bf16", 0, 3)
    y = layers.linear8(x, xs, w, ws, bias, residual, layers.ACT_GELU)
    for n in (1, 16, 17, 64):
        assert torch.equal(layers.linear8(x[:n], xs[:n], w, ws, bias, residual[:n], layers.ACT_GELU), y[:n])


def test_entries_beyond_32_bit_offsets():
    ld, rows = (1 << 21) + 16, 2200
    buf = torch.zeros(rows * ld, dtype=torch.int8, device="cuda")
    x = buf.view(rows, ld)[:, :272]
    _, xs, w, ws = operands(rows, 272, 80, 0, 5)
    x.copy_(torch.randint(-127, 128, (rows, 272), device="cuda", generator=generator(3)))
    check(x, xs, w, ws, None, None, "none", layers.linear8(x, xs, w, ws), None)


@pytest.mark.parametrize("tokens", [3, 300])
def test_calls_replay_from_a_captured_graph(tokens):
    x, xs, w, ws = operands(tokens, 1000, 200, 0, 12)
    bias, residual = others(tokens, 200, "f16", 0, 4)
    y, pre = torch.empty(tokens, 200, device="cuda").half(), torch.empty(tokens, 200, device="cuda").half()
    room = torch.empty(layers.linear8_workspace_bytes(tokens, 1000, 200, False) + 256, dtype=torch.uint8, device="cuda")

    def call():
        layers.linear8(x, xs, w, ws, bias, residual, layers.ACT_SILU, pre=pre, out=y, workspace=room)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        x.copy_(torch.randint(-127, 128, x.shape, device="cuda", generator=generator(turn)))
        call()
        torch.cuda.synchronize()
        want = [y.clone(), pre.clone()]
        y.fill_(float("nan")), pre.fill_(float("nan")), room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(pre, want[1])


def test_other_streams_give_the_same_bits():
    x, xs, w, ws = operands(40, 8192, 300, 0, 11)
    want = layers.linear8(x, xs, w, ws)
    torch.cuda.synchronize()
    sides, results = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(3):
        for side in sides:
            with torch.cuda.stream(side):
                results.append(layers.linear8(x, xs, w, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in results)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("name", ACTS)
def test_activations_over_their_range(name, kind):
    # one product a sum: z = 2^-7 (-127 ... 127) times scales that reach from 2^-10 to 2^8, and infinities and NaN
    x = torch.arange(-127, 128, device="cuda", dtype=torch.int16).to(torch.int8)[:, None].contiguous()
    w = torch.full((64, 1), 64, dtype=torch.int8, device="cuda")
    xs, ws = torch.full((255,), 2.0 ** -13, device="cuda"), torch.exp2(torch.linspace(-10, 8, 64, device="cuda"))
    y = layers.linear8(x, xs, w, ws, activation=layers.ACTIVATIONS[name], dtype=TYPES[kind])
    check(x, xs, w, ws, None, None, name, y, None)
    for value in (float("inf"), -float("inf"), float("nan"), 1e30, -1e30):
        bias = torch.full((64,), value, device="cuda").to(TYPES[kind])
        y = layers.linear8(x, xs, w, ws, bias, activation=layers.ACTIVATIONS[name], dtype=TYPES[kind])
        if value != value:
            assert bool(torch.isnan(y).all())
        elif value > 0 or name == "none":
            assert torch.equal(y, bias.expand_as(y))
        else:                                   # 0 from below, or 0 times infinity
            assert bool(((y == 0) | torch.isnan(y)).all())


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(1, 100, 40), (40, 0, 100), (300, 0, 24), (300, 100, 264), (3, 2000, 264)])
def test_scales_bias_and_operands_at_any_alignment(shape, kind):
    # (scales off 16 bytes, a bias off its rows', operands that start at any byte)
    tokens, n_in, n_out = shape
    x, xs, w, ws = operands(*shape, 0, 6)
    bias, residual = others(tokens, n_out, kind, 0, 3)
    want = layers.linear8(x, xs, w, ws, bias, residual, layers.ACT_GELU)
    check(x, xs, w, ws, bias, residual, "gelu", want, None)

    def moved(t, by):
        buf = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
        view = buf[by:].view(t.shape)
        return view.copy_(t)

    for by in (1, 2, 3, 7):
        y = layers.linear8(moved(x, by), moved(xs, by), moved(w, by), moved(ws, by), moved(bias, by), moved(residual, by), layers.ACT_GELU,
                           out=moved(torch.empty_like(want), by))
        assert torch.equal(y, want)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,n_in", [(3, 16), (40, 16), (300, 16), (300, 16384)])
def test_gelu_far_from_zero(tokens, n_in, kind):
    # z is the bias; the header's bounds: 1e-5 of |z| Phi(-|z|) down to -6, 1e-13 beyond (1 + erf has no digits there)
    x, w = (torch.zeros(n, n_in, dtype=torch.int8, device="cuda") for n in (tokens, 520))
    bias = torch.linspace(-12.5, 12.5, 520, device="cuda").to(TYPES[kind])
    y = layers.linear8(x, torch.ones(tokens, device="cuda"), w, torch.ones(520, device="cuda"), bias, activation=layers.ACT_GELU)
    z = bias.double()
    tail = z.abs() * 0.5 * torch.erfc(z.abs() * 0.5 ** 0.5)
    want = z.clamp_min(0.0) - tail
    error = torch.where(z.abs() <= 6, 1e-5 * tail, 1e-13) + U32 * want.abs()
    for row in y:
        within(row, want, error * (1 + ROUND[TYPES[kind]]) + rounded(want, TYPES[kind]), "y")
