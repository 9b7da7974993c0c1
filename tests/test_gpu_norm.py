"""ozimmu_rms_norm, its results in 8 bits and its gradients, and ozimmu_quantise: against 64-bit forms, codes bit for bit."""
import itertools

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.eight_reference import codes_of, codes_untouched, depth, guarded_codes, norm, root_error
from tests.layers_reference import TYPES, U32, guarded, rounded, untouched, within

EPS = 1e-5
# (tokens, width): a row of a wavefront, of a work-group, of more than registers hold; ends inside a group of 8 and inside a wavefront
SIZES = [(1, 1), (5, 2), (3, 7), (4, 8), (9, 9), (1, 64), (70, 65), (6, 511), (1, 512), (7, 513), (300, 1000), (3, 1024), (2, 1025), (33, 2048),
         (1, 2049), (5, 4095), (1, 4096), (3, 4104), (1, 8192), (2, 8200), (3, 16384), (2, 16385), (1, 20001), (2, 70000), (0, 16), (3, 0),
         (2050, 1201), (8195, 1536), (2051, 1544), (8200, 2047), (3, 6144), (3, 6150), (2, 9001), (3, 12288), (2, 12300), (2, 24577), (3, 32768), (2, 32776), (257, 2100), (300, 4096)]


def values(shape, kind, seed, std=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(TYPES[kind])


def place(x, extra):
    return guarded(*x.shape, x.shape[1] + extra, x.dtype, x)[0] if x.shape[1] + extra else x


def check_scale(scale, want, error):
    want = want.to(scale.device)
    assert torch.equal(torch.isnan(scale), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert bool(((scale.double() - want).abs() <= error * want.abs() + 2.0 ** -149)[fine].all())


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,width", SIZES)
def test_norm(tokens, width, kind, extra):
    x, res = (place(values((tokens, width), kind, 11 * tokens + width + i, 1.5), extra) for i in (0, 1))
    weight = values((width,), kind, 3, 0.7)
    print(tokens, width, kind, extra, flush=True)
    for residual, w in itertools.product((None, res), (None, weight)):
        h = x.double() if residual is None else x.double() + residual.double()
        h32 = x.float() if residual is None else x.float() + residual.float()
        r, y = norm(h, w, EPS)
        (out, obuf), (total, tbuf) = (guarded(tokens, width, width + extra, x.dtype) if width else (torch.empty_like(x), None) for _ in range(2))
        got, kept = layers.rms_norm(x, w, residual, EPS, total=total, out=out)
        codes, cbuf = guarded_codes(tokens, width, width + extra) if width else (torch.empty((tokens, 0), dtype=torch.int8, device="cuda"), None)
        got8, scale, kept8 = layers.rms_norm8(x, w, residual, EPS, out=codes)
        torch.cuda.synchronize()
        assert got is out and kept is total and got8 is codes
        within(out, y, y.abs() * (root_error(width) + 4 * U32) + rounded(y, x.dtype), "y")
        within(total, h, rounded(h, x.dtype) + U32 * h.abs(), "total")
        assert torch.equal(kept8, total) if residual is not None else kept8 is x
        want, top = codes_of(h32 if w is None else h32 * w.float())
        assert torch.equal(got8.cpu(), want)
        check_scale(scale, top * r[:, 0].cpu() if width else top, root_error(width) + 4 * U32)
        if width:
            assert untouched(out, obuf) and untouched(total, tbuf) and codes_untouched(codes, cbuf)


@pytest.mark.parametrize("extra", [0, 16, 5])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantise(rows, cols, kind, extra):
    x = place(values((rows, cols), kind, rows + cols, 0.02), extra)
    codes, buf = guarded_codes(rows, cols, cols + extra) if cols else (None, None)
    print(rows, cols, kind, extra, flush=True)
    got, scale = layers.quantise(x, out=codes)
    again = layers.quantise(x)
    torch.cuda.synchronize()
    want, top = codes_of(x.float())
    assert torch.equal(got.cpu(), want) and torch.equal(again[0], got) and torch.equal(again[1], scale)
    check_scale(scale, top, 2 * U32)
    assert not cols or codes_untouched(got, buf)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", [24, 600, 3000, 20000])
def test_ties_go_to_the_even_code(width, kind):
    # a row whose largest magnitude is 127: codes are the values themselves, rounded
    x = (torch.arange(width, device="cuda") % 508 - 254).float() * 0.5
    x = torch.stack((x, -x)).to(TYPES[kind])
    codes, scale = layers.quantise(x)
    assert torch.equal(codes.float(), torch.round(x.float())) and bool((scale == 1.0).all())


def special_rows(kind, width):
    top = torch.finfo(TYPES[kind]).max
    x = values((12, width), kind, 5)
    x[1] = 0
    x[2, width // 2] = float("nan")
    x[3, width - 1] = float("inf")
    x[4, 0] = -float("inf")
    x[5] = x[5] * 0 + top                          # squares that leave the range of 32 bits (not in float16)
    x[6, 1] = -top
    x[7] = x[7].float().mul(2.0 ** -14 if kind == "f16" else 2.0 ** -110).to(x.dtype)
    x[8] = 0
    x[8, 3] = torch.finfo(TYPES[kind]).tiny
    x[9] = torch.where(x[9] > 0, top / 4, -top / 8).to(x.dtype)
    x[10, 0], x[10, 1] = float("inf"), float("nan")
    return x


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", [24, 600, 3000, 20000])
def test_rows_that_are_not_ordinary(width, kind):
    x = special_rows(kind, width)
    weight = values((width,), kind, 9, 0.5)
    codes, scale = layers.quantise(x)
    want, top = codes_of(x.float())
    assert torch.equal(codes.cpu(), want)
    check_scale(scale, top, 2 * U32)

    y, _ = layers.rms_norm(x, weight, eps=EPS)
    codes, scale, _ = layers.rms_norm8(x, weight, eps=EPS)
    r, exact = norm(x, weight, EPS)
    fine = torch.isfinite(x).all(1)
    assert bool(torch.isfinite(y[fine]).all()) and bool(torch.isfinite(scale[fine]).all())
    error = root_error(width) + 4 * U32
    # (h w is rounded in 32 bits before it is multiplied by r: by up to 2^-150 where it is below the normal numbers, which r, here up to
    # 1 / sqrt(EPS), makes r 2^-150 of y)
    within(y[fine], exact[fine], exact[fine].abs() * error + rounded(exact[fine], x.dtype) + r[fine] * 2.0 ** -150, "y")
    # the values that codes stand for: half a code off at most, or rows that are held as zeros
    held = codes.double() * scale.double()[:, None]
    most = exact.abs().amax(1, keepdim=True)
    tiny = (x.double() * weight.double()).abs().amax(1, keepdim=True) < 2.0 ** -100
    assert torch.equal(scale[fine] == 0, tiny[fine, 0])
    within(held[fine], torch.where(tiny, 0.0, exact)[fine], (most * (0.5 / 127 * (1 + 2 ** -16) + error + 4 * U32)).expand_as(exact)[fine], "8 bits")
    # what is not finite: a NaN takes its row, an infinity itself (and r, so that the others are 0)
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(scale[[2, 3, 4, 10]]).all()) and bool((codes[[2, 3, 4, 10]] == 0).all())
    for row, at in ((3, width - 1), (4, 0)):
        others = torch.ones(width, dtype=torch.bool, device="cuda")
        others[at] = False
        assert bool(torch.isnan(y[row, at])) and bool((y[row, others] == 0).all())


def test_a_total_beyond_its_type():
    # (float16: the sum is beyond 65504, which its total cannot hold; y goes by the sum itself)
    x = torch.full((2, 96), 60000.0, dtype=torch.float16, device="cuda")
    y, total = layers.rms_norm(x, None, x.clone(), EPS)
    assert bool(torch.isinf(total).all()) and bool((y == 1).all())


@pytest.mark.parametrize("width", [100, 1500, 20000])
def test_total_in_place(width):
    x, res, weight = values((9, width), "bf16", 1), values((9, width), "bf16", 2), values((width,), "bf16", 3)
    codes, scale, total = layers.rms_norm8(x, weight, res)
    y, _ = layers.rms_norm(x, weight, res)
    for place_of in (0, 1):
        a, b = x.clone(), res.clone()
        stream = (a, b)[place_of]
        got = layers.rms_norm8(a, weight, b, total=stream)
        assert got[2] is stream and all(torch.equal(p, q) for p, q in zip(got, (codes, scale, total)))
        a, b = x.clone(), res.clone()
        assert torch.equal(layers.rms_norm(a, weight, b, total=(a, b)[place_of])[0], y)


def grad_reference(dy, h, weight, add, eps):
    r, _ = norm(h, None, eps)
    dy, n = dy.double(), h.double() * r
    g = dy if weight is None else dy * weight.double()
    m = (g * n).mean(1, keepdim=True)
    dx = r * (g - n * m) + (0.0 if add is None else add.double())
    return r, g, n, dx, (dy * n).sum(0), (dy * n).abs().sum(0)


def check_grad(dx, dw, dy, h, weight, add, eps=EPS):
    tokens, width = h.shape
    r, g, n, want_dx, want_dw, size_dw = grad_reference(dy, h, weight, add, eps)
    # r (g - n m): r twice and m's own (the sum's depth, g, n and r in it), products and differences one each
    error = 3 * root_error(width) + (depth(width) + 12) * U32
    size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    if dx is not None:
        within(dx, want_dx, size * error + U32 * want_dx.abs() + rounded(want_dx, h.dtype), "dx")
    if dw is not None:
        within(dw, want_dw, size_dw * (root_error(width) + (tokens + 24) * U32) + rounded(want_dw, h.dtype), "dw")


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,width", SIZES + [(1500, 24), (5000, 1), (2100, 1024), (1100, 2056), (70, 20000)])
def test_norm_gradients(tokens, width, kind, extra):
    h, dy, add = (place(values((tokens, width), kind, 7 * tokens + width + i), extra) for i in range(3))
    weight = values((width,), kind, 3, 0.7)
    print(tokens, width, kind, extra, flush=True)
    for w, more in itertools.product((None, weight), (None, add)):
        dx, dbuf = guarded(tokens, width, width + extra, h.dtype) if width else (torch.empty_like(h), None)
        dw, wbuf = guarded(1, width, width + extra, h.dtype) if width else (h.new_empty((1, 0)), None)
        got = layers.rms_norm_grad(dy, h, w, EPS, add=more, dx=dx, dw=dw[0])
        only_dx, none = layers.rms_norm_grad(dy, h, w, EPS, add=more, want=("dx",))
        nothing, only_dw = layers.rms_norm_grad(dy, h, w, EPS, add=more, want=("dw",))
        torch.cuda.synchronize()
        check_grad(*got, dy, h, w, more)
        assert none is None and nothing is None and torch.equal(only_dx, dx) and torch.equal(only_dw, dw[0])
        if width:
            assert untouched(dx, dbuf) and untouched(dw, wbuf)


@pytest.mark.parametrize("width", [40, 700, 3000, 20000])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_gradients_of_large_rows(width, kind):
    # rows whose squares leave the range of 32 bits beside ordinary ones; dx of theirs is below the least number, dw is ordinary
    top = torch.finfo(TYPES[kind]).max
    h, dy, weight = values((7, width), kind, 1), values((7, width), kind, 2), values((width,), kind, 3)
    h[2] = torch.where(h[2] > 0, top / 2, -top / 4).to(h.dtype)
    h[5] = h[5].float().mul(2.0 ** 80).to(h.dtype)
    check_grad(*layers.rms_norm_grad(dy, h, weight, EPS), dy, h, weight, None)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("width", [40, 3000, 20000])
def test_gradients_of_zeros_and_tiny_rows(width, kind):
    h, dy, weight = values((6, width), kind, 1), values((6, width), kind, 2), values((width,), kind, 3)
    h[1], h[4] = 0, h[4].float().mul(1e-30).to(h.dtype)
    check_grad(*layers.rms_norm_grad(dy, h, weight, EPS), dy, h, weight, None)


@pytest.mark.parametrize("width", [40, 700, 3000, 20000])
def test_gradients_in_place(width):
    h, dy, add = (values((70, width), "bf16", i) for i in range(3))
    weight = values((width,), "bf16", 3)
    dx, dw = layers.rms_norm_grad(dy, h, weight, EPS, add=add)
    for i in range(3):
        given = [dy.clone(), h.clone(), add.clone()]
        got = layers.rms_norm_grad(given[0], given[1], weight, EPS, add=given[2], dx=given[i])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


@pytest.mark.parametrize("width", [5, 300])
def test_gradients_against_differences(width):
    # central differences of the norm in 64 bits, of the function that the kernel's outputs are the gradients of
    h, dy, weight = values((3, width), "f32", 1), values((3, width), "f32", 2), values((width,), "f32", 3)
    dx, dw = layers.rms_norm_grad(dy, h, weight, EPS)
    step = 2.0 ** -14

    def loss(h, w):
        return (norm(h, w, EPS)[1] * dy.double()).sum()

    for at in ((0, 0), (1, width // 2), (2, width - 1)):
        e = torch.zeros_like(h, dtype=torch.float64)
        e[at] = step
        slope = (loss(h.double() + e, weight) - loss(h.double() - e, weight)) / (2 * step)
        # the third derivative's part, step^2, and 32 bits
        assert abs(float(slope - dx[at])) <= 1e-5 * float(dy.abs().max()) * 4
        e = torch.zeros(width, dtype=torch.float64, device="cuda")
        e[at[1]] = 1.0
        slope = loss(h, weight.double() + e) - loss(h, weight)
        assert abs(float(slope - dw[at[1]])) <= 1e-5 * 4 * float(dy.abs().max())


def test_calls_in_a_graph_and_on_two_streams():
    x, res, weight = values((70, 1500), "bf16", 1), values((70, 1500), "bf16", 2), values((1500,), "bf16", 3)
    total, codes, scale = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(70, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(weight)
    ws = torch.empty(layers.rms_norm_grad_workspace_bytes(70, 1500), dtype=torch.uint8, device="cuda")

    def both():
        layers.rms_norm8(x, weight, res, total=total, out=codes, scale=scale)
        layers.rms_norm_grad(x, total, weight, add=res, dx=dx, dw=dw, workspace=ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(4):
        x.copy_(values(x.shape, "bf16", 20 + turn))
        for t in (total, codes, scale, dx, dw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (total, codes, scale, dx, dw)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (total, codes, scale, dx, dw)))
    streams, results = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(layers.rms_norm_grad(x, total, weight, add=res))
    torch.cuda.synchronize()
    assert all(torch.equal(a, dx) and torch.equal(b, dw) for a, b in results)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", [100, 2056, 20000])
def test_tensors_at_any_alignment(width, kind):
    x, res, dy = (values((5, width), kind, i) for i in range(3))
    weight = values((width,), kind, 3)
    want = layers.rms_norm8(x, weight, res) + layers.rms_norm(x, weight, res)[:1] + layers.rms_norm_grad(dy, x, weight, add=res)

    def moved(t, by):
        view = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")[by:].view(t.shape)
        return view.copy_(t)

    for by in (1, 3):
        a, b, d, w = (moved(t, by) for t in (x, res, dy, weight))
        empty = [moved(torch.empty_like(t), by) for t in want]
        got = layers.rms_norm8(a, w, b, out=empty[0], scale=empty[1], total=empty[2]) + layers.rms_norm(a, w, b, out=empty[3])[:1]
        got = got + layers.rms_norm_grad(d, a, w, add=b, dx=empty[4], dw=empty[5])
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_one_tensor_for_several_arguments():
    # x that is its own residual, dy that is h: inputs may be the same
    x, weight = values((9, 300), "bf16", 1), values((300,), "bf16", 3)
    assert all(torch.equal(a, b) for a, b in zip(layers.rms_norm8(x, weight, x), layers.rms_norm8(x, weight, x.clone())))
    assert all(torch.equal(a, b) for a, b in zip(layers.rms_norm_grad(x, x, weight, add=x), layers.rms_norm_grad(x, x.clone(), weight, add=x.clone())))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("width", [24, 600, 3000, 20000])
def test_norms_of_large_and_small_weights(width, kind):
    # h weight may leave the range of 32 bits where h r weight does not
    for size, gain in ((1e12, 1e30), (1e20, 1e-36), (1e-3, 1e-36), (1.0, 1e37)):
        x, weight = values((3, width), kind, 1).float().mul(size).to(TYPES[kind]), values((width,), kind, 3).float().mul(gain).to(TYPES[kind])
        r, want = norm(x, weight, EPS)
        y, _ = layers.rms_norm(x, weight, eps=EPS)
        within(y, want, want.abs() * (root_error(width) + 4 * U32) + rounded(want, x.dtype) + 2.0 ** -150, "y")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("width", [24, 600, 3000, 20000])
def test_an_eps_beside_squares_beyond_32_bits(width, kind):
    # the sum of the squares, or their mean with eps, leaves the range
    for size, eps in ((2e19, 3e38), (1e18, 3.4e38), (1e19, 3.4e38), (1e25, 3e38)):
        h, dy, weight = (values(s, kind, i) for i, s in enumerate(((3, width), (3, width), (width,))))
        h = h.float().clamp(-2.0, 2.0).mul(size).to(h.dtype)
        r, want = norm(h, weight, eps)
        y, _ = layers.rms_norm(h, weight, eps=eps)
        within(y, want, want.abs() * (root_error(width) + 4 * U32) + rounded(want, h.dtype), "y")
        codes, scale, _ = layers.rms_norm8(h, weight, eps=eps)
        check_scale(scale, ((h.double() * weight.double()).abs().amax(1) * r[:, 0] / 127).cpu(), root_error(width) + 4 * U32)
        check_grad(*layers.rms_norm_grad(dy, h, weight, eps), dy, h, weight, None, eps)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,width", [(1, 1), (5, 7), (300, 1000), (9, 2100), (3, 9001), (2, 20001)])
def test_the_norm_and_its_8_bits_in_one_call(tokens, width, kind):
    x, res, weight = values((tokens, width), kind, 1), values((tokens, width), kind, 2), values((width,), kind, 3)
    want = layers.rms_norm(x, weight, res, EPS) + layers.rms_norm8(x, weight, res, EPS)[:2]
    got = [torch.zeros_like(t) for t in want]
    y, total, codes, scale = (t.data_ptr() for t in got)
    assert layers.lib().ozimmu_rms_norm(tokens, width, layers._TYPES[x.dtype], x.data_ptr(), width, res.data_ptr(), width, weight.data_ptr(), EPS, total, width,
                                        y, width, codes, width, scale, torch.cuda.current_stream().cuda_stream) == layers.OK
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
