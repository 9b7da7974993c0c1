"""ozimmu_adamw against the formulas in 64 bits: moments in 32 and in 8 bits, every alignment, lists of many tensors."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.layers_reference import ROUND, TYPES, U32, rounded, within

HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.02)
SIZES = [1, 2, 255, 256, 257, 1000, 4096, 5000, 70001]


def step64(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay):
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps)
    return p - lr * weight_decay * p - lr * update, m, v, lr * update


def values(n, kind, std, gen, offset=0):
    """n values that start `offset` entries behind an aligned address."""
    return torch.randn(n + offset, device="cuda", generator=gen).mul_(std).to(TYPES[kind])[offset:]


def decoded(codes, scale):
    x = codes.double().view(-1)
    return x * scale.double().repeat_interleave(256)[:x.numel()]


@pytest.mark.parametrize("param,grad,copy", [("f32", "f32", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", None),
                                             ("f16", "f32", None)])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_moments_in_32_bits(param, grad, copy, offset):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    ps, gs = [values(n, param, 0.05, gen, offset) for n in SIZES], [values(n, grad, 1e-2, gen, offset) for n in SIZES]
    ms, vs = [values(n, "f32", 1e-2, gen, offset) for n in SIZES], [values(n, "f32", 1e-4, gen, offset).abs() for n in SIZES]
    copies = [values(n, copy, 1.0, gen, offset) for n in SIZES] if copy else None
    before = [[t.double().clone() for t in x] for x in (ps, gs, ms, vs)]
    layers.AdamW(ps, ms, vs, copies=copies).step(gs, 3, **HYPER)
    torch.cuda.synchronize()
    for i in range(len(SIZES)):
        p, m, v, update = step64(*(b[i] for b in before), 3, **HYPER)
        # at most four operations with constants rounded to 32 bits for m and v, a dozen for p; m cancels
        mb = 6 * U32 * (0.9 * before[2][i].abs() + 0.1 * before[1][i].abs())
        within(ms[i], m, mb, "m")
        within(vs[i], v, 8 * U32 * v + 2.0 ** -148, "v")
        root = (v / (1 - 0.999 ** 3)).sqrt() + 1e-8
        pb = 8 * U32 * p.abs() + 20 * U32 * update.abs() + HYPER["lr"] / (1 - 0.9 ** 3) * mb / root
        within(ps[i], p, pb + (rounded(p, ps[i].dtype) + ROUND[ps[i].dtype] * pb if param != "f32" else 0), "p")
        if copies:
            within(copies[i], ps[i].double(), rounded(ps[i].double(), copies[i].dtype), "copy")


@pytest.mark.parametrize("param,grad,copy", [("f32", "bf16", "bf16"), ("bf16", "bf16", None), ("f16", "f16", None)])
@pytest.mark.parametrize("offset", [0, 1])
def test_moments_in_8_bits(param, grad, copy, offset):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    ps = [values(n, param, 0.05, gen, offset) for n in SIZES]
    ms, vs, msc, vsc = layers.adamw_state(ps, bits=8)
    copies = [values(n, copy, 1.0, gen, offset) for n in SIZES] if copy else None
    plan = layers.AdamW(ps, ms, vs, msc, vsc, copies)
    for step in range(1, 5):
        gs = [values(n, grad, 10.0 ** -step, gen, offset) for n in SIZES]
        old = [(p.double().clone(), decoded(m, a).clone(), decoded(v, b).clone()) for p, m, v, a, b in zip(ps, ms, vs, msc, vsc)]
        plan.step(gs, step, seed=17 * step, **HYPER)
        torch.cuda.synchronize()
        for i, (p0, m0, r0) in enumerate(old):
            p, m, v, update = step64(p0, gs[i].double().view(-1), m0, r0 * r0, step, **HYPER)
            mb = 8 * U32 * (0.9 * m0.abs() + 0.1 * gs[i].double().abs())
            root = (v / (1 - 0.999 ** step)).sqrt() + 1e-8
            pb = 8 * U32 * p.abs() + 24 * U32 * update.abs() + HYPER["lr"] / (1 - 0.9 ** step) * mb / root
            within(ps[i], p, pb + (rounded(p, ps[i].dtype) + ROUND[ps[i].dtype] * pb if param != "f32" else 0), "p")
            for what, x, codes, scale in (("m", m, ms[i], msc[i]), ("v", v.sqrt(), vs[i], vsc[i])):
                blocks = torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)
                top = blocks.abs().amax(1)
                within(scale, top / 448.0, 12 * U32 * (top / 448.0) + (mb.max() / 448.0 if what == "m" else 0) + 2.0 ** -148, what + " scale")
                # never further from its value than a unit of e4m3 there (less than an eighth of it, 2^-9 of the scale below 2^-6)
                full = scale.double().repeat_interleave(256)[:x.numel()]
                unit = torch.maximum(x.abs() / 8, full * 2.0 ** -9)
                within(decoded(codes, scale), x, unit * (1 + 1e-5) + (mb if what == "m" else 0), what)
                assert bool(((decoded(codes, scale) == 0) <= ((x == 0) | (what == "m"))).all())


def test_8_bit_rounding_is_right_in_the_mean_and_set_by_the_seed():
    # 0.999 v + 0.001 g^2 moves v by far less than a unit: to nearest it would stand still
    n, steps = 1 << 16, 200
    p = [torch.zeros(n, device="cuda")]
    m, v, ms, vs = layers.adamw_state(p, bits=8)
    g = [torch.full((n,), 1e-2, device="cuda")]
    g[0][::256] = 2e-2                       # a block's largest values, which set its scale
    plan = layers.AdamW(p, m, v, ms, vs)
    for step in range(1, steps + 1):
        plan.step(g, step, lr=0.0, weight_decay=0.0, beta1=0.9, beta2=0.99, seed=step)
    rest = torch.arange(n, device="cuda") % 256 != 0
    root = decoded(v[0], vs[0])[rest]
    want = 1e-2 * math.sqrt(1 - 0.99 ** steps)
    # a root moves between neighbours a tenth of it apart at most; its mean over 65280 values stays within 2 %, the
    # spread of one (0.1 of it) over 255 and the second-order effect of averaging squares
    assert abs(float(root.mean()) / want - 1) < 0.02
    mean = decoded(m[0], ms[0])[rest]
    assert abs(float(mean.mean()) / 1e-2 - 1) < 0.005

    def codes(seed):
        p = [torch.zeros(4096, device="cuda")]
        state = layers.adamw_state(p, bits=8)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        layers.AdamW(p, *state).step([torch.randn(4096, device="cuda", generator=gen)], 1, seed=seed)
        return state[0][0].view(torch.uint8), state[1][0].view(torch.uint8)

    a, b, c = codes(1), codes(1), codes(2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not torch.equal(a[0], c[0]) and not torch.equal(a[1], c[1])


def test_more_tensors_than_a_launch_takes_of_mixed_types():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    n = 130
    kinds = ["f32" if i < 100 else "bf16" for i in range(n)]
    ps = [values(1 + 37 * i % 3001, k, 0.1, gen) for i, k in enumerate(kinds)]
    ps[50] = torch.empty(0, device="cuda")
    gs = [values(p.numel(), "f16" if i % 70 == 69 else "f32", 0.1, gen) for i, p in enumerate(ps)]
    before = [p.double().clone() for p in ps]
    m, v, _, _ = layers.adamw_state(ps)
    layers.AdamW(ps, m, v).step(gs, 1, **HYPER)
    torch.cuda.synchronize()
    for p, b, g in zip(ps, before, gs):
        zero = torch.zeros_like(b)
        want, _, _, update = step64(b, g.double(), zero, zero, 1, **HYPER)
        bound = 8 * U32 * want.abs() + 40 * U32 * update.abs()
        within(p, want, bound + (rounded(want, p.dtype) + ROUND[p.dtype] * bound if p.dtype != torch.float32 else 0), "p")


def test_a_step_in_parts_and_the_whole_step_agree():
    # the words that round 8-bit moments go by the place in the list: the same list gives the same bits on another stream
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    ps = [values(n, "bf16", 0.1, gen) for n in SIZES]
    gs = [values(n, "bf16", 0.1, gen) for n in SIZES]
    results = []
    for side in (False, True):
        p = [x.clone() for x in ps]
        state = layers.adamw_state(p, bits=8)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream() if side else torch.cuda.current_stream()):
            layers.AdamW(p, *state).step(gs, 1, seed=9)
        torch.cuda.synchronize()
        results.append([x.view(torch.uint8).clone() if x.dtype == torch.float8_e4m3fn else x.clone() for x in p + state[0] + state[1] + state[2] + state[3]])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("bits", [8, 32])
def test_non_finite_gradients_stay_where_they_are(bits):
    p = [torch.ones(700, device="cuda")]
    state = layers.adamw_state(p, bits=bits)
    g = [torch.full((700,), 0.25, device="cuda")]
    g[0][5], g[0][300] = float("nan"), float("inf")
    plan = layers.AdamW(p, *state)
    plan.step(g, 1, lr=1e-2)
    plan.step([torch.full((700,), 0.25, device="cuda")], 2, lr=1e-2)
    bad = torch.isnan(p[0])
    assert bad[5] and bad[300] and int(bad.sum()) == 2
    rest = ~bad
    assert bool(torch.isfinite(state[0][0].float()[rest]).all()) and bool(torch.isfinite(state[1][0].float()[rest]).all())


def test_zero_and_tiny_gradients_in_8_bits():
    p = [torch.ones(1024, device="cuda")]
    state = layers.adamw_state(p, bits=8)
    plan = layers.AdamW(p, *state)
    plan.step([torch.zeros(1024, device="cuda")], 1, weight_decay=0.0)
    assert bool((p[0] == 1).all()) and not state[0][0].float().any() and not state[1][0].float().any()
    plan.step([torch.full((1024,), 1e-38, device="cuda")], 2, weight_decay=0.0)
    assert bool(torch.isfinite(p[0]).all()) and bool(torch.isfinite(state[1][0].float()).all())


def test_a_step_replays_from_a_captured_graph():
    p = [torch.ones(5000, device="cuda"), torch.ones(77, device="cuda")]
    g = [torch.full_like(x, 0.5) for x in p]
    state = layers.adamw_state(p)
    plan = layers.AdamW(p, *state)
    plan.step(g, 1)
    torch.cuda.synchronize()
    start = [x.clone() for x in p + state[0] + state[1]]
    plan.step(g, 2)
    torch.cuda.synchronize()
    want = [x.clone() for x in p + state[0] + state[1]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.step(g, 2)
    for _ in range(3):
        for x, s in zip(p + state[0] + state[1], start):
            x.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p + state[0] + state[1], want))


def test_the_plan_refuses_what_does_not_fit():
    p = [torch.zeros(300, device="cuda")]
    m, v, ms, vs = layers.adamw_state(p, bits=8)
    m32, v32, _, _ = layers.adamw_state(p)
    for make in (lambda: layers.AdamW(p, m, v), lambda: layers.AdamW(p, m, v32, ms, vs), lambda: layers.AdamW(p, m32, []),
                 lambda: layers.AdamW(p, m32, [torch.zeros(299, device="cuda")]), lambda: layers.AdamW([p[0].double()], m32, v32),
                 lambda: layers.AdamW(p, m, v, [ms[0][:1]], vs), lambda: layers.AdamW(p, m32, v32, copies=[torch.zeros(300, device="cuda")]),
                 lambda: layers.AdamW([torch.zeros(600, device="cuda")[::2]], m32, v32)):
        with pytest.raises(ValueError):
            make()
    plan = layers.AdamW(p, m32, v32)
    for grads in ([], [torch.zeros(299, device="cuda")], [torch.zeros(300)], [torch.zeros(600, device="cuda")[::2]], [torch.zeros(300, device="cuda").double()]):
        with pytest.raises(ValueError):
            plan.step(grads, 1)
    with pytest.raises(layers.OzimmuError):
        plan.step([torch.zeros(300, device="cuda")], 0)
