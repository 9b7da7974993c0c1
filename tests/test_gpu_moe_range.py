"""ozimmu_moe where values leave the range of 16 bits, or are not finite: each goes where the formula takes it and nowhere else."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_11277_amd import layers
from tests.layers_reference import TYPES, act


def small(tokens, width, hidden, experts, kind, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).to(TYPES[kind])

    return (normal(tokens, width), normal(experts, width, std=width ** -0.5), normal(experts, 2 * hidden, width, std=width ** -0.5),
            normal(experts, width, hidden, std=hidden ** -0.5))


def formula(x, router, w_in, w_out, chosen, gates):
    """y in 64 bits from the choices and gates that the library reports, and the sum of its terms' magnitudes."""
    X, hidden = x.double(), w_out.shape[2]
    Y, size = torch.zeros(x.shape, device="cuda", dtype=torch.float64), torch.zeros(x.shape, device="cuda", dtype=torch.float64)
    for t in range(x.shape[0]):
        for e, g in zip(chosen[t].tolist(), gates[t].double()):
            both = (w_in[e].double() * X[t]).sum(1)
            h = g * act("silu", both[:hidden]) * both[hidden:]
            Y[t] += (w_out[e].double() * h).sum(1)
            size[t] += (w_out[e].double() * h).abs().sum(1)
    return Y, size


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 64, 48, 4, 2), (6, 128, 80, 16, 4), (20, 96, 200, 8, 2), (50, 40, 33, 24, 3), (8, 512, 1024, 64, 8)])
@pytest.mark.parametrize("size", [3e4, 7e4, 3e5, 1e9])
def test_hidden_values_beyond_16_bits(case, kind, size):
    tokens, width, hidden, experts, top_k = case
    x, router, w_in, w_out = small(tokens, width, hidden, experts, kind, 7)
    # a few hidden features are outliers, of about `size` where silu(a) is near a (both rows are scaled), and the output's weights
    # are small enough for the result to fit
    some = torch.arange(hidden, device="cuda") % 7 == 3
    factor = min(size ** 0.5, 3e4)
    w_in[:, :hidden][:, some] *= factor
    w_in[:, hidden:][:, some] *= factor
    w_out *= 2000.0 / size / 8
    y, chosen, gates = layers.moe(x, router, w_in, w_out, top_k)
    want, terms = formula(x, router, w_in, w_out, chosen, gates)
    assert bool(torch.isfinite(y).all())
    # both products' sums in 32 bits (an outlier is the product of two sums, each off by at most (width + 8) 2^-24 of its terms'
    # magnitudes, which for random rows is several times its own size) and one rounding
    u = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}[kind]
    off = (y.double() - want).abs()
    assert bool((off <= u * want.abs() + 2e-5 * terms.amax(1, keepdim=True) + 2.0 ** -24).all()), float((off / terms).max())


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("case", [(6, 96, 64, 12, 2), (40, 130, 100, 16, 3), (8, 512, 1024, 64, 8)])
def test_an_expert_s_weights_reach_only_those_who_chose_it(case, bad, kind):
    tokens, width, hidden, experts, top_k = case
    x, router, w_in, w_out = small(tokens, width, hidden, experts, kind, 8)
    y, chosen, gates = layers.moe(x, router, w_in, w_out, top_k)
    count = torch.zeros(experts, dtype=torch.long, device="cuda").index_add_(0, chosen.flatten().long(), torch.ones_like(chosen.flatten()).long())
    expert = int(((count > 0) & (count < tokens)).nonzero()[0])
    takes = (chosen == expert).any(1)
    rows = torch.arange(width, device="cuda") % 5 == 2            # output features that have the bad weight
    w_out[expert, rows, hidden // 3] = bad
    got, _, _ = layers.moe(x, router, w_in, w_out, top_k)
    assert torch.equal(got[~takes], y[~takes])
    assert torch.equal(got[takes][:, ~rows], y[takes][:, ~rows])
    # the rest: a NaN, or an infinity of the sign of its hidden value (which is not 0)
    want, _ = formula(x, router, w_in, w_out, chosen, gates)
    there = got[takes][:, rows].double()
    assert torch.equal(torch.nan_to_num(there, nan=7.0), torch.nan_to_num(want[takes][:, rows], nan=7.0))
    assert not torch.isfinite(there).any()


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_hidden_values_that_are_not_finite_stay_their_token_s(kind):
    tokens, width, hidden, experts, top_k = 9, 64, 40, 6, 2
    x, router, w_in, w_out = small(tokens, width, hidden, experts, kind, 9)
    y, chosen, gates = layers.moe(x, router, w_in, w_out, top_k)
    expert = int(chosen[0, 0])
    w_in[expert, hidden + 5, 0] = float("inf")                    # an up row: h is an infinity for every token of this expert
    got, _, _ = layers.moe(x, router, w_in, w_out, top_k)
    takes = (chosen == expert).any(1)
    want, _ = formula(x, router, w_in, w_out, chosen, gates)
    assert torch.equal(got[~takes], y[~takes])
    assert torch.equal(got[takes].isnan(), want[takes].isnan()) and torch.equal(got[takes].isinf(), want[takes].isinf())
    assert torch.equal(torch.sign(got[takes].double()), torch.sign(want[takes]))
    router[expert] = float("nan")                                 # every token takes it, with a NaN for its gate
    got, chosen, gates = layers.moe(x, router, w_in, w_out, top_k)
    assert bool((chosen == expert).any(1).all()) and bool(got.isnan().all())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("case", [(40, 64, 32, 4), (8, 200, 24, 6), (3, 512, 48, 5)])
def test_the_hidden_layer_is_not_rounded_to_16_bits(case, kind):
    # tokens with one entry, a 1, that choose one expert, whose gate is 1: the hidden layer's sums are exact, and of the result's error
    # there is left what the activation has, the second product's sums in 32 bits, h's two numbers, and one rounding
    tokens, width, hidden, experts = case
    x, router, w_in, w_out = small(tokens, width, hidden, experts, kind, 10)
    w_in *= width ** 0.5
    x.zero_()
    x[torch.arange(tokens), torch.arange(tokens) * 7 % width] = 1.0
    y, chosen, gates = layers.moe(x, router, w_in, w_out, 1)
    assert bool((gates == 1).all())
    both = torch.stack([w_in[e].double()[:, t * 7 % width] for t, e in enumerate(chosen[:, 0].tolist())])
    a, b = both[:, :hidden], both[:, hidden:]
    s, W = act("silu", a), w_out[chosen[:, 0].long()].double()
    h = s * b
    # (a number of p bits is off by up to 2^-p of itself, two of them by 2^-2p)
    u32, least, part = 2.0 ** -24, *{"bf16": (0.0, 2.0 ** -16), "f16": (2.0 ** -25, 2.0 ** -22)}[kind]
    hb = 16 * u32 * (s.abs() + a.abs() * (1 + a.abs())) * b.abs() + 4 * u32 * h.abs() + part * h.abs() + least

    def product(v):
        return torch.matmul(W, v.unsqueeze(2)).squeeze(2)

    want, size = product(h), torch.matmul(W.abs(), h.abs().unsqueeze(2)).squeeze(2)
    bound = size * ((2 * hidden + 8) * u32) + torch.matmul(W.abs(), hb.unsqueeze(2)).squeeze(2)
    least, most = (want - bound).to(TYPES[kind]), (want + bound).to(TYPES[kind])       # what rounding once can make of it
    assert bool(((y >= least) & (y <= most)).all())
    # ... which one number of 16 bits would not keep to
    once = product(h.to(TYPES[kind]).double()).to(TYPES[kind])
    assert int(((once < least) | (once > most)).sum()) > want.numel() // 100
