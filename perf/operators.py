"""Performance cases of the feed-forward operators: a linear layer with its epilogue, that layer's gradients, the AdamW
step that uses them, and the mixture-of-experts layer that a serving loop runs on a few tokens.

With `own` false a pass is the operator's plain form (elementary torch operations in 32 bits, rounded once at the end),
otherwise the calls a program makes of `paper_2506_11277_amd.layers`.  Both take the same tensors.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_BLOCK = 256                      # values that share a scale where AdamW's states are held in 8 bits
_BETA1, _BETA2, _EPS, _LR, _DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01


def listed():
    return [
        # one token in a serving loop through a narrow layer: what a call costs
        dict(name="linear_token", op="linear", type="bf16", tokens=1, n_in=1024, n_out=4096, act="gelu_tanh", bias=True,
             residual=False, pre=False, ld=0),
        # a batch of sequences decoded together, back to the width of the residual stream that it is added to
        dict(name="linear_decode", op="linear", type="bf16", tokens=48, n_in=8192, n_out=2048, act="none", bias=False,
             residual=True, pre=False, ld=0),
        # sizes that fit no tile and rows that start off 16 bytes, everything in the epilogue
        dict(name="linear_ragged", op="linear", type="f16", tokens=1531, n_in=1001, n_out=777, act="relu", bias=True,
             residual=True, pre=False, ld=0),
        # the wide layer of a training step: the values before the activation are kept for the gradients
        dict(name="linear_wide", op="linear", type="bf16", tokens=8192, n_in=4096, n_out=8192, act="gelu", bias=True,
             residual=False, pre=True, ld=0),
        # gradients of a small layer in 32 bits
        dict(name="grad_small", op="grad", type="f32", tokens=500, n_in=512, n_out=384, act="silu", bias=True, ld=0),
        # gradients at an ordinary width, inputs that are columns of a wider matrix
        dict(name="grad_1024", op="grad", type="f16", tokens=1777, n_in=1024, n_out=2304, act="relu", bias=True, ld=64),
        # gradients of the wide layer of a training step
        dict(name="grad_wide", op="grad", type="bf16", tokens=8192, n_in=4096, n_out=8192, act="gelu", bias=True, ld=0),
        # a small model's tensors, most of them a few thousand values: launches count
        dict(name="adamw_small", op="adamw", tensors=90, least=64, most=1 << 16, param="f32", grad="f32", bits=32,
             copy=False),
        # 32-bit weights and states, 16-bit gradients, and the 16-bit weights for the next step written along
        dict(name="adamw_copy", op="adamw", tensors=24, least=1000, most=1 << 24, param="f32", grad="bf16", bits=32,
             copy=True),
        # large tensors with the states in 8 bits
        dict(name="adamw_8bit", op="adamw", tensors=40, least=1000, most=1 << 25, param="bf16", grad="bf16", bits=8,
             copy=False),
        # one token through a layer of few experts
        dict(name="moe_token", op="moe", type="bf16", tokens=1, width=1024, hidden=704, experts=16, top_k=2, norm=True),
        # eight sequences decoded together, many experts
        dict(name="moe_batch", op="moe", type="bf16", tokens=8, width=2048, hidden=1024, experts=64, top_k=8, norm=False),
    ]


def _sizes(case):
    """Sizes of the tensors of an AdamW case: spread evenly over their logarithm, odd ones among them."""
    n, lo, hi = case["tensors"], math.log(case["least"]), math.log(case["most"])
    at = [((i * 0.6180339887498949) % 1.0 if n > 1 else 1.0) for i in range(n)]
    at[-1] = 1.0
    return [max(1, round(math.exp(lo + t * (hi - lo))) - i % 3) for i, t in enumerate(at)]


def draw(rng):
    def size(lo, hi):
        v = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return v // 64 * 64 if v > 128 and rng.random() < 0.5 else v

    while True:
        op = rng.choice(["linear", "linear", "grad", "adamw", "moe"])
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("linear", "grad"):
            case = dict(op=op, type=kind, tokens=size(1, 8192), n_in=size(64, 8192), n_out=size(64, 8192),
                        act=rng.choice(_ACTIVATIONS), bias=rng.random() < 0.7, ld=rng.choice([0, 0, 0, 64, rng.randrange(1, 100)]))
            if op == "linear":
                case.update(residual=rng.random() < 0.5, pre=rng.random() < 0.3)
            if case["tokens"] * case["n_in"] * case["n_out"] <= (1 << 38) // (4 if kind == "f32" else 1):
                return case
        elif op == "adamw":
            param = rng.choice(["f32", "f32", "bf16", "f16"])
            case = dict(op=op, tensors=rng.randrange(1, 150), least=rng.choice([1, 64, 1000]), most=size(1 << 12, 1 << 25),
                        param=param, grad=rng.choice(["f32", "bf16", "f16"]), bits=rng.choice([8, 32]),
                        copy=param == "f32" and rng.random() < 0.5)
            if sum(_sizes(case)) <= 100_000_000:
                return case
        else:
            experts = rng.choice([4, 8, 16, 32, 33, 60, 64, 128])
            case = dict(op=op, type=kind, tokens=size(1, 64), width=size(256, 4096), hidden=size(128, 4096), experts=experts,
                        top_k=min(experts, rng.choice([1, 2, 2, 3, 4, 6, 8])), norm=rng.random() < 0.5)
            if experts * case["width"] * case["hidden"] <= 64 * 2048 * 1024:
                return case


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(shape, gen, std=1.0, dtype=torch.float32, ld=0):
    """Normal values, the leading columns of a matrix `ld` columns wider."""
    wide = torch.empty((*shape[:-1], shape[-1] + ld), dtype=dtype, device="cuda")
    wide.normal_(0.0, std, generator=gen)
    return wide[..., :shape[-1]]


def prepare(case, seed):
    gen, state = _generator(seed), dict(case=case)
    if case["op"] in ("linear", "grad"):
        kind, ld = _TYPES[case["type"]], case["ld"]
        tokens, n_in, n_out = case["tokens"], case["n_in"], case["n_out"]
        state["x"] = _normal((tokens, n_in), gen, 1.0, kind, ld)
        state["w"] = _normal((n_out, n_in), gen, n_in ** -0.5, kind)
        state["bias"] = _normal((n_out,), gen, 0.5, kind) if case["bias"] else None
        if case["op"] == "linear":
            state["residual"] = _normal((tokens, n_out), gen, 1.0, kind, ld) if case["residual"] else None
            state["out"] = torch.empty((tokens, n_out), dtype=kind, device="cuda")
            state["pre"] = torch.empty_like(state["out"]) if case["pre"] else None
        else:
            state["dy"] = _normal((tokens, n_out), gen, 0.05, kind, ld)
            # the values before the activation, as the forward pass keeps them
            pre = state["x"].float() @ state["w"].float().t()
            state["pre"] = (pre if state["bias"] is None else pre + state["bias"].float()).to(kind)
            state["dx"] = torch.empty((tokens, n_in), dtype=kind, device="cuda")
            state["dw"] = torch.empty_like(state["w"])
            state["db"] = torch.empty(n_out, dtype=kind, device="cuda") if case["bias"] else None
    elif case["op"] == "adamw":
        # every tensor is a piece of one buffer and starts at a whole block, as where a trainer keeps them together
        sizes = _sizes(case)
        starts, total = [], 0
        for n in sizes:
            starts.append(total)
            total += -(-n // _BLOCK) * _BLOCK
        used = torch.zeros(total, dtype=torch.bool, device="cuda")
        for s, n in zip(starts, sizes):
            used[s:s + n] = True
        g_last = torch.empty(total, device="cuda").normal_(0.0, 1e-3, generator=gen).mul_(used)
        flat = dict(p=torch.empty(total, device="cuda").normal_(0.0, 0.02, generator=gen).mul_(used).to(_TYPES[case["param"]]),
                    g=torch.empty(total, device="cuda").normal_(0.0, 1e-3, generator=gen).mul_(used).to(_TYPES[case["grad"]]))
        m, v = 0.3 * g_last, g_last.square() * 0.02
        if case["bits"] == 32:
            flat.update(m=m, v=v)
        else:
            for name, x in (("m", m), ("v", v.sqrt())):       # of the second moment the root is held
                scale = x.view(-1, _BLOCK).abs().amax(1) / 448.0
                flat[name + "_scale"] = scale
                flat[name] = (x.view(-1, _BLOCK) / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)
        if case["copy"]:
            flat["copy"] = flat["p"].to(torch.bfloat16)
        state["flat"] = flat
        state["pieces"] = {name: [x[s:s + n] for s, n in zip(starts, sizes)] for name, x in flat.items() if "_scale" not in name}
        for name in ("m", "v"):
            if case["bits"] == 8:
                state["pieces"][name + "_scale"] = [flat[name + "_scale"][s // _BLOCK:(s + n + _BLOCK - 1) // _BLOCK] for s, n in zip(starts, sizes)]
        state["seed"] = seed & 0x7fffffff
    else:
        kind, width, hidden, experts = _TYPES[case["type"]], case["width"], case["hidden"], case["experts"]
        state["x"] = _normal((case["tokens"], width), gen, 1.0, kind)
        state["router"] = _normal((experts, width), gen, 1.5 * width ** -0.5, kind)
        state["w_in"] = _normal((experts, 2 * hidden, width), gen, width ** -0.5, kind)       # gate rows, then up rows
        state["w_out"] = _normal((experts, width, hidden), gen, hidden ** -0.5, kind)
        state["out"] = torch.empty_like(state["x"])
    return state


# ---- the plain forms: 32 bits unless said otherwise (exact() runs none of them)

def _act(name, z):
    if name == "relu":
        return torch.clamp_min(z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z) if name == "silu" else z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if name == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1.0 + z * (1.0 - s))


def _plain_linear(state):
    case, kind = state["case"], state["x"].dtype
    z = state["x"].float() @ state["w"].float().t()
    if state["bias"] is not None:
        z = z + state["bias"].float()
    y = _act(case["act"], z)
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return (y.to(kind), z.to(kind)) if case["pre"] else y.to(kind)


def _plain_grad(state):
    case, kind = state["case"], state["x"].dtype
    dz = state["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(case["act"], state["pre"].float())
    dx, dw = dz @ state["w"].float(), dz.t() @ state["x"].float()
    return (dx.to(kind), dw.to(kind)) + ((dz.sum(0).to(kind),) if case["bias"] else ())


_STEP = 7       # the step whose bias corrections the pass applies


def _words(n, seed, step):
    """The 32-bit words that round the states: a hash of the place, the seed and the step, in integers."""
    low = 0xffffffff
    h = torch.arange(n, dtype=torch.int64, device="cuda")
    h = (((h & low) + (h >> 32) * 0x6a09e667) * 0x9e3779b1 + ((seed + step * 0xbb67ae85) & low)) & low
    h = ((h ^ (h >> 15)) * 0x6a09e667) & low
    h = ((h ^ (h >> 13)) * 0xbb67ae85) & low
    return h ^ (h >> 16)


def _hold(x, words):
    """x, whole blocks of it, in 8 bits: scale and e4m3 values.  The lower bits round up where their sum with the word's
    20 bits carries; a value that is not zero stays so where it has no sign."""
    x = x.view(-1, _BLOCK)
    top = x.abs().amax(1, keepdim=True)
    inverse = torch.where(top > 0, torch.div(torch.full_like(top, 448.0), top), 0.0)
    y = torch.clamp_max(x.abs() * inverse, 448.0)
    bits = (y * 2.0 ** -120).view(torch.int32)      # the bits of e4m3, further left
    return (top * (1.0 / 448.0)).view(-1), torch.clamp_max((bits + words.view(-1, _BLOCK).to(torch.int32)) >> 20, 0x7e)


def _corrections(step):
    return _LR / (1.0 - _BETA1 ** step), 1.0 / math.sqrt(1.0 - _BETA2 ** step), 1.0 - _LR * _DECAY


def _plain_adamw(state):
    case, flat = state["case"], state["flat"]
    eight = case["bits"] == 8
    g, p = flat["g"].float(), flat["p"].float()
    if eight:
        m = (flat["m"].float().view(-1, _BLOCK) * flat["m_scale"][:, None]).view(-1)
        root = (flat["v"].float().view(-1, _BLOCK) * flat["v_scale"][:, None]).view(-1)
        v = root * root
    else:
        m, v = flat["m"], flat["v"]
    rate, correction, keep = _corrections(_STEP)
    m = m * _BETA1 + g * (1.0 - _BETA1)
    v = v * _BETA2 + (g * g) * (1.0 - _BETA2)
    root = torch.sqrt(v)
    p = p * keep - (m / (root * correction + _EPS)) * rate
    flat["p"].copy_(p)
    if case["copy"]:
        flat["copy"].copy_(p)
    if eight:
        words = _words(p.numel(), state["seed"], _STEP)
        scale, code = _hold(m, words & 0xfffff)
        flat["m_scale"].copy_(scale)
        flat["m"].copy_((code + torch.where(torch.signbit(m).view(-1, _BLOCK), 0x80, 0)).to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
        scale, code = _hold(root, words >> 12)
        code = torch.where((code == 0) & (root > 0).view(-1, _BLOCK), 1, code)
        flat["v_scale"].copy_(scale)
        flat["v"].copy_(code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
    else:
        flat["m"].copy_(m)
        flat["v"].copy_(v)
    return {name: x for name, x in flat.items() if name != "g"}


def _plain_moe(state):
    case, x = state["case"], state["x"].float()
    logits = x @ state["router"].float().t()
    # the k largest, ties to the lowest index: how many come before each
    before = (logits[:, None, :] > logits[:, :, None]) | ((logits[:, None, :] == logits[:, :, None]) & (
        torch.arange(case["experts"], device="cuda")[None, None, :] < torch.arange(case["experts"], device="cuda")[None, :, None]))
    chosen = before.sum(2) < case["top_k"]
    gate = torch.exp(logits - logits.amax(1, keepdim=True))
    gate = gate / (gate * chosen if case["norm"] else gate).sum(1, keepdim=True) * chosen
    experts = chosen.nonzero()[:, 1].view(-1, case["top_k"])
    # every expert on every token; what the gates leave out is multiplied by zero
    h = torch.matmul(x, state["w_in"].float().transpose(1, 2))
    h = _act("silu", h[..., :case["hidden"]]) * h[..., case["hidden"]:]
    y = torch.matmul(h, state["w_out"].float().transpose(1, 2))
    y = (y * gate.t()[:, :, None]).sum(0)
    return y.to(state["x"].dtype), experts.to(torch.int32), gate.gather(1, experts)


# ---- the framework's calls

def _own(state):
    from paper_2506_11277_amd import layers
    case = state["case"]
    if case["op"] == "linear":
        y = layers.linear(state["x"], state["w"], state["bias"], state["residual"], layers.ACTIVATIONS[case["act"]],
                          pre=state["pre"], out=state["out"])
        return (y, state["pre"]) if case["pre"] else y
    if case["op"] == "grad":
        dx, dw, db = layers.linear_grad(state["dy"], state["x"], state["w"], state["pre"], layers.ACTIVATIONS[case["act"]],
                                        bias=case["bias"], dx=state["dx"], dw=state["dw"], db=state["db"])
        return (dx, dw, db) if case["bias"] else (dx, dw)
    if case["op"] == "adamw":
        pieces = state["pieces"]
        if "plan" not in state:         # a program makes it once for its tensors
            state["plan"] = layers.AdamW(pieces["p"], pieces["m"], pieces["v"], pieces.get("m_scale"), pieces.get("v_scale"),
                                         pieces.get("copy"))
        state["plan"].step(pieces["g"], _STEP, lr=_LR, beta1=_BETA1, beta2=_BETA2, eps=_EPS, weight_decay=_DECAY,
                           seed=state["seed"])
        return {name: x for name, x in state["flat"].items() if name != "g"}
    return layers.moe(state["x"], state["router"], state["w_in"], state["w_out"], case["top_k"], normalise=case["norm"],
                      out=state["out"])


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "grad": _plain_grad, "adamw": _plain_adamw, "moe": _plain_moe}[state["case"]["op"]](state)


def work(case):
    """Inputs read once, outputs written once; products of matrices as multiplications and additions, AdamW's arithmetic
    as sixteen operations a value, of the experts those that are expected to be chosen."""
    if case["op"] in ("linear", "grad"):
        t, i, o, size = case["tokens"], case["n_in"], case["n_out"], _BYTES[case["type"]]
        if case["op"] == "linear":
            return {"bytes": size * (t * i + o * i + t * o * (1 + case["residual"] + case["pre"]) + o * case["bias"]), "flops": 2 * t * i * o}
        return {"bytes": size * (t * o * (1 if case["act"] == "none" else 2) + 2 * t * i + 2 * o * i + o * case["bias"]), "flops": 4 * t * i * o}
    if case["op"] == "adamw":
        n, p = sum(_sizes(case)), _BYTES[case["param"]]
        state = 16 if case["bits"] == 32 else 4 + 16 / _BLOCK
        return {"bytes": n * (2 * p + _BYTES[case["grad"]] + state + (2 if case["copy"] else 0)), "flops": 16 * n}
    t, d, f, e, k = case["tokens"], case["width"], case["hidden"], case["experts"], case["top_k"]
    size = _BYTES[case["type"]]
    used = e * (1.0 - (1.0 - k / e) ** t)
    return {"bytes": size * (2 * t * d + e * d + 3 * used * d * f) + 8 * t * k, "flops": 2 * t * d * e + 6 * t * k * d * f}


# ---- 64 bits, from the definitions

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        z = torch.matmul(state["x"].double(), state["w"].double().t())
        z = z if state["bias"] is None else z + state["bias"].double()
        y = _exact_act(case["act"], z)
        y = y if state["residual"] is None else y + state["residual"].double()
        return (y, z) if case["pre"] else y
    if case["op"] == "grad":
        dz = state["dy"].double()
        if case["act"] != "none":
            with torch.enable_grad():       # the slope by differentiation of the activation itself
                z = state["pre"].double().requires_grad_(True)
                dz = dz * torch.autograd.grad(_exact_act(case["act"], z).sum(), z)[0]
        dx, dw = torch.matmul(dz, state["w"].double()), torch.matmul(dz.t(), state["x"].double())
        return (dx, dw, dz.sum(0)) if case["bias"] else (dx, dw)
    if case["op"] == "adamw":
        return _exact_adamw(case, state)
    x = state["x"].double()
    share = torch.softmax(torch.matmul(x, state["router"].double().t()), 1)
    experts = torch.sort(share, dim=1, descending=True, stable=True).indices[:, :case["top_k"]].sort(1).values
    gate = share.gather(1, experts)
    gate = gate / gate.sum(1, keepdim=True) if case["norm"] else gate
    y = torch.zeros_like(x)
    for e in range(case["experts"]):        # the tokens of an expert together
        token, place = (experts == e).nonzero(as_tuple=True)
        if token.numel():
            both = torch.matmul(x[token], state["w_in"][e].double().t())
            h = _exact_act("silu", both[:, :case["hidden"]]) * both[:, case["hidden"]:]
            y.index_add_(0, token, gate[token, place][:, None] * torch.matmul(h, state["w_out"][e].double().t()))
    return y, None, gate


def _exact_act(name, z):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3)))
    return z / (1.0 + torch.exp(-z)) if name == "silu" else z


def _exact_adamw(case, state):
    flat = state["flat"]
    g, p = flat["g"].double(), flat["p"].double()

    def held(name):
        x = flat[name].double()
        return x if case["bits"] == 32 else (x.view(-1, _BLOCK) * flat[name + "_scale"].double()[:, None]).view(-1)

    m = torch.lerp(g, held("m"), _BETA1)
    v = torch.lerp(g.square(), held("v") if case["bits"] == 32 else held("v").square(), _BETA2)
    unbiased_m, unbiased_v = m / (1.0 - _BETA1 ** _STEP), v / (1.0 - _BETA2 ** _STEP)
    p = p - _LR * (_DECAY * p + unbiased_m / (unbiased_v.sqrt() + _EPS))
    answer = dict(p=p, m=m, v=v)
    if case["copy"]:
        answer["copy"] = p
    if case["bits"] == 8:
        words = _words(p.numel(), state["seed"], _STEP)
        for name, x, share in (("m", m, (words & 0xfffff).double() / 2 ** 20), ("v", v.sqrt(), (words >> 12).double() / 2 ** 20)):
            scale = x.view(-1, _BLOCK).abs().amax(1) / 448.0
            y = (x.view(-1, _BLOCK) / torch.where(scale > 0, scale, 1.0)[:, None]).view(-1)
            unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)       # of e4m3 at this value
            least = 2.0 ** -9 * ((y > 0) if name == "v" else 0.0)
            answer[name + "_scale"] = scale
            answer[name] = torch.sign(y) * torch.clamp(torch.floor(y.abs() / unit + share) * unit, max=448.0).clamp_min(least)
    return answer
