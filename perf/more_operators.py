"""Performance cases of the feed-forward layer in 8 bits: the root-mean-square norm in front of it with the residual's
addition and its results in 8 bits, that norm's gradients, rows held in 8 bits, the product of two matrices that are held so,
and a linear layer's gradients from operands that the forward pass kept in 8 bits.

8 bits: whole numbers from -127 to 127 with one float32 scale for each row (a token of an activation, an output feature of a
weight): code = t * (127 / a) rounded to nearest, ties to even, for the row's values t in 32 bits and a = max |t|.

With `own` false a pass is the operator's plain form (elementary torch operations in 32 bits, rounded once at the end),
otherwise the calls a program makes of `paper_2506_11277_amd.layers`.  Both take the same tensors.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_EPS = 1e-6
_MOST = 127.0


def listed():
    return [
        # one token in a serving loop, between two layers: the residual is added, the norm goes into an 8-bit product
        dict(name="norm_token", op="norm", type="bf16", tokens=1, width=4096, residual=True, eight=True, ld=0),
        # the same for a training step's tokens, or a long prompt's
        dict(name="norm_wide", op="norm", type="bf16", tokens=16384, width=4096, residual=True, eight=True, ld=0),
        # gradients of the norm in a small model whose width fits nothing, rows off 16 bytes
        dict(name="norm_grad_ragged", op="norm_grad", type="f16", tokens=1531, width=1001, add=False, ld=3),
        # ... in a training step, with the gradient that comes along the residual stream
        dict(name="norm_grad_wide", op="norm_grad", type="bf16", tokens=8192, width=8192, add=True, ld=0),
        # a small weight in 32 bits to 8, when a model is loaded
        dict(name="quantise_small", op="quantise", type="f32", rows=777, cols=1001, ld=0),
        # the wide layer's activations of a training step, kept for its gradients
        dict(name="quantise_wide", op="quantise", type="bf16", rows=8192, cols=8192, ld=0),
        # one token through a narrow layer: what a call costs
        dict(name="linear8_token", op="linear8", type="bf16", tokens=1, n_in=1024, n_out=4096, act="gelu_tanh", bias=True,
             residual=False, pre=False, ld=0),
        # a batch of sequences decoded together, back to the width of the residual stream that it is added to
        dict(name="linear8_decode", op="linear8", type="bf16", tokens=48, n_in=8192, n_out=2048, act="none", bias=False,
             residual=True, pre=False, ld=0),
        # sizes that fit no tile and rows off 16 bytes, everything in the epilogue
        dict(name="linear8_ragged", op="linear8", type="f16", tokens=1531, n_in=1001, n_out=777, act="relu", bias=True,
             residual=True, pre=False, ld=0),
        # the wide layer of a training step, the values before the activation written along
        dict(name="linear8_wide", op="linear8", type="bf16", tokens=8192, n_in=4096, n_out=8192, act="gelu", bias=True,
             residual=False, pre=True, ld=0),
        # gradients of a small layer in 32 bits, everything that the forward pass read held in 8
        dict(name="grad8_small", op="grad8", type="f32", tokens=500, n_in=512, n_out=384, act="silu", bias=True, w8=True, pre8=True, ld=0),
        # gradients of the wide layer of a training step: input and pre-activation kept in 8 bits, the weight in 16
        dict(name="grad8_wide", op="grad8", type="bf16", tokens=8192, n_in=4096, n_out=8192, act="gelu", bias=True, w8=False, pre8=True, ld=0),
    ]


def draw(rng):
    def size(lo, hi):
        v = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return v // 64 * 64 if v > 128 and rng.random() < 0.5 else v

    while True:
        op = rng.choice(["norm", "norm_grad", "quantise", "linear8", "linear8", "grad8"])
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        ld = rng.choice([0, 0, 0, 64, rng.randrange(1, 100)])
        if op in ("norm", "norm_grad"):
            case = dict(op=op, type=kind, tokens=size(1, 16384), width=size(16, 16384), ld=ld)
            if op == "norm":
                case.update(residual=rng.random() < 0.7, eight=rng.random() < 0.7)
            else:
                case.update(add=rng.random() < 0.6)
            if case["tokens"] * case["width"] <= (1 << 26) // (2 if kind == "f32" else 1):
                return case
        elif op == "quantise":
            case = dict(op=op, type=kind, rows=size(1, 16384), cols=size(16, 16384), ld=ld)
            if case["rows"] * case["cols"] <= (1 << 26) // (2 if kind == "f32" else 1):
                return case
        else:
            case = dict(op=op, type=kind, tokens=size(1, 8192), n_in=size(64, 8192), n_out=size(64, 8192),
                        act=rng.choice(_ACTIVATIONS), bias=rng.random() < 0.7, ld=ld)
            if op == "linear8":
                case.update(residual=rng.random() < 0.5, pre=rng.random() < 0.3)
            else:
                case.update(w8=rng.random() < 0.5, pre8=rng.random() < 0.7)
            if case["tokens"] * case["n_in"] * case["n_out"] <= (1 << 38) // (4 if kind == "f32" and op == "grad8" else 1):
                return case


def _columns(shape, dtype, ld=0):
    """The leading columns of a matrix `ld` columns wider."""
    return torch.empty((*shape[:-1], shape[-1] + ld), dtype=dtype, device="cuda")[..., :shape[-1]]


def _normal(shape, gen, std=1.0, dtype=torch.float32, ld=0):
    x = _columns(shape, dtype, ld)
    return x.copy_(torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen))


def _stream(shape, gen, dtype, ld=0):
    """Values of a residual stream: channels of different sizes, a few of them large."""
    x = torch.empty(shape, device="cuda").normal_(generator=gen)
    return _columns(shape, dtype, ld).copy_(x * torch.empty(shape[-1], device="cuda").normal_(0.0, 0.5, generator=gen).exp_())


def _eight(x, ld=0):
    """Rows in 8 bits, as the programs in front of these calls leave them: (codes, scales)."""
    codes, scale = _codes(x)
    return _columns(x.shape, torch.int8, ld).copy_(codes), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, ld, state = _TYPES[case["type"]], case["ld"], dict(case=case)
    if case["op"] in ("norm", "norm_grad"):
        shape = (case["tokens"], case["width"])
        state["weight"] = (1.0 + _normal(shape[1:], gen, 0.2)).to(kind)
        state["x"] = _stream(shape, gen, kind, ld)
        if case["op"] == "norm":
            state["residual"] = _stream(shape, gen, kind, ld) if case["residual"] else None
            state["total"] = torch.empty(shape, dtype=kind, device="cuda") if case["residual"] else None
            state["out"] = torch.empty(shape, dtype=torch.int8 if case["eight"] else kind, device="cuda")
            state["scale"] = torch.empty(shape[0], device="cuda") if case["eight"] else None
        else:
            state["dy"] = _normal(shape, gen, 0.05, kind, ld)
            state["add"] = _normal(shape, gen, 0.05, kind, ld) if case["add"] else None
            state["dx"] = torch.empty(shape, dtype=kind, device="cuda")
            state["dw"] = torch.empty_like(state["weight"])
    elif case["op"] == "quantise":
        shape = (case["rows"], case["cols"])
        state["x"] = _stream(shape, gen, kind, ld)
        state["out"] = torch.empty(shape, dtype=torch.int8, device="cuda")
        state["scale"] = torch.empty(shape[0], device="cuda")
    else:
        tokens, n_in, n_out = case["tokens"], case["n_in"], case["n_out"]
        state["x"], state["x_scale"] = _eight(_stream((tokens, n_in), gen, torch.float32), ld)
        w = _normal((n_out, n_in), gen, n_in ** -0.5)
        state["bias"] = _normal((n_out,), gen, 0.5, kind) if case["bias"] else None
        if case["op"] == "linear8":
            state["w"], state["w_scale"] = _eight(w)
            state["residual"] = _normal((tokens, n_out), gen, 1.0, kind, ld) if case["residual"] else None
            state["out"] = torch.empty((tokens, n_out), dtype=kind, device="cuda")
            state["pre"] = torch.empty_like(state["out"]) if case["pre"] else None
        else:
            # the values before the activation, as the forward pass keeps them
            pre = (state["x"].float() @ w.t()) * state["x_scale"][:, None]
            pre = pre if state["bias"] is None else pre + state["bias"].float()
            state["pre"], state["pre_scale"] = (_eight(pre) if case["pre8"] else (pre.to(kind), None)) if case["act"] != "none" else (None, None)
            state["w"], state["w_scale"] = _eight(w) if case["w8"] else (w.to(kind), None)
            state["dy"] = _normal((tokens, n_out), gen, 0.05, kind, ld)
            state["dx"] = torch.empty((tokens, n_in), dtype=kind, device="cuda")
            state["dw"] = torch.empty((n_out, n_in), dtype=kind, device="cuda")
            state["db"] = torch.empty(n_out, dtype=kind, device="cuda") if case["bias"] else None
    return state


# ---- the plain forms: 32 bits (exact() runs none of them)

def _codes(t, factor=None):
    """Rows of t in 8 bits; the scales stand for the rows of t times `factor`."""
    top = t.float().abs().amax(1)
    inverse = torch.where(top > 0, torch.div(torch.full_like(top, _MOST), top), 0.0)
    scale = top * (1.0 / _MOST)
    return torch.round(t.float() * inverse[:, None]).to(torch.int8), scale if factor is None else scale * factor


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


def _plain_norm(state):
    case, kind, h = state["case"], state["x"].dtype, state["x"].float()
    if case["residual"]:
        h = h + state["residual"].float()
    r = torch.rsqrt(h.square().mean(1) + _EPS)
    t = h * state["weight"].float()
    # (in 8 bits the norm's factor is in the scale alone: the codes are those of the row without it)
    answer = _codes(t, r) if case["eight"] else ((t * r[:, None]).to(kind),)
    return answer + ((h.to(kind),) if case["residual"] else ())


def _plain_norm_grad(state):
    kind, h, dy = state["x"].dtype, state["x"].float(), state["dy"].float()
    r = torch.rsqrt(h.square().mean(1, keepdim=True) + _EPS)
    n, g = h * r, dy * state["weight"].float()
    dx = (g - n * (g * n).mean(1, keepdim=True)) * r
    if state["add"] is not None:
        dx = dx + state["add"].float()
    return dx.to(kind), (dy * n).sum(0).to(kind)


def _plain_quantise(state):
    return _codes(state["x"])


def _plain_linear8(state):
    case, kind = state["case"], state["out"].dtype
    z = (state["x"].float() @ state["w"].float().t()) * state["x_scale"][:, None] * state["w_scale"]
    if state["bias"] is not None:
        z = z + state["bias"].float()
    y = _act(case["act"], z)
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return (y.to(kind), z.to(kind)) if case["pre"] else y.to(kind)


def _plain_grad8(state):
    case, kind = state["case"], state["dy"].dtype
    x, w, dz = state["x"].float() * state["x_scale"][:, None], state["w"].float(), state["dy"].float()
    if case["w8"]:
        w = w * state["w_scale"][:, None]
    if case["act"] != "none":
        z = state["pre"].float()
        dz = dz * _act_slope(case["act"], z * state["pre_scale"][:, None] if case["pre8"] else z)
    dx, dw = dz @ w, dz.t() @ x
    return (dx.to(kind), dw.to(kind)) + ((dz.sum(0).to(kind),) if case["bias"] else ())


# ---- the framework's calls

def _own(state):
    from paper_2506_11277_amd import layers
    case = state["case"]
    if case["op"] == "norm":
        if case["eight"]:
            codes, scale, total = layers.rms_norm8(state["x"], state["weight"], state["residual"], _EPS, total=state["total"],
                                                   out=state["out"], scale=state["scale"])
            return (codes, scale, total) if case["residual"] else (codes, scale)
        y, total = layers.rms_norm(state["x"], state["weight"], state["residual"], _EPS, total=state["total"], out=state["out"])
        return (y, total) if case["residual"] else (y,)
    if case["op"] == "norm_grad":
        return layers.rms_norm_grad(state["dy"], state["x"], state["weight"], _EPS, add=state["add"], dx=state["dx"], dw=state["dw"])
    if case["op"] == "quantise":
        return layers.quantise(state["x"], out=state["out"], scale=state["scale"])
    if case["op"] == "linear8":
        y = layers.linear8(state["x"], state["x_scale"], state["w"], state["w_scale"], state["bias"], state["residual"],
                           layers.ACTIVATIONS[case["act"]], pre=state["pre"], out=state["out"])
        return (y, state["pre"]) if case["pre"] else y
    dx, dw, db = layers.linear8_grad(state["dy"], state["x"], state["w"], state["pre"], layers.ACTIVATIONS[case["act"]],
                                     x_scale=state["x_scale"], w_scale=state["w_scale"], pre_scale=state["pre_scale"], bias=case["bias"],
                                     dx=state["dx"], dw=state["dw"], db=state["db"])
    return (dx, dw, db) if case["bias"] else (dx, dw)


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "quantise": _plain_quantise, "linear8": _plain_linear8,
            "grad8": _plain_grad8}[state["case"]["op"]](state)


def work(case):
    """Inputs read once, outputs written once; products of matrices as multiplications and additions, a handful of
    operations for each value of a norm or of rows that go to 8 bits."""
    size = _BYTES[case["type"]]
    if case["op"] == "norm":
        t, n = case["tokens"], case["width"]
        return {"bytes": t * n * (size * (3 if case["residual"] else 1) + (1 if case["eight"] else size)) + n * size + 4 * t * case["eight"],
                "flops": 6 * t * n}
    if case["op"] == "norm_grad":
        t, n = case["tokens"], case["width"]
        return {"bytes": size * (t * n * (4 if case["add"] else 3) + 2 * n), "flops": 12 * t * n}
    if case["op"] == "quantise":
        t, n = case["rows"], case["cols"]
        return {"bytes": t * n * (size + 1) + 4 * t, "flops": 3 * t * n}
    t, i, o = case["tokens"], case["n_in"], case["n_out"]
    if case["op"] == "linear8":
        return {"bytes": t * i + o * i + 4 * (t + o) + size * (t * o * (1 + case["residual"] + case["pre"]) + o * case["bias"]), "flops": 2 * t * i * o}
    pre = 0 if case["act"] == "none" else 1 if case["pre8"] else size
    return {"bytes": t * o * (size + pre) + t * i * (1 + size) + o * i * ((1 if case["w8"] else size) + size) + size * o * case["bias"] +
            4 * (t + (o if case["w8"] else 0) + (t if pre == 1 else 0)), "flops": 4 * t * i * o}


# ---- 64 bits, from the definitions

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        h = state["x"].double()
        if case["residual"]:
            h = torch.add(h, state["residual"].double())
        y = h * state["weight"].double() / (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["width"] + _EPS).sqrt()
        answer = (None, y.abs().max(1).values / _MOST) if case["eight"] else (y,)
        return answer + ((h,) if case["residual"] else ())
    if case["op"] == "norm_grad":
        with torch.enable_grad():       # by differentiation of the norm itself
            h, w = state["x"].double().requires_grad_(True), state["weight"].double().requires_grad_(True)
            y = h * w / (h.pow(2).mean(1, keepdim=True) + _EPS).sqrt()
            dx, dw = torch.autograd.grad(y, (h, w), state["dy"].double())
        return (dx if state["add"] is None else torch.add(dx, state["add"].double())), dw
    if case["op"] == "quantise":
        return None, state["x"].double().abs().max(1).values / _MOST
    x = state["x"].double() * state["x_scale"].double().unsqueeze(1)
    w = state["w"].double()
    if state["w_scale"] is not None:
        w = w * state["w_scale"].double().unsqueeze(1)
    if case["op"] == "linear8":
        z = torch.matmul(x, w.t())
        z = z if state["bias"] is None else z + state["bias"].double()
        y = _exact_act(case["act"], z)
        y = y if state["residual"] is None else y + state["residual"].double()
        return (y, z) if case["pre"] else y
    dz = state["dy"].double()
    if case["act"] != "none":
        with torch.enable_grad():       # the slope by differentiation of the activation itself
            z = state["pre"].double()
            z = (z if state["pre_scale"] is None else z * state["pre_scale"].double().unsqueeze(1)).requires_grad_(True)
            dz = dz * torch.autograd.grad(_exact_act(case["act"], z).sum(), z)[0]
    dx, dw = torch.matmul(dz, w), torch.matmul(dz.t(), x)
    return (dx, dw, dz.sum(0)) if case["bias"] else (dx, dw)


def _exact_act(name, z):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3)))
    return z / (1.0 + torch.exp(-z)) if name == "silu" else z
