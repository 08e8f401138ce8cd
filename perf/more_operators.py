"""More operators of a transformer's training step that the library offers, as cases that can be timed and compared: layer
norm, rotary positions, and the linear layer with what follows it (bias, activation, residual), each with its gradients.

A case is a dict of plain values.  Its "op" says which operator and direction it takes:

  norm         normalised rows, their means and reciprocal deviations   (Context.layer_norm_forward)
  norm_grad    gradients of rows, weight and bias                       (Context.layer_norm_backward)
  rotary       queries and keys turned by their positions, or back      (Context.rotary)
  linear       act(x W^T + bias) + residual                             (Context.linear_forward)
  linear_grad  gradients of x, W and bias                               (Context.linear_backward)

Sizes follow the shapes of paper_2601_02311_b200/synth.py: hidden sizes that are multiples of 128, heads of 128, a
feed-forward layer four times as wide, sequences of 2048 to 32768, 1 to 64 sequences a micro-batch.
"""
import functools
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}


def norm(name, rows, cols, op="norm", dtype="bf16", eps=1e-5, residual=False, wide=False):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, eps=eps, residual=residual, wide=wide)


def rotary(name, batch, length, heads, kv_heads, dim=128, rotary_dim=0, dtype="bf16", interleaved=False, inverse=False, base=10000.0,
           factor=1.0, original=0.0, magnitude=1.0, first=0, packed=False):
    return dict(name=name, op="rotary", batch=batch, length=length, heads=heads, kv_heads=kv_heads, dim=dim, rotary_dim=rotary_dim or dim,
                dtype=dtype, interleaved=interleaved, inverse=inverse, base=base, factor=factor, original=original, low=1.0, high=32.0,
                magnitude=magnitude, first=first, packed=packed)


def linear(name, tokens, inputs, outputs, op="linear", dtype="bf16", activation="none", bias=True, residual=False, keep=False, below="none",
           wide=False):
    return dict(name=name, op=op, tokens=tokens, inputs=inputs, outputs=outputs, dtype=dtype, activation=activation, bias=bias,
                residual=residual, keep=keep, below=below, wide=wide)


def listed():
    return [
        # before a sublayer of the smallest shape, a few hundred tokens: what a call costs
        norm("norm_short", 384, 768),
        # before a sublayer of a large shape: sixteen sequences of 4096
        norm("norm_large", 65536, 8192),
        # the gradient in 32 bits, of a width that is no multiple of anything
        norm("norm_grad_odd", 12301, 5003, op="norm_grad", dtype="f32"),
        # a large shape's gradient, with the one that went past the sublayer added
        norm("norm_grad_large", 65536, 8192, op="norm_grad", residual=True),
        # the smallest shape's queries and keys
        rotary("rotary_short", 1, 384, 6, 6),
        # the gradient for long sequences with shared key heads, of a context stretched by eight
        rotary("rotary_long_back", 2, 32768, 64, 8, interleaved=True, inverse=True, base=500000.0, factor=8.0, original=4096.0, magnitude=1.2),
        # the smallest shape's projection to queries, keys and values
        linear("linear_short", 384, 768, 2304),
        # tokens and widths that fill no tile, back onto a residual
        linear("linear_odd", 1003, 5003, 4999, dtype="f16", residual=True),
        # into a large shape's feed-forward layer, with what its gradient needs kept
        linear("linear_up", 16384, 8192, 32768, activation="gelu", keep=True),
        # the smallest shape's gradients
        linear("linear_grad_short", 384, 768, 2304, op="linear_grad"),
        # gradients through an activation of the layer's own, the weight's in 32 bits
        linear("linear_grad_odd", 5003, 1416, 2503, op="linear_grad", dtype="f16", activation="silu", wide=True),
        # out of a large shape's feed-forward layer, down to before its activation
        linear("linear_grad_down", 16384, 32768, 8192, op="linear_grad", below="gelu"),
    ]


def between(rng, lo, hi):
    """A whole number, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "norm_grad", "rotary", "rotary", "linear", "linear", "linear", "linear_grad", "linear_grad", "linear_grad"])
    if op.startswith("norm"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        cols = rng.choice([between(rng, 1, 32768), 128 * rng.randint(6, 256)])
        rows = between(rng, 1, min(131072, (250_000_000 if dtype == "f32" else 500_000_000) // cols))
        case = norm("", rows, cols, op, dtype, rng.choice([1e-5, 1e-6]), rng.random() < 0.4, rng.random() < 0.3)
    elif op == "rotary":
        dim = rng.choice([128, 128, 64, 96, 80, 2 * rng.randint(1, 64)])
        part = rng.choice([dim, dim, dim, max(2, dim // 4 * 2)])
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 7, 8])
        batch = rng.choice([1, 1, 2, 3, 8])
        length = between(rng, 1, min(32768, 600_000_000 // (batch * kv_heads * (group + 1) * dim)))
        factor = rng.choice([1.0, 1.0, 4.0, 8.0])
        case = rotary("", batch, length, kv_heads * group, kv_heads, dim, part, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.5,
                      rng.random() < 0.4, rng.choice([10000.0, 500000.0]), factor, rng.choice([0.0, 4096.0]) if factor > 1.0 else 0.0,
                      0.1 * math.log(factor) + 1.0, rng.choice([0, 0, rng.randrange(1 << 20)]), rng.random() < 0.4)
    else:
        inputs, outputs = (rng.choice([between(rng, 1, 16384), 128 * rng.randint(6, 128), 128 * rng.randint(6, 128)]) for _ in range(2))
        if rng.random() < 0.25:
            outputs = 4 * inputs if rng.random() < 0.5 else (inputs + 3) // 4
        tokens = between(rng, 1, min(65536, 400_000_000_000 // (inputs * outputs), 500_000_000 // max(inputs, outputs)))
        activation = rng.choice(["none", "none", "gelu", "gelu_tanh", "silu", "relu"])
        case = linear("", tokens, inputs, outputs, op, rng.choice(["bf16", "bf16", "f16"]), activation, rng.random() < 0.7, rng.random() < 0.4,
                      activation != "none" and rng.random() < 0.7, "none" if op == "linear" else rng.choice(["none", "none", "gelu", "silu"]),
                      rng.random() < 0.4)
    del case["name"]
    return case


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, size=1.0, mean=0.0):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(mean, size, generator=gen)

    def matrix(rows, cols, size=1.0):
        """Rows that begin at multiples of 16 bytes, as the linear layer takes them."""
        return normal(rows, (cols + 7) // 8 * 8, size=size)[:, :cols]

    state = dict(case=case)
    if case["op"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        state["x"] = normal(rows, cols, size=1.5, mean=0.3)
        state["weight"], state["bias"] = normal(cols, size=0.2, mean=1.0), normal(cols, size=0.1)
        if case["op"] == "norm_grad":
            state["d_y"] = normal(rows, cols, size=0.01)
            state["residual"] = normal(rows, cols, size=0.01) if case["residual"] else None
            _, state["mean"], state["rstd"] = plain_norm(state)
    elif case["op"] == "rotary":
        batch, length, dim = case["batch"], case["length"], case["dim"]
        state["q"], state["k"] = normal(batch, length, case["heads"], dim), normal(batch, length, case["kv_heads"], dim)
        state["positions"] = None
        if case["packed"]:
            # documents behind one another, each from position 0 on
            begins = torch.rand(batch, length, device="cuda", generator=gen) < 3.0 / length
            at = torch.arange(length, device="cuda").expand(batch, length)
            state["positions"] = (at - torch.where(begins, at, 0).cummax(1).values).int()
    else:
        tokens, inputs, outputs = case["tokens"], case["inputs"], case["outputs"]
        state["x"], state["weight"] = matrix(tokens, inputs), matrix(outputs, inputs, size=inputs ** -0.5)
        if case["op"] == "linear":
            state["bias"] = normal(outputs, size=0.1) if case["bias"] else None
            state["residual"] = matrix(tokens, outputs) if case["residual"] else None
        else:
            state["d_y"] = matrix(tokens, outputs, size=0.01)
            state["pre"] = matrix(tokens, outputs) if case["activation"] != "none" else None
            state["below"] = matrix(tokens, inputs) if case["below"] != "none" else None
            state["residual"] = matrix(tokens, inputs, size=0.01) if case["residual"] else None
    return state


# ---- the operators in their plain form

def plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + s["case"]["eps"])
    y = x * rstd * s["weight"].float() + s["bias"].float()
    return y.to(s["x"].dtype), mean.flatten(), rstd.flatten()


def plain_norm_grad(s):
    case, dtype = s["case"], s["x"].dtype
    d_y, rstd = s["d_y"].float(), s["rstd"][:, None]
    normed = (s["x"].float() - s["mean"][:, None]) * rstd
    wide = torch.float32 if case["wide"] else dtype
    d_weight, d_bias = (d_y * normed).sum(0).to(wide), d_y.sum(0).to(wide)
    g = d_y * s["weight"].float()
    d_x = rstd * (g - g.mean(1, keepdim=True) - normed * (g * normed).mean(1, keepdim=True))
    if s["residual"] is not None:
        d_x = d_x + s["residual"].float()
    return {"d_x": d_x.to(dtype), "d_weight": d_weight, "d_bias": d_bias}


def plain_rotary(s):
    case = s["case"]
    half = case["rotary_dim"] // 2
    freq = case["base"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    if case["factor"] != 1.0:
        keep = torch.zeros_like(freq)
        if case["original"]:
            turns = case["original"] * freq / (2 * math.pi)
            keep = ((turns - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
        freq = freq * (keep + (1.0 - keep) / case["factor"])
    positions = torch.arange(case["length"], device="cuda")[None] if s["positions"] is None else s["positions"]
    angle = (positions + case["first"])[:, :, None, None].double() * freq
    if case["inverse"]:
        angle = -angle
    cos, sin = ((f(angle) * case["magnitude"]).float() for f in (torch.cos, torch.sin))
    out = []
    for x in (s["q"], s["k"]):
        turned, rest = x[..., :2 * half].float(), x[..., 2 * half:]
        if case["interleaved"]:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = turned[..., :half], turned[..., half:]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        out.append(torch.cat((turned.to(x.dtype), rest), -1))
    return out


SQRT_HALF, TANH_FACTOR, TANH_CUBE = math.sqrt(0.5), math.sqrt(2.0 / math.pi), 0.044715


def activated(v, activation):
    if activation == "relu":
        return torch.where(v > 0, v, 0.0)
    if activation == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * SQRT_HALF))
    if activation == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(TANH_FACTOR * (v + TANH_CUBE * v * v * v)))
    return v / (1.0 + torch.exp(-v)) if activation == "silu" else v


def slope(v, activation):
    if activation == "relu":
        return (v > 0).float()
    if activation == "gelu":
        return 0.5 * (1.0 + torch.erf(v * SQRT_HALF)) + v * torch.exp(-0.5 * v * v) * (0.5 * TANH_FACTOR)
    if activation == "gelu_tanh":
        t = torch.tanh(TANH_FACTOR * (v + TANH_CUBE * v * v * v))
        return 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * TANH_FACTOR * (1.0 + 3.0 * TANH_CUBE * v * v)
    s = 1.0 / (1.0 + torch.exp(-v))
    return s * (1.0 + v * (1.0 - s))


def plain_linear(s):
    case, dtype = s["case"], s["x"].dtype
    pre = s["x"].float() @ s["weight"].float().t()
    if s["bias"] is not None:
        pre = pre + s["bias"].float()
    y = activated(pre, case["activation"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(dtype), pre.to(dtype)) if case["keep"] else y.to(dtype)


def plain_linear_grad(s):
    case, dtype = s["case"], s["x"].dtype
    d_pre = s["d_y"].float()
    if s["pre"] is not None:
        d_pre = d_pre * slope(s["pre"].float(), case["activation"])
    d_x = d_pre @ s["weight"].float()
    if s["below"] is not None:
        d_x = d_x * slope(s["below"].float(), case["below"])
    if s["residual"] is not None:
        d_x = d_x + s["residual"].float()
    wide = torch.float32 if case["wide"] else dtype
    return {"d_x": d_x.to(dtype), "d_weight": (d_pre.t() @ s["x"].float()).to(wide), "d_bias": d_pre.sum(0).to(wide)}


PLAIN = dict(norm=plain_norm, norm_grad=plain_norm_grad, rotary=plain_rotary, linear=plain_linear, linear_grad=plain_linear_grad)


# ---- the library's calls

@functools.lru_cache(maxsize=None)
def context(device, stream):
    from paper_2601_02311_b200 import ps
    return ps.Context(device, torch.cuda.ExternalStream(stream, device) if stream else None)


def run(state):
    case = state["case"]
    if not own:
        return PLAIN[case["op"]](state)
    ctx = context(torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)
    if case["op"] == "norm":
        return ctx.layer_norm_forward(state["x"], state["weight"], state["bias"], eps=case["eps"])
    if case["op"] == "norm_grad":
        d_x, d_weight, d_bias = ctx.layer_norm_backward(state["d_y"], state["x"], state["mean"], state["rstd"], state["weight"],
                                                        residual=state["residual"], dtype=torch.float32 if case["wide"] else None)
        return {"d_x": d_x, "d_weight": d_weight, "d_bias": d_bias}
    if case["op"] == "rotary":
        return ctx.rotary(state["q"], state["k"], positions=state["positions"], first=case["first"], base=case["base"],
                          dims=case["rotary_dim"], interleaved=case["interleaved"], factor=case["factor"], original=case["original"],
                          low=case["low"], high=case["high"], magnitude=case["magnitude"], inverse=case["inverse"])
    if case["op"] == "linear":
        return ctx.linear_forward(state["x"], state["weight"], state["bias"], activation=case["activation"], residual=state["residual"],
                                  keep=case["keep"])
    d_x, d_weight, d_bias = ctx.linear_backward(state["d_y"], state["x"], state["weight"], pre=state["pre"], activation=case["activation"],
                                                below=state["below"], below_activation=case["below"], residual=state["residual"],
                                                dtype=torch.float32 if case["wide"] else None)
    return {"d_x": d_x, "d_weight": d_weight, "d_bias": d_bias}


# ---- what a pass cannot do without

def work(case):
    w = WIDTH[case["dtype"]]
    wide = 4 if case.get("wide") else w
    if case["op"].startswith("norm"):
        n, rows, cols = case["rows"] * case["cols"], case["rows"], case["cols"]
        if case["op"] == "norm":
            return {"bytes": 2 * n * w + 8 * rows + 2 * cols * w, "flops": 8 * n}
        return {"bytes": (4 if case["residual"] else 3) * n * w + 8 * rows + cols * (w + 2 * wide), "flops": 14 * n}
    if case["op"] == "rotary":
        rows = case["batch"] * case["length"]
        heads = rows * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * heads * case["dim"] * w + (4 * rows if case["packed"] else 0), "flops": 3 * heads * case["rotary_dim"]}
    t, k, n = case["tokens"], case["inputs"], case["outputs"]
    if case["op"] == "linear":
        return {"bytes": w * (t * k + n * k + t * n * (1 + case["residual"] + case["keep"]) + n * case["bias"]), "flops": 2 * t * k * n}
    arrays = t * n * (1 + (case["activation"] != "none")) + n * k + t * k * (2 + (case["below"] != "none") + case["residual"])
    return {"bytes": w * arrays + wide * (n * k + n), "flops": 4 * t * k * n + t * n}


# ---- the definitions in 64 bits

def exact_norm(s):
    case = s["case"]
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    rstd = (var + case["eps"]).pow(-0.5)
    if case["op"] == "norm":
        y = torch.addcmul(s["bias"].double(), (x - mean[:, None]).mul_(rstd[:, None]), s["weight"].double())
        return y, mean, rstd
    # the call is given the mean and the deviation as they were kept
    mean, rstd = s["mean"].double(), s["rstd"].double()
    x.sub_(mean[:, None]).mul_(rstd[:, None])
    d_y = s["d_y"].double()
    d_weight, d_bias = torch.einsum("rc,rc->c", d_y, x), torch.einsum("rc->c", d_y)
    d_y.mul_(s["weight"].double())
    along, across = torch.einsum("rc,rc->r", d_y, x) / case["cols"], torch.einsum("rc->r", d_y) / case["cols"]
    d_x = d_y.sub_(across[:, None]).sub_(x.mul_(along[:, None])).mul_(rstd[:, None])
    if s["residual"] is not None:
        d_x.add_(s["residual"])
    return {"d_x": d_x, "d_weight": d_weight, "d_bias": d_bias}


def exact_rotary(s):
    case = s["case"]
    pairs = case["rotary_dim"] // 2
    speeds = []
    for i in range(pairs):
        f = math.exp(-2.0 * i / case["rotary_dim"] * math.log(case["base"]))
        slow = f / case["factor"]
        if case["factor"] != 1.0 and case["original"]:
            ramp = (case["original"] * f / math.tau - case["low"]) / (case["high"] - case["low"])
            slow += min(1.0, max(0.0, ramp)) * (f - slow)
        speeds.append(-slow if case["inverse"] else slow)
    at = torch.arange(case["length"], device="cuda").expand(case["batch"], -1) if s["positions"] is None else s["positions"]
    angle = torch.outer((at.flatten() + case["first"]).double(), torch.tensor(speeds, device="cuda", dtype=torch.float64))
    turn = torch.polar(torch.full_like(angle, case["magnitude"]), angle).view(case["batch"], case["length"], 1, pairs)
    out = []
    for x in (s["q"], s["k"]):
        y = x.double()
        for h in range(0, x.shape[2], 8):
            part = y[:, :, h:h + 8, :2 * pairs].unflatten(-1, (pairs, 2) if case["interleaved"] else (2, pairs))
            if not case["interleaved"]:
                part = part.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
            y[:, :, h:h + 8, :2 * pairs] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return out


def exact_activation(v, activation, with_slope):
    """The activation of v, or its derivative there."""
    if activation == "relu":
        return torch.heaviside(v, torch.zeros((), device=v.device, dtype=v.dtype)) if with_slope else torch.relu(v)
    if activation == "gelu":
        below = 0.5 * torch.erfc(v / -math.sqrt(2.0))
        return below + v * torch.exp(v * v / -2.0) / math.sqrt(math.tau) if with_slope else v * below
    if activation == "gelu_tanh":
        inner = math.sqrt(8.0 / math.pi) * (v + 0.044715 * v ** 3)       # (1 + tanh(z)) / 2 is the sigmoid of 2 z
        share = torch.sigmoid(inner)
        if not with_slope:
            return v * share
        return share + v * share * torch.sigmoid(-inner) * math.sqrt(8.0 / math.pi) * (1.0 + 0.134145 * v ** 2)
    share = torch.sigmoid(v)
    return share * (1.0 + v * torch.sigmoid(-v)) if with_slope else v * share


def exact_linear(s):
    case = s["case"]
    if case["op"] == "linear":
        pre = torch.einsum("tk,nk->tn", s["x"].double(), s["weight"].double())
        if s["bias"] is not None:
            pre += s["bias"].double()
        y = pre if case["activation"] == "none" else exact_activation(pre, case["activation"], False)
        if s["residual"] is not None:
            y = y + s["residual"]
        return (y, pre) if case["keep"] else y
    d_pre = s["d_y"].double()
    if s["pre"] is not None:
        d_pre *= exact_activation(s["pre"].double(), case["activation"], True)
    d_weight, d_bias = torch.einsum("tn,tk->nk", d_pre, s["x"].double()), torch.einsum("tn->n", d_pre)
    d_x = torch.einsum("tn,nk->tk", d_pre, s["weight"].double())
    if s["below"] is not None:
        d_x *= exact_activation(s["below"].double(), case["below"], True)
    if s["residual"] is not None:
        d_x += s["residual"]
    return {"d_x": d_x, "d_weight": d_weight, "d_bias": d_bias}


def exact(case, seed):
    s = prepare(case, seed)
    return exact_norm(s) if case["op"].startswith("norm") else exact_rotary(s) if case["op"] == "rotary" else exact_linear(s)
