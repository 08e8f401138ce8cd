"""Layer norm, rotary positions and linear layers on the GPU, against their definitions in 64 bits.

Bounds are counted as in test_gpu_train_operators.py: u = eps / 2 of a type for one rounding to it, F = 2^-24 for one in
float32.  A sum whose terms pass through at most d additions is off by at most d F times the sum of their magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_train_operators import F, TYPES, normal, tiny_of, u_of, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    import paper_2601_02311_b200.ps as m
    return m


@pytest.fixture(scope="module")
def ctx(ps):
    return ps.Context(0)


def rounded(want, dtype):
    """What one rounding to the type adds to a bound."""
    return u_of(dtype) * want.abs() + tiny_of(dtype)


# ------------------------------------------------------------------ layer norm

def depth(cols):
    """Additions that a term of a row's sum passes through: 32 of a thread (its walk in wide rows), 10 between threads."""
    return max(32, -(-cols // 1024)) + 10


def norm_want(x, weight, bias, eps):
    x, cols = x.double(), x.shape[1]
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    w = torch.ones(cols, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    y = (x - mean) * rstd * w + b
    d = depth(cols) + 2
    mean_err = d * F * x.abs().mean(1, keepdim=True)
    # the squares are of distances from a mean that is off; their sum; eps, the root and the quotient
    rstd_err = rstd * (((d + 4) * F * var + mean_err.square()) / (var + eps) / 2 + 4 * F)
    err = w.abs() * ((x - mean).abs() * (rstd_err + 4 * F * rstd) + mean_err * rstd) + 2 * F * (y.abs() + b.abs())
    return y, mean, rstd, err, mean_err, rstd_err


NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (2, 31), (9, 128), (130, 768), (7, 1000), (3, 1024), (5, 1032), (3, 1155), (11, 2048), (2, 2056),
               (6, 4099), (3, 4104), (4, 5003), (2, 8192), (3, 8200), (2, 9001), (3, 16384), (2, 16392), (2, 20000), (2, 32768), (2, 32776), (1, 40001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", NORM_SHAPES)
def test_layer_norm(ctx, dtype, rows, cols):
    gen = torch.Generator("cuda").manual_seed(rows * 100003 + cols)
    x = normal(gen, rows, cols, dtype=TYPES[dtype], size=1.5) + 3.0
    weight, bias = normal(gen, cols, dtype=TYPES[dtype]), normal(gen, cols, dtype=TYPES[dtype])
    for w, b, eps in ((weight, bias, 1e-5), (None, None, 1e-6), (weight, None, 1e-5), (None, bias, 0.1)):
        want, mean, rstd, err, mean_err, rstd_err = norm_want(x, w, b, eps)
        y, m, r = ctx.layer_norm_forward(x, w, b, eps)
        ctx.check_status()
        within(y, want, err + rounded(want, x.dtype), "y")
        within(m, mean[:, 0], mean_err[:, 0] + F * mean[:, 0].abs(), "mean")
        within(r, rstd[:, 0], rstd_err[:, 0] + F * rstd[:, 0], "rstd")


def grad_want(d_y, x, mean, rstd, weight, residual):
    x, d_y, m, r = x.double(), d_y.double(), mean.double()[:, None], rstd.double()[:, None]
    rows, cols = x.shape
    w = torch.ones(cols, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    xn, g = (x - m) * r, d_y * w
    along, across = g.mean(1, keepdim=True), (g * xn).mean(1, keepdim=True)
    d_x = r * (g - along - xn * across)
    d = depth(cols) + 2
    err = r * (3 * F * g.abs() + (d + 1) * F * g.abs().mean(1, keepdim=True) + xn.abs() * (d + 4) * F * (g * xn).abs().mean(1, keepdim=True)
               + 6 * F * (xn * across).abs() + 3 * F * along.abs()) + 2 * F * d_x.abs()
    if residual is not None:
        d_x = d_x + residual.double()
        err = err + F * (d_x.abs() + residual.double().abs())
    # rows in order within blocks, then the blocks' sums: each term passes through fewer additions than there are rows and 16 more
    n = rows + 16
    return (d_x, err, (d_y * xn).sum(0), (n + 3) * F * (d_y * xn).abs().sum(0), d_y.sum(0), n * F * d_y.abs().sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", NORM_SHAPES + [(3000, 257), (1500, 768), (700, 4096), (701, 5003), (3001, 8), (200, 33000)])
def test_layer_norm_gradients(ctx, dtype, rows, cols):
    t = TYPES[dtype]
    gen = torch.Generator("cuda").manual_seed(rows * 7 + cols)
    x, d_y, res = normal(gen, rows, cols, dtype=t, size=1.5) + 0.5, normal(gen, rows, cols, dtype=t), normal(gen, rows, cols, dtype=t)
    weight = normal(gen, cols, dtype=t)
    _, mean, rstd = ctx.layer_norm_forward(x, weight)
    for w, residual, wide in ((weight, res, None), (None, None, torch.float32)):
        d_x, x_err, d_w, w_err, d_b, b_err = grad_want(d_y, x, mean, rstd, w, residual)
        got = ctx.layer_norm_backward(d_y, x, mean, rstd, w, residual, wide)
        ctx.check_status()
        within(got[0], d_x, x_err + rounded(d_x, t), "d_x")
        within(got[1], d_w, w_err + rounded(d_w, wide or t), "d_weight")
        within(got[2], d_b, b_err + rounded(d_b, wide or t), "d_bias")
        # the same bits again, and without the columns' sums
        again = ctx.layer_norm_backward(d_y, x, mean, rstd, w, residual, wide)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        alone = torch.empty_like(d_x, dtype=t)
        ctx.layer_norm_backward_into(d_y, x, mean, rstd, alone, w, residual)
        assert torch.equal(alone, got[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [768, 1155, 4100, 8192, 33000])
def test_layer_norm_gradients_add_up(ctx, dtype, cols):
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(cols)
    x, d_y = normal(gen, 37, cols, dtype=t), normal(gen, 37, cols, dtype=t)
    _, mean, rstd = ctx.layer_norm_forward(x)
    _, _, d_w, w_err, d_b, b_err = grad_want(d_y, x, mean, rstd, None, None)
    w0, b0 = normal(gen, cols), normal(gen, cols)
    got_w, got_b, only_b, d_x = w0.clone(), b0.clone(), b0.clone(), torch.empty_like(x)
    ctx.layer_norm_backward_into(d_y, x, mean, rstd, d_x, d_weight=got_w, d_bias=got_b, accumulate=True)
    ctx.layer_norm_backward_into(d_y, x, mean, rstd, d_x, d_bias=only_b, accumulate=True)
    ctx.check_status()
    within(got_w, d_w + w0.double(), w_err + F * (d_w + w0.double()).abs() + F * d_w.abs())
    within(got_b, d_b + b0.double(), b_err + F * (d_b + b0.double()).abs() + F * d_b.abs())
    assert torch.equal(got_b, only_b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols, offset, pitch", [(768, 0, 800), (768, 1, 801), (1155, 3, 1200), (4096, 8, 4104), (4096, 5, 4111), (33000, 1, 33001)])
def test_layer_norm_of_rows_in_a_larger_tensor(ctx, dtype, cols, offset, pitch):
    """Bits depend on the rows' values alone, not on where they lie; what lies around them is left alone; results may stand in
    their inputs' place."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(pitch)
    whole = [normal(gen, 9, pitch + 8, dtype=t) for _ in range(4)]
    x, d_y, res, out = (w[:, offset:offset + cols] for w in whole)
    weight, bias = (normal(gen, cols + 1, dtype=t)[1:] for _ in range(2))
    before = whole[3].clone()
    want = ctx.layer_norm_forward(x.contiguous(), weight.clone(), bias.clone())
    mean, rstd = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    ctx.layer_norm_forward_into(x, out, weight, bias, mean=mean, rstd=rstd)
    assert torch.equal(out, want[0]) and torch.equal(mean, want[1]) and torch.equal(rstd, want[2])
    grads = ctx.layer_norm_backward(d_y.contiguous(), x.contiguous(), mean, rstd, weight.clone(), res.contiguous())
    ctx.layer_norm_backward_into(d_y, x, mean, rstd, out, weight, res)
    assert torch.equal(out, grads[0])
    whole[3][:, offset:offset + cols] = before[:, offset:offset + cols]
    assert torch.equal(whole[3], before)
    for target in (d_y, x, res):
        kept, d_w, d_b = target.clone(), torch.empty_like(weight), torch.empty_like(bias)
        ctx.layer_norm_backward_into(d_y, x, mean, rstd, target, weight, res, d_w, d_b)
        assert torch.equal(target, grads[0]) and torch.equal(d_w, grads[1]) and torch.equal(d_b, grads[2])
        target.copy_(kept)
    ctx.layer_norm_forward_into(x, x, weight, bias)
    ctx.check_status()
    assert torch.equal(x, want[0])


@pytest.mark.parametrize("cols", [8, 1000, 5003])
def test_layer_norm_rows_do_not_see_each_other(ctx, cols):
    """A row's bits are its own: of any part of the rows, and beside rows of NaN and infinity."""
    gen = torch.Generator("cuda").manual_seed(cols)
    x, d_y = normal(gen, 400, cols, dtype=torch.bfloat16), normal(gen, 400, cols, dtype=torch.bfloat16)
    y, mean, rstd = ctx.layer_norm_forward(x)
    d_x = ctx.layer_norm_backward(d_y, x, mean, rstd)[0]
    part = ctx.layer_norm_forward(x[37:40])
    assert torch.equal(part[0], y[37:40])
    assert torch.equal(ctx.layer_norm_backward(d_y[37:40], x[37:40], mean[37:40], rstd[37:40])[0], d_x[37:40])
    bad = x.clone()
    bad[36], bad[40] = math.nan, math.inf
    got = ctx.layer_norm_forward(bad)[0]
    ctx.check_status()
    keep = [i for i in range(400) if i not in (36, 40)]
    assert torch.equal(got[keep], y[keep]) and got[36].isnan().all() and got[40].isnan().all()


def test_layer_norm_of_constant_and_far_rows(ctx):
    """Rows without spread have a deviation of sqrt(eps); a mean far above the spread costs nothing but the inputs' own digits."""
    x = torch.full((3, 4096), 7.0, device="cuda")
    y, mean, rstd = ctx.layer_norm_forward(x, eps=1e-4)
    assert y.eq(0).all() and mean.eq(7).all() and (rstd - 100).abs().max() < 100 * 4 * F + 1e-5
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.randint(-8, 9, (5, 4096), device="cuda", generator=gen).float() + 4096.0
    want, mean, rstd, err, _, _ = norm_want(x, None, None, 1e-5)
    y, _, _ = ctx.layer_norm_forward(x)
    # distances of whole numbers from a mean that is off by a rounding of 4096
    within(y, want, err + rounded(want, torch.float32))
    assert (y.double() - want).abs().max() < 1e-3


def test_layer_norm_of_no_rows(ctx):
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    y, mean, rstd = ctx.layer_norm_forward(x)
    d_x, d_w, d_b = ctx.layer_norm_backward(x, x, mean, rstd)
    wide = ctx.layer_norm_backward(torch.empty(0, 40000, device="cuda"), torch.empty(0, 40000, device="cuda"), mean, rstd)
    ctx.check_status()
    assert y.shape == x.shape and d_x.shape == x.shape and all(t.eq(0).all() for t in (d_w, d_b, wide[1], wide[2]))


def test_layer_norm_gradients_against_differences(ctx):
    """The gradients of sum(y * d_y) in float32, against central differences in 64 bits of the formula."""
    gen = torch.Generator("cuda").manual_seed(5)
    x, d_y, weight = normal(gen, 6, 50), normal(gen, 6, 50), normal(gen, 50)
    y, mean, rstd = ctx.layer_norm_forward(x, weight)
    d_x, d_w, d_b = ctx.layer_norm_backward(d_y, x, mean, rstd, weight)

    def value(x, w, b):
        x = x - x.mean(1, keepdim=True)
        return ((x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w + b) * d_y.double()).sum().item()
    step, args = 1e-5, [x.double(), weight.double(), torch.zeros(50, device="cuda", dtype=torch.float64)]
    for which, grad in enumerate((d_x, d_w, d_b)):
        for at in range(0, grad.numel(), 17):
            ends = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[at] += sign * step
                ends.append(value(*moved))
            # third derivatives here stay below 1e3, so the difference is off by less than 1e3 step^2; float32's sums by 1e-5
            assert abs((ends[0] - ends[1]) / (2 * step) - grad.view(-1)[at].item()) < 3e-5 * max(1.0, grad.abs().max().item())


# ------------------------------------------------------------------ rotary positions

def rotary_want(x, positions, first, base, dims, interleaved, factor, original, low, high, magnitude, inverse):
    """In 64 bits, the angles in the 64 bits of mantissa of a long double."""
    half = dims // 2
    f = np.longdouble(base) ** (-np.arange(half, dtype=np.longdouble) / half)
    if factor != 1.0:
        turns = original * f / (2 * np.longdouble(np.pi))
        s = np.clip((turns - low) / (high - low), 0, 1) if original else np.zeros_like(f)
        f = f * (s + (1 - s) / np.longdouble(factor))
    at = positions.cpu().numpy().astype(object) + first
    angle = np.array(at.tolist(), dtype=np.longdouble)[..., None] * f
    pi = np.longdouble("3.14159265358979323846264338327950288")
    angle = np.remainder(angle, 2 * pi)
    cos, sin = (torch.from_numpy(np.asarray(g(angle), dtype=np.float64)).cuda()[:, :, None] * magnitude for g in (np.cos, np.sin))
    if inverse:
        sin = -sin
    y = x.double().clone()
    a, b = (y[..., 0:dims:2], y[..., 1:dims:2]) if interleaved else (y[..., :half], y[..., half:dims])
    size = a.abs() + b.abs()
    a_new, b_new = a * cos - b * sin, b * cos + a * sin
    err = torch.zeros_like(y)
    if interleaved:
        y[..., 0:dims:2], y[..., 1:dims:2] = a_new, b_new
        err[..., 0:dims:2] = err[..., 1:dims:2] = size
    else:
        y[..., :half], y[..., half:dims] = a_new, b_new
        err[..., :half] = err[..., half:dims] = size
    # an angle of up to an eighth of a turn in a float (0.8 F), sine and cosine (2 units of 2 F at most), their product with the
    # magnitude, and two products and a sum
    err = 8 * F * abs(magnitude) * err
    err[..., :dims] += rounded(y[..., :dims], x.dtype)
    return y, err


ROTARY = dict(first=0, base=10000.0, dims=None, interleaved=False, factor=1.0, original=0.0, low=1.0, high=32.0, magnitude=1.0, inverse=False)


def check_rotary(ctx, q, k, positions, **how):
    how = dict(ROTARY, **how)
    batch, length, _, dim = q.shape
    at = torch.arange(length, device="cuda").expand(batch, length) if positions is None else positions.expand(batch, length)
    got = ctx.rotary(q, k, positions=positions, **how)
    ctx.check_status()
    how["dims"] = how["dims"] or dim
    for x, y in zip((q, k), got if k is not None else (got,)):
        want, err = rotary_want(x, at, **how)
        within(y, want, err)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim, dims", [(128, 128), (64, 64), (80, 80), (96, 64), (128, 32), (2, 2), (6, 4), (7, 6), (250, 250), (256, 256), (24, 16), (40, 20)])
def test_rotary(ctx, dtype, interleaved, dim, dims):
    gen = torch.Generator("cuda").manual_seed(dim + dims)
    for batch, length, heads, kv_heads in ((1, 1, 1, 1), (2, 33, 5, 2), (1, 70, 12, 0), (3, 5, 40, 8)):
        q = normal(gen, batch, length, heads, dim, dtype=TYPES[dtype])
        k = normal(gen, batch, length, kv_heads, dim, dtype=TYPES[dtype]) if kv_heads else None
        check_rotary(ctx, q, k, None, interleaved=interleaved, dims=dims)


@pytest.mark.parametrize("how", [dict(first=1 << 20), dict(first=-5), dict(first=(1 << 31) - 7), dict(first=-(1 << 40)), dict(base=500000.0, inverse=True),
                                 dict(factor=4.0), dict(factor=8.0, original=4096.0), dict(factor=8.0, original=100.0, low=1.0, high=4.0, magnitude=1.21),
                                 dict(magnitude=-0.5, inverse=True), dict(base=1.0), dict(factor=3.0, original=1e9)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_angles(ctx, how, interleaved):
    gen = torch.Generator("cuda").manual_seed(3)
    q, k = normal(gen, 2, 50, 3, 64), normal(gen, 2, 50, 1, 64)
    check_rotary(ctx, q, k, None, interleaved=interleaved, **how)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_rotary_positions(ctx, kind):
    gen = torch.Generator("cuda").manual_seed(4)
    q, k = normal(gen, 3, 40, 4, 32, dtype=torch.bfloat16), normal(gen, 3, 40, 2, 32, dtype=torch.bfloat16)
    far = torch.randint(-(1 << 31), 1 << 31, (3, 40), device="cuda", generator=gen)
    check_rotary(ctx, q, k, far.to(kind))
    check_rotary(ctx, q, k, far[0].to(kind), first=11)
    check_rotary(ctx, q, k, torch.cat((far, far), 1).to(kind)[:, 13:53])
    if kind == torch.int64:
        check_rotary(ctx, q, k, far * 500)
    # a shard of the sequence, and of the heads, has the whole one's bits
    whole = ctx.rotary(q, k)
    part = ctx.rotary(q[:, 25:, 1:3], k[:, 25:], first=25)
    assert torch.equal(part[0], whole[0][:, 25:, 1:3]) and torch.equal(part[1], whole[1][:, 25:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dims", [64, 40])
def test_rotary_in_place_and_strides(ctx, interleaved, dims):
    """Heads inside a packed projection, in their own place; any order of dimensions; broadcast heads; unaligned heads."""
    gen = torch.Generator("cuda").manual_seed(dims)
    how = dict(interleaved=interleaved, dims=dims)
    packed = normal(gen, 2, 30, 9, 64, dtype=torch.bfloat16)
    want = ctx.rotary(packed[:, :, :5].contiguous(), packed[:, :, 5:7].contiguous(), **how)
    before = packed.clone()
    ctx.rotary_into(packed[:, :, :5], packed[:, :, :5], packed[:, :, 5:7], packed[:, :, 5:7], **how)
    assert torch.equal(packed[:, :, :5], want[0]) and torch.equal(packed[:, :, 5:7], want[1]) and torch.equal(packed[:, :, 7:], before[:, :, 7:])
    # turned back
    back = ctx.rotary(packed[:, :, :7], inverse=True, **how)
    # two roundings, the second of a value that the first may have moved
    want = before[:, :, :7].double()
    within(back, want, 2.02 * u_of(torch.bfloat16) * (want.abs() + want.view(2, 30, 7, 64).norm(dim=-1, keepdim=True)))
    swapped = normal(gen, 3, 2, 30, 64).permute(1, 2, 0, 3)
    assert torch.equal(ctx.rotary(swapped, **how), ctx.rotary(swapped.contiguous(), **how))
    one = normal(gen, 2, 30, 1, 64).expand(2, 30, 4, 64)
    assert torch.equal(ctx.rotary(one, **how), ctx.rotary(one.contiguous(), **how))
    odd = normal(gen, 2, 30, 3, 67)[..., 1:65]
    out = torch.zeros(2, 30, 3, 67, device="cuda")
    ctx.rotary_into(odd, out[..., 2:66], **how)
    assert torch.equal(out[..., 2:66], ctx.rotary(odd.contiguous(), **how)) and out[..., :2].eq(0).all() and out[..., 66].eq(0).all()
    ctx.check_status()


def test_rotary_of_nothing(ctx):
    assert ctx.rotary(torch.empty(0, 5, 2, 8, device="cuda")).shape == (0, 5, 2, 8)
    assert ctx.rotary(torch.empty(2, 0, 2, 8, device="cuda")).shape == (2, 0, 2, 8)
    ctx.check_status()


# ------------------------------------------------------------------ linear layers

def matrix(gen, rows, cols, dtype, size=1.0, tail=math.nan):
    """Rows at multiples of 16 bytes, with something unusable behind each."""
    t = normal(gen, rows, (cols + 7) // 8 * 8, dtype=dtype, size=size)
    t[:, cols:] = tail
    return t[:, :cols]


def whole_numbers(gen, rows, cols, dtype, most=2):
    t = torch.full((rows, (cols + 7) // 8 * 8), math.nan, device="cuda", dtype=dtype)
    t[:, :cols] = torch.randint(-most, most + 1, (rows, cols), device="cuda", generator=gen).to(dtype)
    return t[:, :cols]


# tokens, inputs, outputs: tiles of 128 x 64, 128 x 128 and, by pairs, 256 x 256, with and without a rest in each direction
SHAPES = [(1, 8, 8), (1, 1, 1), (3, 5, 7), (1, 768, 768), (17, 64, 130), (128, 128, 128), (129, 72, 65), (200, 1000, 333), (384, 768, 2304), (1000, 70, 1200),
          (1, 2100, 9000), (1290, 136, 1290), (2500, 100, 2100), (2049, 328, 3333), (4097, 40, 2311)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens, inputs, outputs", SHAPES)
def test_linear_of_whole_numbers(ctx, dtype, tokens, inputs, outputs):
    """Sums of whole numbers are exact in 32 bits, so every result is the true one, rounded once."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(tokens + inputs)
    x, w, d_y = (whole_numbers(gen, *s, t) for s in ((tokens, inputs), (outputs, inputs), (tokens, outputs)))
    bias = torch.randint(-9, 10, (outputs,), device="cuda", generator=gen).to(t)
    res, in_res = whole_numbers(gen, tokens, outputs, t, 9), whole_numbers(gen, tokens, inputs, t, 9)
    sums = x.double() @ w.double().t()
    for b, r in ((None, None), (bias, res)):
        want = sums + (0 if b is None else b.double()) + (0 if r is None else r.double())
        assert torch.equal(ctx.linear_forward(x, w, b, residual=r), want.to(t))
    y, pre = ctx.linear_forward(x, w, bias, "relu", res, keep=True)
    assert torch.equal(pre, (sums + bias.double()).to(t)) and torch.equal(y, ((sums + bias.double()).clamp(min=0) + res.double()).to(t))
    for r, wide in ((None, None), (in_res, torch.float32)):
        d_x, d_w, d_b = ctx.linear_backward(d_y, x, w, residual=r, dtype=wide)
        ctx.check_status()
        assert torch.equal(d_x, (d_y.double() @ w.double() + (0 if r is None else r.double())).to(t))
        assert torch.equal(d_w, (d_y.double().t() @ x.double()).to(wide or t))
        assert torch.equal(d_b, d_y.double().sum(0).to(wide or t))
    # a gradient through relu is exact as well: of the layer's own, and of the one below
    at, below = whole_numbers(gen, tokens, outputs, t), whole_numbers(gen, tokens, inputs, t)
    d_x, d_w, d_b = ctx.linear_backward(d_y, x, w, at, "relu", below, "relu", in_res)
    d_pre = d_y.double() * (at > 0)
    assert torch.equal(d_x, ((d_pre @ w.double()) * (below > 0) + in_res.double()).to(t))
    assert torch.equal(d_w, (d_pre.t() @ x.double()).to(t)) and torch.equal(d_b, d_pre.sum(0).to(t))
    ctx.check_status()
