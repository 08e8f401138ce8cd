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
               (300, 2), (700, 6), (129, 33), (65, 200), (40, 255), (41, 257), (6, 4099), (3, 4104), (4, 5003), (2, 8192), (3, 8200), (2, 9001), (3, 16384), (2, 16392), (2, 20000), (2, 32768), (2, 32776), (1, 40001), (2, 65536), (3, 70000), (2, 70001)]


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
@pytest.mark.parametrize("rows, cols", NORM_SHAPES + [(3000, 257), (1500, 768), (700, 4096), (701, 5003), (3001, 8), (200, 33000), (500, 12000), (300, 70000)])
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


def activation_want(v, name, with_slope):
    """An activation or its derivative in 64 bits."""
    v = v.detach().clone().requires_grad_()
    y = {"none": lambda: v * 1.0, "relu": lambda: v.clamp(min=0.0), "gelu": lambda: v * 0.5 * torch.erfc(-v * math.sqrt(0.5)),
         "gelu_tanh": lambda: 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))), "silu": lambda: v * torch.sigmoid(v)}[name]()
    if not with_slope:
        return y.detach()
    return torch.where(v > 0, 1.0, 0.0).double() if name == "relu" else torch.autograd.grad(y.sum(), v)[0]


ACTIVATIONS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def products_err(a, b, dims):
    """Sums on the tensor cores: sixteen products at a time, then one sum after the other, bits cut off rather than rounded (2 F)."""
    return 2 * F * (dims / 16 + 16) * (a.double().abs() @ b.double().abs())


def function_err(v, name):
    """What the fast exponential (2 + 1.2 |argument| units of 2 F, arguments up to 1.6 |v| + 0.08 |v|^3 and up to 88), erf (1.5e-7, 2.6 F) and the
    few operations around them do to an activation, relative to 1 + |v|."""
    v = v.abs()
    argument = {"none": 0 * v, "relu": 0 * v, "gelu": v * v / 2, "gelu_tanh": 1.6 * v + 0.072 * v ** 3, "silu": v}[name].clamp(max=88)
    return 2 * F * (8 + 1.2 * argument) * (1 + v) * torch.where(argument >= 88, 0.0, 1.0) + 8 * F * (1 + v)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("tokens, inputs, outputs", [(3, 40, 70), (260, 200, 333), (1300, 264, 1301), (2500, 72, 2100)])
def test_linear(ctx, dtype, activation, tokens, inputs, outputs):
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(tokens)
    x, w = matrix(gen, tokens, inputs, t), matrix(gen, outputs, inputs, t, 2 * inputs ** -0.5)
    bias, res = normal(gen, outputs, dtype=t), matrix(gen, tokens, outputs, t)
    want = x.double() @ w.double().t() + bias.double()
    err = products_err(x, w.t(), inputs) + F * want.abs()
    y, pre = ctx.linear_forward(x, w, bias, activation, res, keep=True)
    within(pre, want, err + rounded(want, t), "pre")
    after = activation_want(want, activation, False)
    # every slope is below 1.13
    act_err = 1.13 * err + function_err(want, activation)
    within(y, after + res.double(), act_err + F * (after + res.double()).abs() + rounded(after + res.double(), t), "y")
    within(ctx.linear_forward(x, w, bias, activation), after, act_err + rounded(after, t), "y alone")
    ctx.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("activation, below", [("none", "none"), ("none", "gelu"), ("gelu", "none"), ("gelu_tanh", "silu"), ("silu", "gelu_tanh"), ("relu", "relu")])
@pytest.mark.parametrize("tokens, inputs, outputs", [(3, 40, 70), (333, 200, 260), (1300, 264, 1301), (5000, 130, 120), (2500, 2100, 72)])
def test_linear_gradients(ctx, dtype, activation, below, tokens, inputs, outputs):
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(tokens + outputs)
    x, w, d_y = matrix(gen, tokens, inputs, t), matrix(gen, outputs, inputs, t, inputs ** -0.5), matrix(gen, tokens, outputs, t)
    pre, under, res = matrix(gen, tokens, outputs, t, 2.0), matrix(gen, tokens, inputs, t, 2.0), matrix(gen, tokens, inputs, t)
    d_pre = d_y.double() * activation_want(pre.double(), activation, True)
    exact_err = d_y.double().abs() * function_err(pre.double(), activation) + F * d_pre.abs()        # before it is rounded
    pre_err = exact_err + (rounded(d_pre, t) if activation != "none" else 0.0)
    slopes = activation_want(under.double(), below, True)
    for wide in (None, torch.float32):
        d_x, d_w, d_b = ctx.linear_backward(d_y, x, w, None if activation == "none" else pre, activation, None if below == "none" else under, below,
                                            res, wide)
        ctx.check_status()
        sums = d_pre @ w.double()
        want = sums * slopes + res.double()
        err = (products_err(d_pre, w, outputs) + pre_err @ w.double().abs()) * slopes.abs() + sums.abs() * function_err(under.double(), below)
        within(d_x, want, 1.01 * err + 2 * F * want.abs() + F * sums.abs() + rounded(want, t), "d_x")
        want = d_pre.t() @ x.double()
        # in 32 bits dPre comes in two parts: what is left out is a rounding of a rounding, of a number 2^12 times as large
        left = exact_err + (u_of(t) * rounded(d_pre, t) + tiny_of(t) / 4096 if activation != "none" else 0.0) if wide else pre_err
        err = 2 * products_err(d_pre.t(), x, tokens) + left.t() @ x.double().abs()
        within(d_w, want, err + 2 * F * want.abs() + rounded(want, wide or t), "d_weight")
        want = d_pre.sum(0)
        within(d_b, want, exact_err.sum(0) + (tokens + 64) * F * d_pre.abs().sum(0) + rounded(want, wide or t), "d_bias")
        again = ctx.linear_backward(d_y, x, w, None if activation == "none" else pre, activation, None if below == "none" else under, below, res, wide)
        assert all(torch.equal(a, b) for a, b in zip((d_x, d_w, d_b), again))


def test_linear_gradients_against_differences(ctx):
    """Of sum(y * d_y) through a gelu, against central differences in 64 bits."""
    gen = torch.Generator("cuda").manual_seed(8)
    x, w, d_y = matrix(gen, 20, 24, torch.float16), matrix(gen, 16, 24, torch.float16, 0.3), matrix(gen, 20, 16, torch.float16)
    bias = normal(gen, 16, dtype=torch.float16)
    _, pre = ctx.linear_forward(x, w, bias, "gelu", keep=True)
    grads = ctx.linear_backward(d_y, x, w, pre, "gelu", dtype=torch.float32)
    args = [a.double().contiguous() for a in (x, w, bias)]

    def value(x, w, b):
        return (activation_want(x @ w.t() + b, "gelu", False) * d_y.double()).sum().item()
    for which, grad in enumerate(grads):
        grad = grad.double().contiguous()
        for at in range(0, grad.numel(), 13):
            ends = []
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[which].view(-1)[at] += sign * 1e-4
                ends.append(value(*moved))
            # pre is rounded to 2^-11 of up to 5, a slope changes by at most 0.8 of that; d_x is rounded; sums of at most 20 such terms of up to 12
            assert abs((ends[0] - ends[1]) / 2e-4 - grad.view(-1)[at].item()) < 20 * 12 * 0.8 * 5 * 2.0 ** -11


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_linear_rows_and_columns_do_not_see_each_other(ctx, dtype):
    """The bits of a row, and of a column, are those of a call that has it alone: in tiles of every shape, beside rows of NaN."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(2)
    x, w = matrix(gen, 2600, 520, t), matrix(gen, 2304, 520, t)
    bias, res = normal(gen, 2304, dtype=t), matrix(gen, 2600, 2304, t)
    y = ctx.linear_forward(x, w, bias, "gelu", res)
    for rows, cols in ((slice(0, 1), slice(0, 2304)), (slice(700, 829), slice(0, 200)), (slice(3, 1003), slice(1000, 2200)), (slice(0, 2600), slice(2300, 2304)),
                       (slice(100, 2148), slice(0, 1600))):
        at = matrix(gen, rows.stop - rows.start, cols.stop - cols.start, t).copy_(res[rows, cols])
        part = ctx.linear_forward(x[rows], w[cols], bias[cols], "gelu", at)
        assert torch.equal(part, y[rows, cols])
    d_y = matrix(gen, 2600, 2304, t)
    below = matrix(gen, 2600, 520, t)
    d_x = ctx.linear_backward(d_y, x, w, below=below, below_activation="silu")[0]
    for rows in (slice(5, 6), slice(64, 200), slice(1000, 2600)):
        part = torch.empty_like(x[rows])
        ctx.linear_backward_into(d_y[rows], None, w, d_x=part, below=below[rows], below_activation="silu")
        assert torch.equal(part, d_x[rows])
    bad = x.clone()
    bad[77] = math.nan
    got = ctx.linear_forward(bad, w, bias, "gelu", res)
    ctx.check_status()
    keep = torch.arange(2600, device="cuda") != 77
    assert torch.equal(got[keep], y[keep]) and got[77].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_linear_into_larger_tensors(ctx, dtype):
    """What lies around a result is left alone; a residual may be the result; parts of the gradients; added to what is there."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(3)
    whole = {n: normal(gen, r, c, dtype=t) for n, r, c in (("x", 150, 200), ("w", 140, 200), ("y", 150, 304), ("pre", 150, 304), ("dx", 150, 200))}
    x, w, y, pre = whole["x"][5:138, 16:165], whole["w"][2:133, 8:157], whole["y"][1:134, 8:139], whole["pre"][7:140, 160:291]
    before = {n: v.clone() for n, v in whole.items()}
    start = y.clone()
    bias = normal(gen, 140, dtype=t)[3:134]
    want = ctx.linear_forward(x, w, bias, "silu", matrix(gen, 133, 131, t).copy_(start), keep=True)
    ctx.linear_forward_into(x, w, y, bias, "silu", residual=y, pre=pre)
    assert torch.equal(y, want[0]) and torch.equal(pre, want[1])
    d_x, d_w, d_b = ctx.linear_backward(y, x, w, pre, "silu", residual=x)
    into = whole["dx"][5:138, 16:165]
    into.copy_(x)
    wide_w, wide_b = normal(gen, 131, 152)[:, :149], normal(gen, 131)
    w0, b0 = wide_w.clone(), wide_b.clone()
    ctx.linear_backward_into(y, None, w, d_x=into, pre=pre, activation="silu", residual=into)
    exact_w, exact_b = ctx.linear_backward(y, x, w, pre, "silu", dtype=torch.float32)[1:]
    ctx.linear_backward_into(y, x, None, d_weight=wide_w, d_bias=wide_b, pre=pre, activation="silu", accumulate=True)
    assert torch.equal(into, d_x) and torch.equal(wide_w, exact_w + w0) and torch.equal(wide_b, exact_b + b0)
    only = torch.empty_like(d_b)
    ctx.linear_backward_into(y, None, None, d_bias=only, pre=pre, activation="silu")
    assert torch.equal(only, d_b)
    narrow_w = matrix(gen, 131, 149, t)
    n0 = narrow_w.clone()
    ctx.linear_backward_into(y, x, None, d_weight=narrow_w, accumulate=True)
    plain_w = ctx.linear_backward(y, x, w, dtype=torch.float32)[1]
    ctx.check_status()
    assert torch.equal(narrow_w, (plain_w + n0.float()).to(t))
    for n, (r, c) in dict(y=(slice(1, 134), slice(8, 139)), pre=(slice(7, 140), slice(160, 291)), dx=(slice(5, 138), slice(16, 165))).items():
        whole[n][r, c] = before[n][r, c]
        assert torch.equal(whole[n], before[n])


@pytest.mark.parametrize("inputs, outputs", [(1603, 1500), (1600, 1501), (2200, 2300)])
def test_weight_gradients_of_several_sums(ctx, inputs, outputs):
    """More tokens than a sum in 32 bits takes at a time: the tile is read and added to, where it was written by boxes and where by lanes.
    Whole numbers, so that the result is exact."""
    t, gen = torch.bfloat16, torch.Generator("cuda").manual_seed(inputs)
    x, d_y, pre = whole_numbers(gen, 9000, inputs, t), whole_numbers(gen, 9000, outputs, t), whole_numbers(gen, 9000, outputs, t)
    old = torch.zeros(outputs, (inputs + 7) // 8 * 8, device="cuda")
    old.copy_(torch.randint(-99, 100, old.shape, device="cuda", generator=gen))
    for activation in (None, "relu"):
        d_pre = d_y.double() * (1 if activation is None else pre > 0)
        want = d_pre.t() @ x.double()
        into, around = old.clone(), old.clone()
        ctx.linear_backward_into(d_y, x, None, d_weight=into[:, :inputs], pre=pre, activation=activation)
        assert torch.equal(into[:, :inputs], want.float())
        ctx.linear_backward_into(d_y, x, None, d_weight=around[:, :inputs], pre=pre, activation=activation, accumulate=True)
        ctx.check_status()
        assert torch.equal(around[:, :inputs], (want + old[:, :inputs].double()).float())
        assert torch.equal(into[:, inputs:], old[:, inputs:]) and torch.equal(around[:, inputs:], old[:, inputs:])


def test_linear_of_no_tokens(ctx):
    x, w = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), torch.ones(32, 64, device="cuda", dtype=torch.bfloat16)
    y = ctx.linear_forward(x, w)
    d_x, d_w, d_b = ctx.linear_backward(y, x, w, y, "gelu", dtype=torch.float32)
    kept = torch.ones(32, 64, device="cuda")
    ctx.linear_backward_into(y, x, w, d_weight=kept, accumulate=True)
    ctx.check_status()
    assert y.shape == (0, 32) and d_x.shape == (0, 64) and d_w.eq(0).all() and d_b.eq(0).all() and kept.eq(1).all()


@pytest.mark.parametrize("activation", ACTIVATIONS[1:])
def test_activations_far_out(ctx, activation):
    """Large arguments and infinities: an activation and its slope go to their limits."""
    v = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 9.0, -9.0, 30.0, -30.0, 88.0, -88.0, 1e3, -1e3, 1e4, -1e4], device="cuda", dtype=torch.bfloat16)
    x = torch.zeros(16, 16, device="cuda", dtype=torch.bfloat16)
    x[:14, 0] = v
    one = torch.zeros(8, 16, device="cuda", dtype=torch.bfloat16)
    one[:, 0] = 1
    y, pre = ctx.linear_forward(x, one, activation=activation, keep=True)
    assert torch.equal(pre[:14, 0], v)
    want = activation_want(v.double(), activation, False)
    # 1 + erf is off by what erf near -1 is, 2 units of 2^-24, however small it is itself: the bound is on the difference, not relative to it
    within(y[:14, 0], want, rounded(want, torch.bfloat16) + function_err(v.double(), activation))
    d_b = torch.empty(16, device="cuda")
    wide = torch.zeros(8, 16, device="cuda", dtype=torch.bfloat16)
    wide[0, :14] = v
    unit = torch.zeros_like(wide)
    unit[0] = 1
    ctx.linear_backward_into(unit, None, None, d_bias=d_b, pre=wide, activation=activation)
    ctx.check_status()
    slope = activation_want(v.double(), activation, True)
    slope = torch.where(slope.isnan(), (v > 0).double(), slope)              # (a product of 0 and infinity in the definition)
    within(d_b[:14], slope, function_err(v.double(), activation) * (1 + v.double().abs()).clamp(max=10.0) + 1e-30)


# ------------------------------------------------------------------ together

def test_operators_on_streams_and_in_graphs(ps):
    """Two contexts on two streams at once, and calls captured into a graph and replayed on other inputs."""
    gen = torch.Generator("cuda").manual_seed(9)
    base = ps.Context(0)
    x, w, d_y = matrix(gen, 1000, 512, torch.bfloat16), matrix(gen, 768, 512, torch.bfloat16), matrix(gen, 1000, 768, torch.bfloat16)
    scale = normal(gen, 512, dtype=torch.bfloat16)

    def step(ctx, x, d_y):
        n, mean, rstd = ctx.layer_norm_forward(x, scale)
        q = ctx.rotary(n.view(1, 1000, 4, 128))
        y, pre = ctx.linear_forward(q.view(1000, 512), w, activation="gelu", keep=True)
        d_q, d_w, d_b = ctx.linear_backward(d_y, q.view(1000, 512), w, pre, "gelu", dtype=torch.float32)
        d_n = ctx.rotary(d_q.view(1, 1000, 4, 128), inverse=True).view(1000, 512)
        return (y, d_w, d_b) + ctx.layer_norm_backward(d_n, x, mean, rstd, scale, residual=x)
    inputs = [(x, d_y), (x * 2 - 0.5, d_y * 0.5)]
    want = [step(base, *i) for i in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    contexts = [ps.Context(0, s) for s in streams]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for i, (s, c) in enumerate(zip(streams, contexts)):
            with torch.cuda.stream(s):
                got[i].append(step(c, *inputs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for run in got[i] for a, b in zip(run, want[i]))
    hold = [t.clone() for t in inputs[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        step(contexts[0], *hold)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        out = step(contexts[0], *hold)
    for i in (1, 0, 1):
        for to, t in zip(hold, inputs[i]):
            to.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    for c in contexts + [base]:
        c.check_status()


def test_a_layer_of_a_transformer(ctx):
    """Norm, projections, rotary positions, attention and a feed-forward layer, and all of their gradients, against
    autograd in 64 bits.  Every tensor between two operators is rounded to bfloat16."""
    gen = torch.Generator("cuda").manual_seed(12)
    t, batch, length, heads, kv_heads, dim = torch.bfloat16, 2, 200, 4, 2, 64
    hidden, rows = heads * dim, batch * length
    x = normal(gen, rows, hidden, dtype=t)
    p = dict(n1=1 + normal(gen, hidden, size=0.1), b1=normal(gen, hidden, size=0.1), qkv=normal(gen, (heads + 2 * kv_heads) * dim, hidden, size=hidden ** -0.5),
             out=normal(gen, hidden, hidden, size=hidden ** -0.5), bo=normal(gen, hidden, size=0.1), n2=1 + normal(gen, hidden, size=0.1),
             b2=normal(gen, hidden, size=0.1), up=normal(gen, 4 * hidden, hidden, size=hidden ** -0.5), bu=normal(gen, 4 * hidden, size=0.1),
             down=normal(gen, hidden, 4 * hidden, size=(4 * hidden) ** -0.5), bd=normal(gen, hidden, size=0.1))
    p = {k: v.to(t) for k, v in p.items()}
    d_out = normal(gen, rows, hidden, dtype=t)

    n1, mean1, rstd1 = ctx.layer_norm_forward(x, p["n1"], p["b1"])
    qkv = ctx.linear_forward(n1, p["qkv"]).view(batch, length, heads + 2 * kv_heads, dim)
    q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads], qkv[:, :, heads + kv_heads:]
    ctx.rotary_into(q, q, k, k)
    o, lse = ctx.attention_forward(q, k, v)
    h = ctx.linear_forward(o.view(rows, hidden), p["out"], p["bo"], residual=x)
    n2, mean2, rstd2 = ctx.layer_norm_forward(h, p["n2"], p["b2"])
    a, pre = ctx.linear_forward(n2, p["up"], p["bu"], "gelu", keep=True)
    y = ctx.linear_forward(a, p["down"], p["bd"], residual=h)

    g = {}
    d_pre, g["down"], g["bd"] = ctx.linear_backward(d_out, a, p["down"], below=pre, below_activation="gelu")
    d_n2, g["up"], g["bu"] = ctx.linear_backward(d_pre, n2, p["up"])
    d_h, g["n2"], g["b2"] = ctx.layer_norm_backward(d_n2, h, mean2, rstd2, p["n2"], residual=d_out)
    d_o, g["out"], g["bo"] = ctx.linear_backward(d_h, o.view(rows, hidden), p["out"])
    d_qkv = torch.empty_like(qkv)
    d_q, d_k, d_v = d_qkv[:, :, :heads], d_qkv[:, :, heads:heads + kv_heads], d_qkv[:, :, heads + kv_heads:]
    ctx.attention_backward_into(q, k, v, o, lse, d_o.view_as(o), d_q, d_k, d_v)
    ctx.rotary_into(d_q, d_q, d_k, d_k, inverse=True)
    d_n1, g["qkv"], _ = ctx.linear_backward(d_qkv.view(rows, -1), n1, p["qkv"])
    g["x"], g["n1"], g["b1"] = ctx.layer_norm_backward(d_n1, x, mean1, rstd1, p["n1"], residual=d_h)
    ctx.check_status()

    e = {k: v.double().requires_grad_() for k, v in p.items()}
    e["x"] = x.double().requires_grad_()

    def layer_norm(x, w, b):
        x = x - x.mean(1, keepdim=True)
        return x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w + b
    at = torch.arange(length, device="cuda", dtype=torch.float64)[:, None, None] * 10000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))

    def turn(x):
        a, b = x[..., :dim // 2], x[..., dim // 2:]
        return torch.cat((a * at.cos() - b * at.sin(), b * at.cos() + a * at.sin()), -1)
    z = (layer_norm(e["x"], e["n1"], e["b1"]) @ e["qkv"].t()).view(batch, length, -1, dim)
    eq, ek, ev = (u.transpose(1, 2) for u in (turn(z[:, :, :heads]), turn(z[:, :, heads:heads + kv_heads]), z[:, :, heads + kv_heads:]))
    ek, ev = (u.repeat_interleave(heads // kv_heads, 1) for u in (ek, ev))
    s = (eq @ ek.transpose(-1, -2) * dim ** -0.5).masked_fill(torch.ones(length, length, device="cuda").triu(1).bool(), -math.inf)
    eo = (torch.softmax(s, -1) @ ev).transpose(1, 2).reshape(rows, hidden)
    eh = eo @ e["out"].t() + e["bo"] + e["x"]
    ea = activation_slow_gelu(layer_norm(eh, e["n2"], e["b2"]) @ e["up"].t() + e["bu"])
    ey = ea @ e["down"].t() + e["bd"] + eh
    ey.backward(d_out.double())
    # a tensor on the way is off by 2^-9 at most, relative and mostly evenly spread, and no path has more than 16 of them; they add up as squares
    assert (y.double() - ey.detach()).norm() <= 4 * 2.0 ** -9 * ey.detach().norm()
    for name, grad in g.items():
        assert (grad.double() - e[name].grad).norm() <= 2 * 4 * 2.0 ** -9 * e[name].grad.norm(), name


def activation_slow_gelu(v):
    return v * 0.5 * torch.erfc(-v * math.sqrt(0.5))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_sums_keep_32_bits(ctx, dtype):
    """A gradient in 32 bits over many tokens: what the tensor cores cut off does not add up.  All terms are positive, so that a
    sum's every step is a large one."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(4)
    x, d_y = matrix(gen, 40000, 72, t).abs_(), matrix(gen, 40000, 136, t).abs_()
    want = d_y.double().t() @ x.double()
    for outputs in (136, 8):
        _, d_w, _ = ctx.linear_backward(d_y[:, :outputs], x, torch.zeros(outputs, 72, device="cuda", dtype=t), dtype=torch.float32)
        ctx.check_status()
        # at most 256 additions of 16 products a time, cut off (2 F each, relative to a sum that grows evenly: half of that), and at most 40 such sums
        within(d_w, want[:outputs], (256 + 16 + 2 * 20) * F * want[:outputs])


def test_products_beside_attention(ps):
    """Kernels that each take all of an SM's tensor memory, from two streams at once."""
    gen = torch.Generator("cuda").manual_seed(31)
    x, w = matrix(gen, 3000, 520, torch.bfloat16), matrix(gen, 2000, 520, torch.bfloat16)
    d_y = matrix(gen, 3000, 2000, torch.bfloat16)
    q = normal(gen, 2, 700, 6, 128, dtype=torch.bfloat16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [ps.Context(0, s) for s in streams]

    def layer(c):
        return (c.linear_forward(x, w, activation="silu"),) + c.linear_backward(d_y, x, w, dtype=torch.float32)

    def attend(c):
        out, lse = c.attention_forward(q, q, q)
        return (out, lse) + c.attention_backward(q, q, q, out, lse, q)
    torch.cuda.synchronize()
    want = []
    for f, c, s in zip((layer, attend), contexts, streams):
        with torch.cuda.stream(s):
            want.append(f(c))
        torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, (f, c, s) in enumerate(zip((layer, attend), contexts, streams)):
            with torch.cuda.stream(s):
                got[i].append(f(c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for run in got[i] for a, b in zip(run, want[i]))
    for c in contexts:
        c.check_status()
