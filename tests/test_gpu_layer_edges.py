"""Layer norm, rotary positions and linear layers on the GPU where their parts meet: columns stored by lanes between copies, rows shared by
clusters, work buffers of the stated size, tails of activations, rows without spread.  Bounds are counted as in test_gpu_layer_operators.py."""
import math

import pytest
import torch

from test_gpu_layer_operators import whole_numbers
from test_gpu_train_operators import F, TYPES, normal, tiny_of, u_of, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    import paper_2601_02311_b200.ps as m
    return m


@pytest.fixture(scope="module")
def ctx(ps):
    return ps.Context(0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width", [259, 1003, 1285])
def test_last_columns_between_copies(ctx, dtype, width):
    """Tile after tile of a block, the last columns of each stored by lanes out of the buffers that the next tile's residual, and the values below it, are
    copied into.  Whole numbers, so that every result is exact."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(width)
    tokens, other = 30011, 72
    x, w = whole_numbers(gen, tokens, other, t), whole_numbers(gen, width, other, t)
    res, below = whole_numbers(gen, tokens, width, t, 9), whole_numbers(gen, tokens, width, t)
    want = (x.double() @ w.double().t() + res.double()).to(t)
    back = w.t().contiguous()
    d_want = ((x.double() @ back.double()) * (below > 0) + res.double()).to(t)
    for _ in range(3):
        y, pre = ctx.linear_forward(x, w, residual=res, keep=True)
        assert torch.equal(y, want) and torch.equal(pre, (x.double() @ w.double().t()).to(t))
        assert torch.equal(ctx.linear_forward(x, w, residual=res), want)
        d_x = whole_numbers(gen, tokens, width, t)
        weight = whole_numbers(gen, other, width, t).copy_(back)
        ctx.linear_backward_into(x, None, weight, d_x=d_x, below=below, below_activation="relu", residual=res)
        ctx.check_status()
        assert torch.equal(d_x, d_want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [4100, 8200, 12000, 16392, 33000, 65536])
def test_shared_rows_without_a_residual(ctx, dtype, cols):
    """A residual that is not there adds what one of zeros does, in every block that shares a row; with the columns' sums and without."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(cols)
    x, d_y, weight = normal(gen, 40, cols, dtype=t), normal(gen, 40, cols, dtype=t), normal(gen, cols, dtype=t)
    _, mean, rstd = ctx.layer_norm_forward(x, weight)
    want = ctx.layer_norm_backward(d_y, x, mean, rstd, weight, torch.zeros_like(x))[0]
    alone = torch.empty_like(x)
    ctx.layer_norm_backward_into(d_y, x, mean, rstd, alone, weight)
    with_sums = ctx.layer_norm_backward(d_y, x, mean, rstd, weight)[0]
    ctx.check_status()
    assert torch.equal(alone, want) and torch.equal(with_sums, want)


@pytest.mark.parametrize("activation", [None, "gelu"])
@pytest.mark.parametrize("wide", [None, torch.float32])
@pytest.mark.parametrize("named", [True, False])
def test_work_of_the_named_size(ctx, activation, wide, named):
    """Buffers of exactly the size that the binding names are taken, and are enough: the results are those of a call that allocates its own."""
    t, gen = torch.bfloat16, torch.Generator("cuda").manual_seed(5)
    x, w, d_y, pre = normal(gen, 700, 72, dtype=t), normal(gen, 120, 72, dtype=t), normal(gen, 700, 120, dtype=t), normal(gen, 700, 120, dtype=t)
    pre = None if activation is None else pre
    want = ctx.linear_backward(d_y, x, w, pre, activation, dtype=wide)
    got = [torch.empty_like(g) for g in want]
    size = ctx.linear_backward_bytes(700, 72, 120, activation, *([wide or t] if named else []))
    whole = torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda")
    ctx.linear_backward_into(d_y, x, w, *got, pre=pre, activation=activation, work=whole[256:256 + size])
    ctx.check_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and whole[:256].eq(77).all() and whole[256 + size:].eq(77).all()


@pytest.mark.parametrize("rows, cols", [(300, 64), (900, 1155), (100, 12000)])
def test_norm_work_of_the_named_size(ctx, rows, cols):
    gen = torch.Generator("cuda").manual_seed(cols)
    x, d_y = normal(gen, rows, cols), normal(gen, rows, cols)
    _, mean, rstd = ctx.layer_norm_forward(x)
    want = ctx.layer_norm_backward(d_y, x, mean, rstd, residual=d_y)
    got = [torch.empty_like(g) for g in want]
    size = ctx.layer_norm_backward_bytes(rows, cols, x.dtype)
    whole = torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda")
    ctx.layer_norm_backward_into(d_y, x, mean, rstd, got[0], None, d_y, *got[1:], work=whole[256:256 + size])
    ctx.check_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and whole[:256].eq(77).all() and whole[256 + size:].eq(77).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gelu_keeps_its_digits_far_out(ctx, dtype):
    """gelu and its slope against bounds relative to the results themselves, which are small on the negative side."""
    t = TYPES[dtype]
    v = torch.cat((torch.linspace(-13, 13, 1000), torch.tensor([-4.01, -6.0, -8.0, -3.0, -9.0, -0.75, 1e-3, -1e-3]))).cuda().to(t)
    n = v.numel()
    x = torch.zeros(n, 8, device="cuda", dtype=t)
    x[:, 0] = v
    one = torch.zeros(8, 8, device="cuda", dtype=t)
    one[:, 0] = 1
    y = ctx.linear_forward(x, one, activation="gelu")[:, 0]
    e = v.double()
    square = e.square() / 2
    tail, density = torch.erfc(e.abs() * math.sqrt(0.5)) / 2, (-square).exp() / math.sqrt(2 * math.pi)
    # the exponential: 2 units of 2 F, and three roundings of its argument, of F each; the polynomial 1.2e-6 = 20 F of the value and 2 F of its quotient; two
    # products.  Results below 2^-126 are 0
    exp_err = F * (4 + 3.4 * square)
    tail_err = tail * (exp_err + 24 * F) + 2.0 ** -126
    share = torch.where(e < 0, tail, 1 - tail)
    within(y, e * share, e.abs() * tail_err + 2 * F * (e * share).abs() + u_of(t) * (e * share).abs() + tiny_of(t), "gelu")
    pre = torch.zeros(4, n, device="cuda", dtype=t)
    pre[0] = v
    unit = torch.zeros_like(pre)
    unit[0] = 1
    slope = torch.empty(n, device="cuda")
    ctx.linear_backward_into(unit, None, None, d_bias=slope, pre=pre, activation="gelu")
    ctx.check_status()
    want = share + e * density
    within(slope, want, tail_err + (e * density).abs() * (exp_err + 4 * F) + 2 * F * (want.abs() + share), "slope")


SPREADS = [3, 7, 60, 250, 300, 1000, 1155, 2056, 5003, 9001, 12000, 16392, 20000, 33000, 70001]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", SPREADS)
def test_rows_of_one_number(ctx, dtype, cols):
    """Equal numbers are their own mean, whatever the sums' and the quotient's roundings: what comes out is the bias, bit by bit."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(cols)
    values = torch.tensor([0.0, 7.1, -100.0, 100.1, 12345.0, 1e4, -3e4, 0.3, 1e-3, 77777.0 if dtype != "f16" else 65504.0], device="cuda").to(t)
    x = values[:, None].expand(-1, cols).contiguous()
    weight, bias = normal(gen, cols, dtype=t), normal(gen, cols, dtype=t)
    y, mean, rstd = ctx.layer_norm_forward(x, weight, bias)
    ctx.check_status()
    assert torch.equal(y, bias.expand_as(y)) and torch.equal(mean, values.float())
    in_place = x.clone()
    ctx.layer_norm_forward_into(in_place, in_place, weight, bias)
    assert torch.equal(in_place, y)
    # the first mean is off by at most depth + 2 roundings; of that square the sums and products leave 6 F
    depth = max(32, -(-cols // 1024)) + 12
    within(rstd, torch.full_like(mean, 1e-5).double().rsqrt(), 10 ** 2.5 * (5 * F + 3 * F * (depth * F * values.double()) ** 2 / 1e-5))


@pytest.mark.parametrize("cols", SPREADS)
def test_rows_far_from_zero(ctx, cols):
    """Of a mean far above the spread only its last rounding is lost."""
    gen = torch.Generator("cuda").manual_seed(cols)
    x = torch.randint(-8, 9, (5, cols), device="cuda", generator=gen).float() + 12345.0
    y, m, rstd = ctx.layer_norm_forward(x)
    ctx.check_status()
    in_place = x.clone()
    ctx.layer_norm_forward_into(in_place, in_place)
    part = ctx.layer_norm_forward(torch.cat((x[3:], torch.zeros_like(x))))[0]          # beside rows that are not far
    ctx.check_status()
    assert torch.equal(in_place, y) and torch.equal(part[:2], y[3:])
    e = x.double()
    mean = e.mean(1, keepdim=True)
    apart, var = e - mean, e.var(1, keepdim=True, unbiased=False)
    root = (var + 1e-5).rsqrt()
    d = max(32, -(-cols // 1024)) + 12
    # the first mean is off by d F of it; distances from it are whole multiples of its unit and exact; their sum, the share and the second mean
    first = d * F * mean
    mean_err = F * mean + (d + 2) * F * (apart.abs().mean(1, keepdim=True) + first)
    root_err = root * (((d + 6) * F * (var + first ** 2) + mean_err ** 2) / (var + 1e-5) / 2 + 4 * F)
    within(m[:, None], mean, mean_err)
    within(rstd[:, None], root, root_err + F * root)
    within(y, apart * root, apart.abs() * (root_err + 4 * F * root) + mean_err * (root + root_err) + 2 * F * (apart * root).abs())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("activation", [None, "gelu"])
def test_long_sums_are_taken_in_short_ones(ctx, dtype, activation):
    """A gradient in 32 bits whose tiles each have a sum over all tokens, of positive terms: its mean error is that of 1536 tokens at a time."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(6)
    tokens, inputs, outputs = 40000, 1600, 1536                      # (156 tiles of 128 x 128: the sum is not cut into parts)
    x, d_y = normal(gen, tokens, inputs, dtype=t).abs_(), normal(gen, tokens, outputs, dtype=t).abs_()
    pre = None if activation is None else normal(gen, tokens, outputs, dtype=t).abs_()
    d_w = torch.empty(outputs, inputs, device="cuda")
    ctx.linear_backward_into(d_y, x, None, d_weight=d_w, pre=pre, activation=activation)
    ctx.check_status()
    d_pre, err = d_y.double(), torch.zeros((), device="cuda", dtype=torch.float64)
    if activation:
        v = pre.double()
        square = v.square() / 2
        tail, density, exp_err = torch.erfc(v * math.sqrt(0.5)) / 2, (-square).exp() / math.sqrt(2 * math.pi), F * (4 + 3.4 * square)
        # the slope as in test_gelu_keeps_its_digits_far_out, and the product with it
        err = d_pre * (tail * (exp_err + 24 * F) + v * density * (exp_err + 4 * F) + 2 * F * (2 - 2 * tail + v * density))
        d_pre = d_pre * (1 - tail + v * density)
        err = (err + F * d_pre).t() @ x.double()
        del v, square, tail, density, exp_err
    want = d_pre.t() @ x.double()
    off = (d_w.double() - want) / want
    # A step of 16 products adds them to the sum with each cut off at a quarter of a unit of the sum's last place, and the whole at a unit (products of 2^-13 and 2^-14
    # beside 2^11 are seen in whole sums of 15 or 16, those of 2^-15 not).  So it loses up to 16 / 4 + 1 = 5 units, half of that on average.  A unit is 2 F of
    # the sum at most.  Of a sum that grows evenly to T it is, on average over the way, (r - 2/3) / r^2 times 2 F T with r = T / 2^floor(log2 T), which is
    # 3/8 at most, at r = 4/3.  24 steps of the kernel are 96 of these: 96 * 2.5 * 0.75 F = 180 F on average, 96 * 5 F = 480 F for one that always loses
    # most (its units add up to half of 96 * 2 F).  A twentieth more, since the sums do not grow quite evenly.  The 27 sums of 1536 tokens are rounded to nearest: 14 F.
    # (With 64 steps at a time half precision lost 380 F on average, bfloat16, whose products are shorter, 150.)
    mean, most = 1.05 * 180 * F, 1.05 * 480 * F + 14 * F
    assert off.mean().abs() <= mean + (err / want).mean()
    # of dPre in two parts, a rounding of a rounding
    parts = 0.0 if activation is None else u_of(t) ** 2 + tiny_of(t) / 4096
    within(d_w, want, (most + parts) * want + err)
    # All entries lose alike, but for their sums' own sizes, a tenth of it; the parts' roundings vanish in so many terms, and 27 of the sums are 2 F.  One part alone
    # would spread by 2^-8 / sqrt(3 * 40000) in bfloat16, 190 F, in half precision by 24 F.
    assert off.std() <= 0.1 * 180 * F + 2 * F


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width", [64, 333, 1000])
def test_input_gradient_in_place_of_the_values_below(ctx, dtype, width):
    """d_x may be `below` itself, alone and with a residual."""
    t, gen = TYPES[dtype], torch.Generator("cuda").manual_seed(width)
    d_y, w = whole_numbers(gen, 3000, 72, t), whole_numbers(gen, 72, width, t)
    below, res = whole_numbers(gen, 3000, width, t), whole_numbers(gen, 3000, width, t, 9)
    for r in (None, res):
        want = ((d_y.double() @ w.double()) * (below > 0) + (0 if r is None else r.double())).to(t)
        into = whole_numbers(gen, 3000, width, t).copy_(below)
        ctx.linear_backward_into(d_y, None, w, d_x=into, below=into, below_activation="relu", residual=r)
        ctx.check_status()
        assert torch.equal(into, want)


def test_rows_far_apart(ctx):
    """Offsets past 32 bits: rows, heads and sequences whose distance is above 2^31 elements give the bits of contiguous ones."""
    t, gen = torch.bfloat16, torch.Generator("cuda").manual_seed(9)
    rows, apart = 4, (1 << 31) + 16
    whole = torch.empty((rows - 1) * apart + (1 << 16), dtype=t, device="cuda")
    taken = [0]

    def far(like):
        """The matrix with its rows far apart, beside those that have been placed so."""
        begin = taken[0]
        taken[0] += (like.shape[1] + 7) // 8 * 8
        return whole.as_strided(like.shape, (apart, 1), begin).copy_(like)
    for cols in (100, 1000, 12000):
        taken[0] = 0
        x, d_y, res = (normal(gen, rows, cols, dtype=t) for _ in range(3))
        weight = normal(gen, cols, dtype=t)
        y, mean, rstd = ctx.layer_norm_forward(x, weight)
        grads = ctx.layer_norm_backward(d_y, x, mean, rstd, weight, res)
        x, d_y, res, into = far(x), far(d_y), far(res), far(torch.zeros_like(x))
        ctx.layer_norm_forward_into(x, into, weight)
        assert torch.equal(into, y)
        got = [torch.empty_like(g) for g in grads[1:]]
        ctx.layer_norm_backward_into(d_y, x, mean, rstd, into, weight, res, *got)
        assert torch.equal(into, grads[0]) and all(torch.equal(a, b) for a, b in zip(got, grads[1:]))
    for inputs, outputs in ((72, 136), (75, 133)):
        taken[0] = 0
        x, w, d_y, pre, res = (whole_numbers(gen, *s, t) for s in ((rows, inputs), (rows, inputs), (rows, rows), (rows, outputs), (rows, outputs)))
        wide = whole_numbers(gen, outputs, inputs, t)
        d_out = whole_numbers(gen, rows, outputs, t)
        want, kept = ctx.linear_forward(x, wide, residual=res, activation="relu", keep=True)
        d_x, d_w, _ = ctx.linear_backward(d_out, x, wide, pre, "relu", residual=x)
        few = ctx.linear_forward(x, w)
        few_grads = ctx.linear_backward(d_y, x, w, dtype=torch.float32)
        y, p, r = far(want), far(kept), far(res)
        y.zero_(), p.zero_()
        x_far, w_far = far(x), far(w)
        ctx.linear_forward_into(x_far, wide, y, residual=r, activation="relu", pre=p)
        assert torch.equal(y, want) and torch.equal(p, kept)
        into = far(torch.zeros_like(x))
        got_w = torch.empty(outputs, (inputs + 7) // 8 * 8, device="cuda", dtype=t)[:, :inputs]
        ctx.linear_backward_into(far(d_out), x_far, wide, into, got_w, pre=far(pre), activation="relu", residual=x_far)
        assert torch.equal(into, d_x) and torch.equal(got_w, d_w)
        assert torch.equal(ctx.linear_forward(x_far, w_far), few)
        floats = whole.view(torch.float32).as_strided((rows, inputs), (apart // 2, 1), 1 << 14)
        ctx.linear_backward_into(d_y, x_far, w_far, d_weight=floats)
        assert torch.equal(floats, few_grads[1])
    q = normal(gen, rows, 5, 3, 64, dtype=t)
    want = ctx.rotary(q)
    for order in ((0, 1, 2, 3), (1, 0, 2, 3), (2, 1, 0, 3)):           # which of sequences, tokens and heads are far apart
        shape = [q.shape[i] for i in order]
        place = whole.as_strided([min(shape[0], rows)] + shape[1:], (apart, shape[2] * 64, 64, 1), 0).permute(*order)
        part = tuple(slice(0, n) for n in place.shape)
        place.copy_(q[part])
        ctx.rotary_into(place, place)
        assert torch.equal(place, want[part])
    ctx.check_status()
