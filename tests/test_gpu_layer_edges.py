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
