"""Operators of a training step where sizes, types or the order of calls are at an edge, against their definitions
in 64 bits.  Bounds are counted as in test_gpu_train_operators.py."""
import math

import pytest
import torch

from test_gpu_train_operators import tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ps():
    import paper_2601_02311_b200.ps as m
    return m


@pytest.fixture(scope="module")
def ctx(ps):
    return ps.Context(0)


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len, k_len", [(0, 1), (0, 4096), (0, 4097), (0, 5000), (1, 0), (4096, 0), (4097, 0), (5000, 0), (0, 0)])
def test_attention_with_an_empty_side(ctx, dtype, dim, q_len, k_len):
    """No queries or no keys, before a side that may be long enough for chunks: every result there is, is zeros."""
    q, k, v, d_out = tensors(21, 2, q_len, k_len, 4, 2, dim, dtype)
    out, lse = ctx.attention_forward(q, k, v)
    assert out.eq(0).all() and lse.eq(-math.inf).all()
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    ctx.attention_backward_into(q, k, v, out, lse, d_out, *grads)
    ctx.check_status()
    assert all(g.eq(0).all() for g in grads)
    # and no error is left behind for the next launch to find
    assert torch.ones(8, device="cuda").sum().item() == 8
