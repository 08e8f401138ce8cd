"""Which results may lie where: a call is refused where a result meets an operand that is still read, or another result, and where it meets neither it is
not.  Without a GPU: in the context used here a kernel has reported a problem, so a call that passes all checks of its arguments ends as E_DEVICE."""
import ctypes as C
import random

import pytest

import paper_2601_02311_b200.ps as ps
import test_layer_refusals as t
from test_train_refusals import AT

REPORTED = C.create_string_buffer(b"\1" * 4096, 4096)
CONTEXT = (C.c_void_p * 64)(*[C.addressof(REPORTED)] * 64)
CTX = C.cast(CONTEXT, C.c_void_p)
TAKEN = ps.E_DEVICE


def answer(call, **change):
    return call(ctx=CTX, **change)


def test_distinct_operands_are_taken():
    assert answer(t.linear) == TAKEN and answer(t.linear_grad) == TAKEN


# where the operands of t.linear lie: x AT (64 bytes), weight AT + 1024 (256), residual AT + 2048 (128), y AT + 3328, pre AT + 4096, bias AT + 5120 (32)
@pytest.mark.parametrize("change", [
    dict(y=(AT + 16, None)), dict(y=(AT - 112, None)), dict(y=(AT + 1024, None)), dict(y=(AT + 1024 + 240, None)), dict(y=(AT + 5120, None)),
    dict(y=(AT + 4096 + 112, None)), dict(pre=(AT, None)), dict(pre=(AT + 48, None)), dict(pre=(AT + 1024 + 16, None)), dict(pre=(AT + 5120 - 112, None)),
    dict(pre=(AT + 2048 + 16, None)), dict(y=(AT + 2048, 24)), dict(y=(AT, 64)),
    # columns of one buffer whose last ones meet
    dict(x=(AT, 64), y=(AT, 64)), dict(x=(AT + 16, 64), y=(AT, 64)), dict(x=(AT, 64), y=(AT + 104 + 8, 64), outputs=12),
    # a single row of each
    dict(tokens=1, y=(AT, 0)), dict(tokens=1, y=(AT + 1024 + 32, 0))])
def test_linear_refuses_results_over_operands(change):
    assert answer(t.linear, **change) == ps.E_RANGE


@pytest.mark.parametrize("change", [
    dict(y=(AT + 2048, None)), dict(y=(AT + 64, None)), dict(y=(AT - 128, None)), dict(y=(AT + 1024 - 128, None)), dict(y=(AT + 1024 + 256, None)),
    # column ranges of one buffer: x before y, behind it, and around pre
    dict(x=(AT, 64), y=(AT + 16, 64)), dict(x=(AT + 32, 64), y=(AT, 64)), dict(x=(AT, 64), y=(AT + 16, 64), pre=(AT + 48, 64), residual=(AT + 80, 64)),
    # rows in turns
    dict(x=(AT, 32), y=(AT + 32, 32)),
    dict(tokens=1, x=(AT, 0), y=(AT + 16, 0)), dict(tokens=1, residual=(AT + 3328, 7))])
def test_linear_takes_results_beside_operands(change):
    assert answer(t.linear, **change) == TAKEN


# d_y AT (128 bytes), x AT + 1024 (64), weight AT + 2048 (256), pre AT + 3328 (128), below AT + 4096 (64), residual AT + 5120 (64), d_x AT + 6144 (64),
# d_weight AT + 7168 (512), d_bias AT + 8192 (64)
@pytest.mark.parametrize("change", [
    dict(d_x=(AT + 16, None)), dict(d_x=(AT - 48, None)), dict(d_x=(AT + 1024 + 48, None)), dict(d_x=(AT + 2048, None)), dict(d_x=(AT + 2048 + 240, None)),
    dict(d_x=(AT + 4096 + 16, None)), dict(d_x=(AT + 5120 - 16, None)), dict(d_x=(AT + 7168 + 16, None)), dict(d_x=(AT + 8192 + 32, None)),
    dict(d_weight=(AT, None)), dict(d_weight=(AT + 1024 - 496, None)), dict(d_weight=(AT + 2048, None)), dict(d_weight=(AT + 4096 + 32, None)),
    dict(d_weight=(AT + 5120, None)), dict(d_weight=(AT + 6144 + 16, None)), dict(d_weight=(AT + 8192 - 496, None)),
    dict(d_bias=AT), dict(d_bias=AT + 1024 + 60), dict(d_bias=AT + 2048), dict(d_bias=AT + 3328 + 124), dict(d_bias=AT + 4096), dict(d_bias=AT + 5120 - 60),
    dict(d_bias=AT + 6144), dict(d_bias=AT + 7168 + 508)])
def test_linear_gradients_refuse_results_over_operands(change):
    assert answer(t.linear_grad, **change) == ps.E_RANGE


@pytest.mark.parametrize("change", [
    dict(d_x=(AT + 5120, None)), dict(d_x=(AT + 4096, None)), dict(d_x=(AT + 4096, None), residual=(AT + 4096, None)), dict(d_x=(AT + 128, None)),
    dict(d_x=(AT, 64), d_y=(AT + 16, 64)), dict(x=None, d_weight=None, d_x=(AT + 1024, None)), dict(weight=None, d_x=None, d_weight=(AT + 2048, None)),
    dict(d_x=(AT + 3328, None)), dict(d_weight=(AT + 7168 + 512, None)), dict(d_weight=None, d_bias=AT + 7168), dict(residual=None, d_x=(AT + 5120 + 16, None))])
def test_linear_gradients_take_results_beside_operands(change):
    assert answer(t.linear_grad, **change) == TAKEN


def elements(at, stride, rows, cols, width):
    return {at + r * stride * width + b for r in range(rows) for b in range(0, cols * width, 2)}


@pytest.mark.parametrize("seed", range(12))
def test_linear_overlaps_against_the_elements_themselves(seed):
    """Matrices anywhere in a small arena, of the same and of other strides."""
    rng = random.Random(seed)
    seen = set()
    for _ in range(400):
        tokens, inputs, outputs = rng.choice([1, 2, 5]), rng.choice([1, 8, 13]), rng.choice([3, 8, 20])
        shape = dict(x=(tokens, inputs), weight=(outputs, inputs), residual=(tokens, outputs), y=(tokens, outputs), pre=(tokens, outputs))
        common = 8 * rng.randint(3, 12)
        at = {n: (AT + 16 * rng.randint(0, 500), common if rng.random() < 0.6 else 8 * rng.randint(3, 12)) for n in shape}
        if rng.random() < 0.3:
            at["residual"] = at["y"]
        for n in ("residual", "pre"):
            if rng.random() < 0.3:
                at[n] = None
        bias = AT + 2 * rng.randint(0, 4000)
        e = {n: set() if at[n] is None else elements(*at[n], *shape[n], 2) for n in shape}
        e["bias"] = elements(bias, 0, 1, outputs, 2)
        same = at["residual"] is not None and at["residual"][0] == at["y"][0] and (tokens == 1 or at["residual"][1] == at["y"][1])
        bad = any(e["y"] & e[n] for n in ("x", "weight", "bias", "pre")) or any(e["pre"] & e[n] for n in ("x", "weight", "bias", "residual")) or \
            bool(e["y"] & e["residual"] and not same)
        got = answer(t.linear, tokens=tokens, inputs=inputs, outputs=outputs, bias=bias, **at)
        assert got == (ps.E_RANGE if bad else TAKEN), (tokens, inputs, outputs, at, bias)
        seen.add(got)
    assert seen == {ps.E_RANGE, TAKEN}
