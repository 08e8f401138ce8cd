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


# q AT (2 x 4 x 4 heads of 8, 512 bytes), q_out AT + 1024, k AT + 2048 (256 bytes), k_out AT + 3328
@pytest.mark.parametrize("change", [
    dict(q_out=(AT + 2, None, None, None)), dict(q_out=(AT + 64, None, None, None)), dict(q_out=(AT - 510, None, None, None)),
    dict(q_out=(AT + 16, None, None, None)), dict(q_out=(AT, None, 8, 32)), dict(q_out=(AT + 2048, None, None, None)), dict(q_out=(AT + 2048 - 500, None, None, None)),
    dict(q_out=(AT + 3328 + 254, None, None, None)), dict(k_out=(AT, None, None, None)), dict(k_out=(AT + 510, None, None, None)),
    dict(k_out=(AT + 2048 + 16, None, None, None)), dict(k_out=(AT + 1024 + 32, None, None, None)),
    dict(positions=AT + 1024), dict(positions=AT + 3328 + 252), dict(positions=AT + 3328 - 16, position_stride=4),
    # a result whose own heads, tokens or sequences meet
    dict(q_out=(None, 128, 32, 4)), dict(q_out=(None, 128, 8, 8)), dict(q_out=(None, 96, 32, 8)), dict(q_out=(None, 8, 16, 24)), dict(k_out=(None, 64, 16, 7))])
def test_rotary_refuses_results_over_operands(change):
    assert answer(t.rotary, **change) == ps.E_RANGE


@pytest.mark.parametrize("change", [
    dict(), dict(q_out=(AT, None, None, None)), dict(q_out=(AT, None, None, None), k_out=(AT + 2048, None, None, None)), dict(q_out=(AT + 512, None, None, None)),
    # heads of one buffer: q, k and a third kind, in place and turned into the third's place
    dict(q=(AT, 256, 64, 8), k=(AT + 64, 256, 64, 8), q_out=(AT, 256, 64, 8), k_out=(AT + 64, 256, 64, 8)),
    dict(q=(AT, 256, 64, 8), k=(AT + 64, 256, 64, 8), k_out=(AT + 96, 256, 64, 8)), dict(q=(AT, 256, 8, 64), q_out=(AT + 64, 256, 8, 64)),
    # every second element of rows, heads before tokens, sequences inside heads
    dict(q_out=(AT + 1024, 32, 64, 8)), dict(q_out=(AT + 1024, 32, 8, 64)), dict(q_out=(AT + 1024, 8, 16, 64)),
    dict(q=(AT, 0, 0, 0)), dict(q=(AT, 0, 32, 8), q_out=(AT + 256, None, None, None)), dict(positions=AT + 512), dict(positions=AT + 1024 - 16)])
def test_rotary_takes_results_beside_operands(change):
    assert answer(t.rotary, **change) == TAKEN


def of_heads(h, batch, length, heads, dim):
    return [h[0] + 2 * (b * h[1] + i * h[2] + n * h[3] + e) for b in range(batch) for i in range(length) for n in range(heads) for e in range(dim)]


@pytest.mark.parametrize("seed", range(12))
def test_rotary_overlaps_against_the_elements_themselves(seed):
    rng = random.Random(seed)
    seen = set()
    for _ in range(300):
        batch, length, heads, kv_heads, dim = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4), rng.randint(0, 2), rng.choice([2, 5, 8])
        count = dict(q=heads, q_out=heads, k=kv_heads, k_out=kv_heads)

        def strides(n):
            order, at, out = rng.sample(range(3), 3), dim + rng.choice([0, 0, 3]), [0, 0, 0]
            for i in order:
                out[i] = at
                at = max(1, at * (batch, length, n)[i] + rng.choice([0, 0, 0, 8, -1]))
            return out
        common = strides(heads + 2 * kv_heads)
        given = {n: (AT + 2 * rng.randint(0, 700), *(common if rng.random() < 0.7 else strides(count[n]))) for n in count}
        for n in ("q", "k"):
            if rng.random() < 0.3:
                given[n + "_out"] = given[n]
        e = {n: of_heads(h, batch, length, count[n], dim) for n, h in given.items()}
        sets = {n: set(v) for n, v in e.items()}

        def same(a, b):
            return given[a][0] == given[b][0] and all(extent == 1 or x == y for extent, x, y in
                                                      zip((batch, length, count[a]), given[a][1:], given[b][1:]))
        bad = any(len(e[n]) != len(sets[n]) for n in ("q_out", "k_out")) or \
            any(sets[a] & sets[b] for a, b in (("q_out", "k"), ("q_out", "k_out"), ("k_out", "q"))) or \
            any(sets[n] & sets[n + "_out"] and not same(n, n + "_out") for n in ("q", "k"))
        got = answer(t.rotary, batch=batch, len=length, heads=heads, kv_heads=kv_heads, dim=dim, rotary_dim=2, **given)
        assert got == (ps.E_RANGE if bad else TAKEN), (batch, length, heads, kv_heads, dim, given)
        seen.add(got)
    assert seen == {ps.E_RANGE, TAKEN}


# x AT (128 bytes), y AT + 1024, weight AT + 2048 (32), bias AT + 2304, mean AT + 2560 (16), rstd AT + 2816
@pytest.mark.parametrize("change", [
    dict(y=(AT + 4, None)), dict(y=(AT - 124, None)), dict(y=(AT, 16)), dict(y=(AT + 2048 + 28, None)), dict(y=(AT + 2304, None)), dict(y=(AT + 2560 - 124, None)),
    dict(y=(AT + 2816, None)), dict(mean=AT + 124), dict(mean=AT + 2048), dict(mean=AT + 2304 + 28), dict(mean=AT + 2816 - 12), dict(rstd=AT),
    dict(rstd=AT + 2048 + 28), dict(rstd=AT + 2304 - 12)])
def test_norm_refuses_results_over_operands(change):
    assert answer(t.norm, **change) == ps.E_RANGE


@pytest.mark.parametrize("change", [
    dict(), dict(y=(AT, None)), dict(y=(AT + 128, None)), dict(x=(AT, 32), y=(AT + 32, 32)), dict(x=(AT + 32, 32), y=(AT, 32)), dict(mean=AT + 128),
    dict(mean=AT + 2816 - 16), dict(weight=AT + 2304), dict(x=(AT, 16), mean=None, rstd=None)])
def test_norm_takes_results_beside_operands(change):
    assert answer(t.norm, **change) == TAKEN


# d_y AT (128 bytes), x AT + 1024, residual AT + 2048, d_x AT + 3328, weight AT + 4096 (32), mean AT + 4352 (16), rstd AT + 4608, d_weight AT + 5120, d_bias AT + 5376
@pytest.mark.parametrize("change", [
    dict(d_x=(AT + 4, None)), dict(d_x=(AT + 1024 + 124, None)), dict(d_x=(AT + 2048 - 4, None)), dict(d_x=(AT + 4096 + 28, None)), dict(d_x=(AT + 4352, None)),
    dict(d_x=(AT + 4608 - 124, None)), dict(d_x=(AT + 5120, None)), dict(d_x=(AT + 5376 + 28, None)), dict(d_weight=AT + 5376 - 28), dict(d_bias=AT + 5120)])
def test_norm_gradients_refuse_results_over_operands(change):
    assert answer(t.norm_grad, **change) == ps.E_RANGE


@pytest.mark.parametrize("change", [
    dict(), dict(d_x=(AT, None)), dict(d_x=(AT + 1024, None)), dict(d_x=(AT + 2048, None)), dict(d_x=(AT + 2048, None), residual=None),
    dict(d_y=(AT, 32), d_x=(AT + 32, 32)), dict(d_weight=AT + 5376 - 32), dict(d_weight=AT + 4096)])
def test_norm_gradients_take_results_beside_operands(change):
    assert answer(t.norm_grad, **change) == TAKEN
