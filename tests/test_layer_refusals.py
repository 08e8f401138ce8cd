"""What layer norm, rotary positions and linear layers refuse, checked without a GPU, as in test_train_refusals.py: every check of
arguments comes before the library looks into its context."""
import ctypes as C
import math

import pytest
import torch

import paper_2601_02311_b200.ps as ps
from test_train_refusals import AT, CTX


class Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_uint64), ("token_stride", C.c_uint64), ("head_stride", C.c_uint64)]


class NormDesc(C.Structure):
    _fields_ = [("rows", C.c_uint64), ("cols", C.c_uint64), ("eps", C.c_double), ("dtype", C.c_uint32), ("grad_dtype", C.c_uint32),
                ("accumulate", C.c_uint32), ("pad", C.c_uint32)]


class RotaryDesc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "len", "heads", "kv_heads", "dim", "rotary_dim", "dtype", "interleaved", "inverse", "position_bytes")] + \
        [("position_stride", C.c_uint64), ("first", C.c_int64)] + [(n, C.c_double) for n in ("base", "factor", "original", "low", "high", "magnitude")]


class LinearDesc(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("tokens", "inputs", "outputs")] + \
        [(n, C.c_uint32) for n in ("dtype", "grad_dtype", "activation", "below_activation", "accumulate", "pad")]


def matrices(defaults, change):
    """Each [address, stride], changed where a pair is given (None keeps a part), or null."""
    out = {}
    for name, at in defaults.items():
        given = change.pop(name, "as it is")
        at = at if given == "as it is" else None if given is None else [a if g is None else g for g, a in zip(given, at)]
        out[name] = None if at is None else C.byref(Matrix(at[0] or None, at[1]))
    return out


def norm(**change):
    args = dict(rows=4, cols=8, eps=1e-5, dtype=0)
    m = matrices(dict(x=[AT, 8], y=[AT + 1024, 8]), change)
    ptr = dict(ctx=CTX, weight=AT + 2048, bias=AT + 2304, mean=AT + 2560, rstd=AT + 2816)
    for k, v in change.items():
        (ptr if k in ptr else args)[k] = v
    return ps._lib.ps_layer_norm_forward(ptr["ctx"], C.byref(NormDesc(**args)), m["x"], ptr["weight"], ptr["bias"], m["y"], ptr["mean"], ptr["rstd"])


def norm_grad(**change):
    args = dict(rows=4, cols=8, eps=0.0, dtype=0, grad_dtype=0, accumulate=0)
    m = matrices(dict(d_y=[AT, 8], x=[AT + 1024, 8], residual=[AT + 2048, 8], d_x=[AT + 3328, 8]), change)
    ptr = dict(ctx=CTX, weight=AT + 4096, mean=AT + 4352, rstd=AT + 4608, d_weight=AT + 5120, d_bias=AT + 5376, work=AT + 16384, work_bytes=1 << 14)
    for k, v in change.items():
        (ptr if k in ptr else args)[k] = v
    return ps._lib.ps_layer_norm_backward(ptr["ctx"], C.byref(NormDesc(**args)), m["d_y"], m["x"], ptr["mean"], ptr["rstd"], ptr["weight"], m["residual"],
                                          m["d_x"], ptr["d_weight"], ptr["d_bias"], ptr["work"], ptr["work_bytes"])


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(x=None), ps.E_NULLPTR), (dict(y=None), ps.E_NULLPTR), (dict(x=(0, 8)), ps.E_NULLPTR),
    (dict(x=(AT + 2, 8)), ps.E_ALIGN), (dict(weight=AT + 2049), ps.E_ALIGN), (dict(bias=AT + 2), ps.E_ALIGN), (dict(mean=AT + 2), ps.E_ALIGN),
    (dict(rstd=AT + 1), ps.E_ALIGN), (dict(rows=1 << 31), ps.E_RANGE), (dict(cols=0), ps.E_RANGE), (dict(cols=(1 << 20) + 1), ps.E_RANGE),
    (dict(eps=-1e-9), ps.E_RANGE), (dict(eps=math.nan), ps.E_RANGE), (dict(eps=1e39), ps.E_RANGE), (dict(dtype=3), ps.E_RANGE),
    (dict(x=(None, 7)), ps.E_RANGE), (dict(y=(None, 7)), ps.E_RANGE), (dict(x=(None, 1 << 62)), ps.E_RANGE),
    (dict(y=(AT + 4, 8)), ps.E_RANGE), (dict(y=(AT, 16)), ps.E_RANGE)])
def test_layer_norm_refuses(change, code):
    assert norm(**change) == code


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(d_y=None), ps.E_NULLPTR), (dict(x=None), ps.E_NULLPTR), (dict(d_x=None), ps.E_NULLPTR),
    (dict(mean=None), ps.E_NULLPTR), (dict(rstd=None), ps.E_NULLPTR), (dict(work=None), ps.E_NULLPTR), (dict(work=AT + 16384 + 128), ps.E_ALIGN),
    (dict(work_bytes=4), ps.E_RANGE), (dict(d_weight=AT + 5121), ps.E_ALIGN), (dict(d_bias=AT + 1), ps.E_ALIGN), (dict(grad_dtype=3), ps.E_RANGE),
    (dict(accumulate=2), ps.E_RANGE), (dict(d_x=(AT + 4, 8)), ps.E_RANGE), (dict(d_x=(AT + 1024 + 4, 8)), ps.E_RANGE),
    (dict(d_x=(AT + 2048, 16)), ps.E_RANGE), (dict(residual=(None, 7)), ps.E_RANGE), (dict(residual=(AT + 2050, 8)), ps.E_ALIGN)])
def test_layer_norm_gradients_refuse(change, code):
    assert norm_grad(**change) == code


def test_layer_norm_of_nothing_is_done():
    assert norm(rows=0, x=(0, 0), y=(0, 0)) == ps.OK
    assert norm_grad(rows=0, d_y=(0, 0), x=(0, 0), residual=None, d_x=(0, 0), mean=None, rstd=None, d_weight=None, d_bias=None, work=None, work_bytes=0) == ps.OK
    assert ps._lib.ps_layer_norm_backward_bytes(C.byref(NormDesc(4, 0, 0.0, 0, 0, 0, 0))) == 0
    assert ps.Context.layer_norm_backward_bytes(4, 8, torch.float32) >= 2 * 8 * 4


def rotary(**change):
    args = dict(batch=2, len=4, heads=4, kv_heads=2, dim=8, rotary_dim=8, dtype=1, interleaved=0, inverse=0, position_bytes=4, position_stride=0, first=0,
                base=1e4, factor=1.0, original=0.0, low=1.0, high=32.0, magnitude=1.0)
    ptr = dict(ctx=CTX, positions=None)
    heads = dict(q=[AT, 128, 32, 8], q_out=[AT + 1024, 128, 32, 8], k=[AT + 2048, 64, 16, 8], k_out=[AT + 3328, 64, 16, 8])
    for k, v in change.items():
        if k in heads:
            heads[k] = None if v is None else [h if x is None else x for x, h in zip(v, heads[k])]
        else:
            (ptr if k in ptr else args)[k] = v
    h = {n: None if v is None else C.byref(Heads(v[0] or None, *v[1:])) for n, v in heads.items()}
    return ps._lib.ps_rotary(ptr["ctx"], C.byref(RotaryDesc(**args)), h["q"], h["q_out"], h["k"], h["k_out"], ptr["positions"])


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(q=None), ps.E_NULLPTR), (dict(q_out=None), ps.E_NULLPTR), (dict(k=None), ps.E_NULLPTR),
    (dict(k_out=(0, None, None, None)), ps.E_NULLPTR), (dict(q=(AT + 1, None, None, None)), ps.E_ALIGN), (dict(positions=AT + 2), ps.E_ALIGN),
    (dict(positions=AT + 4, position_bytes=8), ps.E_ALIGN), (dict(batch=65536), ps.E_RANGE), (dict(len=(1 << 24) + 1), ps.E_RANGE),
    (dict(heads=0), ps.E_RANGE), (dict(heads=32769), ps.E_RANGE), (dict(kv_heads=32769), ps.E_RANGE), (dict(dim=257, rotary_dim=2), ps.E_RANGE),
    (dict(dim=1, rotary_dim=2), ps.E_RANGE), (dict(rotary_dim=10), ps.E_RANGE), (dict(rotary_dim=3), ps.E_RANGE), (dict(rotary_dim=0), ps.E_RANGE),
    (dict(dtype=3), ps.E_RANGE), (dict(interleaved=2), ps.E_RANGE), (dict(inverse=2), ps.E_RANGE), (dict(position_bytes=2), ps.E_RANGE),
    (dict(base=0.5), ps.E_RANGE), (dict(base=math.inf), ps.E_RANGE), (dict(base=math.nan), ps.E_RANGE), (dict(factor=0.5), ps.E_RANGE),
    (dict(factor=math.nan), ps.E_RANGE), (dict(original=-1.0), ps.E_RANGE), (dict(original=4.0, factor=2.0, low=3.0, high=3.0), ps.E_RANGE),
    (dict(low=math.nan), ps.E_RANGE), (dict(high=math.inf), ps.E_RANGE), (dict(magnitude=1e39), ps.E_RANGE), (dict(magnitude=math.nan), ps.E_RANGE),
    (dict(q_out=(None, 0, None, None)), ps.E_RANGE), (dict(k_out=(None, None, None, 0)), ps.E_RANGE), (dict(q=(None, 1 << 38, None, None)), ps.E_RANGE),
    (dict(q_out=(AT, 256, None, None)), ps.E_RANGE), (dict(k_out=(AT + 1024, None, None, None)), ps.E_RANGE),
    (dict(batch=65535, len=1 << 24, heads=8), ps.E_RANGE)])
def test_rotary_refuses(change, code):
    assert rotary(**change) == code


@pytest.mark.parametrize("change", [dict(batch=0), dict(len=0), dict(batch=0, q=None, q_out=None, k=None, k_out=None)])
def test_rotary_of_nothing_is_done(change):
    assert rotary(**change) == ps.OK


def linear(**change):
    args = dict(tokens=4, inputs=8, outputs=16, dtype=1, grad_dtype=1, activation=0)
    m = matrices(dict(x=[AT, 8], weight=[AT + 1024, 8], residual=[AT + 2048, 16], y=[AT + 3328, 16], pre=[AT + 4096, 16]), change)
    ptr = dict(ctx=CTX, bias=AT + 5120)
    for k, v in change.items():
        (ptr if k in ptr else args)[k] = v
    return ps._lib.ps_linear_forward(ptr["ctx"], C.byref(LinearDesc(**args)), m["x"], m["weight"], ptr["bias"], m["residual"], m["y"], m["pre"])


def linear_grad(**change):
    args = dict(tokens=4, inputs=8, outputs=16, dtype=1, grad_dtype=0, activation=2, below_activation=2, accumulate=0)
    m = matrices(dict(d_y=[AT, 16], x=[AT + 1024, 8], weight=[AT + 2048, 8], pre=[AT + 3328, 16], below=[AT + 4096, 8], residual=[AT + 5120, 8],
                      d_x=[AT + 6144, 8], d_weight=[AT + 7168, 8]), change)
    ptr = dict(ctx=CTX, d_bias=AT + 8192, work=AT + 16384, work_bytes=1 << 14)
    for k, v in change.items():
        (ptr if k in ptr else args)[k] = v
    return ps._lib.ps_linear_backward(ptr["ctx"], C.byref(LinearDesc(**args)), m["d_y"], m["x"], m["weight"], m["pre"], m["below"], m["residual"], m["d_x"],
                                      m["d_weight"], ptr["d_bias"], ptr["work"], ptr["work_bytes"])


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(x=None), ps.E_NULLPTR), (dict(weight=None), ps.E_NULLPTR), (dict(y=None), ps.E_NULLPTR),
    (dict(residual=(0, None)), ps.E_NULLPTR), (dict(x=(AT + 2, None)), ps.E_ALIGN), (dict(x=(None, 12)), ps.E_ALIGN), (dict(weight=(None, 9)), ps.E_ALIGN),
    (dict(y=(AT + 3328 + 8, None)), ps.E_ALIGN), (dict(pre=(None, 20)), ps.E_ALIGN), (dict(bias=AT + 1), ps.E_ALIGN), (dict(y=(None, 8)), ps.E_RANGE),
    (dict(tokens=(1 << 30) + 1), ps.E_RANGE), (dict(inputs=0), ps.E_RANGE), (dict(outputs=(1 << 24) + 1), ps.E_RANGE), (dict(dtype=0), ps.E_RANGE),
    (dict(dtype=3), ps.E_RANGE), (dict(grad_dtype=2), ps.E_RANGE), (dict(activation=5), ps.E_RANGE), (dict(below_activation=5), ps.E_RANGE),
    (dict(accumulate=2), ps.E_RANGE), (dict(x=(None, 1 << 50)), ps.E_RANGE), (dict(y=(AT + 2048 + 16, None)), ps.E_RANGE), (dict(y=(AT, None)), ps.E_RANGE),
    (dict(pre=(AT + 3328, None)), ps.E_RANGE), (dict(pre=(AT + 2048, None)), ps.E_RANGE), (dict(tokens=1 << 30, inputs=1 << 20), ps.E_RANGE)])
def test_linear_refuses(change, code):
    assert linear(**change) == code


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(d_y=None), ps.E_NULLPTR), (dict(x=None), ps.E_NULLPTR), (dict(weight=None), ps.E_NULLPTR),
    (dict(pre=None), ps.E_NULLPTR), (dict(below=None), ps.E_NULLPTR), (dict(work=None), ps.E_NULLPTR), (dict(work=AT + 16384 + 16), ps.E_ALIGN),
    (dict(work_bytes=0), ps.E_RANGE), (dict(d_bias=AT + 2), ps.E_ALIGN), (dict(d_weight=(AT + 7168 + 8, None)), ps.E_ALIGN),
    (dict(d_weight=(None, 10)), ps.E_ALIGN), (dict(d_x=(AT, 16)), ps.E_RANGE), (dict(d_x=(AT + 1024, None)), ps.E_RANGE),
    (dict(d_x=(AT + 5120 + 16, None)), ps.E_RANGE), (dict(d_x=(AT + 4096, 16)), ps.E_RANGE), (dict(activation=9), ps.E_RANGE), (dict(grad_dtype=2), ps.E_RANGE)])
def test_linear_gradients_refuse(change, code):
    assert linear_grad(**change) == code


def test_linear_of_nothing_is_done():
    assert linear(tokens=0, x=(0, 0), y=(0, 0), residual=None, pre=None) == ps.OK
    assert linear_grad(x=None, weight=None, below=None, residual=None, d_x=None, d_weight=None, d_bias=None) == ps.OK
    assert ps._lib.ps_linear_backward_bytes(C.byref(LinearDesc(4, 0, 8, 1, 1, 0, 0, 0, 0))) == 0
    assert ps.Context.linear_backward_bytes(100, 64, 32, "gelu") > ps.Context.linear_backward_bytes(100, 64, 32) > 0


@pytest.fixture
def fake():
    """A context that has only what the binding looks at before it calls; tensors on the CPU have device -1."""
    ctx = object.__new__(ps.Context)
    ctx.device, ctx._h, ctx._raw_stream, ctx.stream = -1, None, 0, None
    ctx.torch_device = torch.device("cpu")
    ctx._enqueue = lambda where, call, *args: pytest.fail("not refused")
    return ctx


def refused(code, call, *args, **kw):
    with pytest.raises(ps.PsError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_binding_refuses(fake):
    x, w, b = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.bfloat16)
    stat = torch.zeros(4)
    for bad in (x[0], x.long(), x.double()):
        refused(ps.E_RANGE, fake.layer_norm_forward, bad)
    refused(ps.E_RANGE, fake.layer_norm_forward, x, weight=torch.zeros(7, dtype=torch.bfloat16))
    refused(ps.E_RANGE, fake.layer_norm_forward, x, weight=torch.zeros(8))
    refused(ps.E_RANGE, fake.layer_norm_forward, x, eps=1e39)
    refused(ps.E_ALIGN, fake.layer_norm_forward, torch.zeros(8, 4, dtype=torch.bfloat16).t())
    refused(ps.E_RANGE, fake.layer_norm_backward, x[:3], x, stat, stat)
    refused(ps.E_RANGE, fake.layer_norm_backward, x, x, stat.double(), stat)
    refused(ps.E_RANGE, fake.layer_norm_backward, x, x, stat, stat, residual=x.float())
    q = torch.zeros(2, 3, 4, 8)
    refused(ps.E_RANGE, fake.rotary, q[0])
    refused(ps.E_RANGE, fake.rotary, q, q[:, :2])
    refused(ps.E_RANGE, fake.rotary, q, dims=10)
    refused(ps.E_RANGE, fake.rotary, q, positions=torch.zeros(4, dtype=torch.int32))
    refused(ps.E_RANGE, fake.rotary, q, positions=torch.zeros(3))
    refused(ps.E_ALIGN, fake.rotary, q, positions=torch.zeros(3, 2, dtype=torch.int32).t())
    refused(ps.E_RANGE, fake.rotary, q, first=1 << 63)
    refused(ps.E_RANGE, fake.rotary, q, magnitude=math.inf)
    refused(ps.E_ALIGN, fake.rotary, torch.zeros(2, 3, 8, 4).transpose(2, 3))
    refused(ps.E_RANGE, fake.linear_forward, x, w[:, :7])
    refused(ps.E_RANGE, fake.linear_forward, x, w, bias=b[:5])
    refused(ps.E_RANGE, fake.linear_forward, x, w, activation="swish")
    refused(ps.E_RANGE, fake.linear_forward, x, w, residual=x)
    refused(ps.E_RANGE, fake.linear_forward, x, w.half())
    d_y = torch.zeros(4, 6, dtype=torch.bfloat16)
    refused(ps.E_RANGE, fake.linear_backward, d_y[:, :5], x, w)
    refused(ps.E_RANGE, fake.linear_backward, d_y, x, w, pre=x, activation="gelu")
    refused(ps.E_RANGE, fake.linear_backward, d_y, x, w, dtype=torch.float16)
    refused(ps.E_NULLPTR, fake.linear_backward_into, d_y, None, w, d_weight=w)
    refused(ps.E_NULLPTR, fake.linear_backward_into, d_y, x, None, d_x=x)
    refused(ps.E_RANGE, fake.linear_backward_into, d_y, x, w, d_bias=b, work=torch.zeros(4))
