"""What the training step's operators refuse, checked without a GPU: every check of arguments comes
before the library looks into its context, so a context that is only a block of zeros is enough."""
import ctypes as C
import math

import pytest
import torch

import paper_2601_02311_b200.ps as ps


class DropoutDesc(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("rows", "cols", "x_stride", "residual_stride", "y_stride", "seed", "stream", "first", "pitch")] + \
        [("p", C.c_double), ("dtype", C.c_uint32), ("pad", C.c_uint32)]


class EmbedDesc(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("tokens", "first_row", "rows", "dim", "table_stride", "out_stride")] + \
        [("scale", C.c_double)] + [(n, C.c_uint32) for n in ("dtype", "grad_dtype", "token_bytes", "accumulate")]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_uint64), ("token_stride", C.c_uint64), ("head_stride", C.c_uint64)]


class AttentionShape(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("batch", "q_len", "k_len", "heads", "kv_heads", "dim", "dtype", "causal")] + \
        [("scale", C.c_float), ("pad", C.c_uint32)]


FAKE = C.create_string_buffer(4096)
CTX = C.cast(FAKE, C.c_void_p)
BUF = C.create_string_buffer(1 << 16)
AT = (C.addressof(BUF) + 255) // 256 * 256


def dropout(**kw):
    args = dict(rows=4, cols=8, x_stride=8, residual_stride=8, y_stride=8, seed=1, stream=0, first=0, pitch=8, p=0.1, dtype=0)
    ptr = dict(ctx=CTX, x=AT, residual=None, y=AT + 4096)
    for k, v in kw.items():
        (ptr if k in ptr else args)[k] = v
    return ps._lib.ps_dropout(ptr["ctx"], C.byref(DropoutDesc(**args)), ptr["x"], ptr["residual"], ptr["y"])


@pytest.mark.parametrize("change, code", [
    (dict(ctx=None), ps.E_NULLPTR), (dict(x=None), ps.E_NULLPTR), (dict(y=None), ps.E_NULLPTR),
    (dict(x=AT + 2), ps.E_ALIGN), (dict(y=AT + 4097, dtype=1), ps.E_ALIGN), (dict(residual=AT + 3), ps.E_ALIGN),
    (dict(dtype=3), ps.E_RANGE), (dict(p=-0.01), ps.E_RANGE), (dict(p=1.01), ps.E_RANGE), (dict(p=math.nan), ps.E_RANGE),
    (dict(y_stride=7), ps.E_RANGE), (dict(rows=1 << 25, cols=1 << 24, y_stride=1 << 24), ps.E_RANGE),
    (dict(first=1 << 63), ps.E_RANGE), (dict(pitch=1 << 62), ps.E_RANGE), (dict(rows=(1 << 64) - 1), ps.E_RANGE),
    (dict(y=AT + 4), ps.E_RANGE),                                  # overlaps x, one element on
    (dict(y=AT, y_stride=16), ps.E_RANGE),                         # x itself with other strides
    (dict(residual=AT + 4096 + 32), ps.E_RANGE),                   # overlaps y
    (dict(x_stride=32, y_stride=32, y=AT + 64, cols=20), ps.E_RANGE),
    (dict(rows=1, x_stride=0, y_stride=0, y=AT + 4), ps.E_RANGE),  # a single row, whose stride says nothing
    (dict(rows=1, x_stride=1, y_stride=1, y=AT + 16), ps.E_RANGE),
    (dict(rows=1, x_stride=99, y_stride=99, y=AT - 28), ps.E_RANGE),
    (dict(rows=1, x_stride=0, y_stride=0, residual_stride=0, residual=AT + 4096 + 4), ps.E_RANGE),
])
def test_dropout_refuses(change, code):
    assert dropout(**change) == code


@pytest.mark.parametrize("change", [dict(rows=0), dict(cols=0), dict(rows=0, x=None, y=None)])
def test_dropout_of_nothing_is_done(change):
    assert dropout(**change) == ps.OK


def embed(backward=False, **kw):
    args = dict(tokens=4, first_row=0, rows=10, dim=8, table_stride=8, out_stride=8, scale=1.0, dtype=1, grad_dtype=0,
                token_bytes=8, accumulate=0)
    ptr = dict(ctx=CTX, table=AT, tokens_at=AT + 4096, out=AT + 8192, work=AT + 16384, work_bytes=1 << 14)
    for k, v in kw.items():
        (ptr if k in ptr else args)[k] = v
    if not backward:
        return ps._lib.ps_embed_forward(ptr["ctx"], C.byref(EmbedDesc(**args)), ptr["table"], ptr["tokens_at"], ptr["out"])
    return ps._lib.ps_embed_backward(ptr["ctx"], C.byref(EmbedDesc(**args)), ptr["out"], ptr["tokens_at"], ptr["table"], ptr["work"],
                                     ptr["work_bytes"])


EMBED = [(dict(ctx=None), ps.E_NULLPTR), (dict(table=None), ps.E_NULLPTR), (dict(tokens_at=None), ps.E_NULLPTR),
         (dict(out=None), ps.E_NULLPTR), (dict(out=AT + 8193), ps.E_ALIGN), (dict(tokens_at=AT + 4100), ps.E_ALIGN),
         (dict(table=AT + 1), ps.E_ALIGN), (dict(rows=0), ps.E_RANGE), (dict(rows=(1 << 30) + 1), ps.E_RANGE),
         (dict(tokens=(1 << 30) + 1), ps.E_RANGE), (dict(dim=0), ps.E_RANGE), (dict(table_stride=7), ps.E_RANGE),
         (dict(out_stride=7), ps.E_RANGE), (dict(dtype=3), ps.E_RANGE), (dict(token_bytes=2), ps.E_RANGE),
         (dict(scale=math.inf), ps.E_RANGE), (dict(scale=-1e39), ps.E_RANGE), (dict(accumulate=2), ps.E_RANGE), (dict(grad_dtype=9), ps.E_RANGE)]


@pytest.mark.parametrize("change, code", EMBED)
@pytest.mark.parametrize("backward", [False, True])
def test_embedding_refuses(backward, change, code):
    assert embed(backward, **change) == code


def test_embedding_gradient_refuses_a_short_work_buffer():
    need = ps.Context.embed_backward_bytes(4, 10, 8)
    if need:
        assert embed(True, work=None) == ps.E_NULLPTR
        assert embed(True, work=AT + 16384 + 128) == ps.E_ALIGN
        assert embed(True, work_bytes=need - 1) == ps.E_RANGE
    assert ps.Context.embed_backward_bytes(4, 0, 8) == 0


def test_lookup_of_no_tokens_is_done():
    assert embed(tokens=0, table=None, tokens_at=None, out=None) == ps.OK


def attention(backward=False, **kw):
    args = dict(batch=2, q_len=4, k_len=4, heads=4, kv_heads=2, dim=8, dtype=1, causal=1, scale=1.0)
    ptr = dict(ctx=CTX, lse=AT + 8192, q_lens=None, k_lens=None, work=AT + 16384, work_bytes=1 << 14)
    names = ["q", "k", "v", "out", "d_out", "d_q", "d_k", "d_v"]
    heads = {n: [AT + 1024 * i, 256, 32, 8] for i, n in enumerate(names)}
    for k, v in kw.items():
        if k in heads and v is not None:
            heads[k] = [h if x is None else x for x, h in zip(v, heads[k])]
        elif k in heads:
            heads[k] = None
        else:
            (ptr if k in ptr else args)[k] = v
    h = {n: None if v is None else C.byref(Heads(*[x or None if i == 0 else x for i, x in enumerate(v)])) for n, v in heads.items()}
    shape = C.byref(AttentionShape(**args))
    if not backward:
        return ps._lib.ps_attention_forward(ptr["ctx"], shape, h["q"], h["k"], h["v"], h["out"], ptr["lse"], ptr["q_lens"], ptr["k_lens"],
                                            ptr["work"], ptr["work_bytes"])
    return ps._lib.ps_attention_backward(ptr["ctx"], shape, h["q"], h["k"], h["v"], h["out"], ptr["lse"], h["d_out"], h["d_q"],
                                         h["d_k"], h["d_v"], ptr["q_lens"], ptr["k_lens"], ptr["work"], ptr["work_bytes"])


ATTENTION = [(dict(ctx=None), ps.E_NULLPTR), (dict(q=None), ps.E_NULLPTR), (dict(lse=None), ps.E_NULLPTR),
             (dict(v=[0, None, None, None]), ps.E_NULLPTR), (dict(k=[AT + 8, None, None, None]), ps.E_ALIGN),
             (dict(q=[None, 260, None, None]), ps.E_ALIGN), (dict(out=[None, None, 36, None]), ps.E_ALIGN),
             (dict(v=[None, None, None, 4]), ps.E_ALIGN), (dict(k=[None, None, None, 0]), ps.E_RANGE),
             (dict(q=[None, 0, None, None]), ps.E_RANGE), (dict(q=[None, 1 << 38, None, None]), ps.E_RANGE),
             (dict(lse=AT + 2), ps.E_ALIGN), (dict(q_lens=AT + 2), ps.E_ALIGN), (dict(dtype=0), ps.E_RANGE),
             (dict(dtype=3), ps.E_RANGE), (dict(dim=12), ps.E_RANGE), (dict(dim=136), ps.E_RANGE), (dict(dim=0), ps.E_RANGE),
             (dict(heads=3), ps.E_RANGE), (dict(kv_heads=0), ps.E_RANGE), (dict(heads=0), ps.E_RANGE), (dict(causal=2), ps.E_RANGE),
             (dict(scale=math.nan), ps.E_RANGE), (dict(batch=1 << 16), ps.E_RANGE), (dict(q_len=(1 << 24) + 1), ps.E_RANGE),
             (dict(batch=65535, heads=32768, kv_heads=1, q_len=129), ps.E_RANGE)]


@pytest.mark.parametrize("change, code", ATTENTION)
@pytest.mark.parametrize("backward", [False, True])
def test_attention_refuses(backward, change, code):
    assert attention(backward, **change) == code


@pytest.mark.parametrize("change, code", [
    (dict(d_out=None), ps.E_NULLPTR), (dict(d_q=None), ps.E_NULLPTR), (dict(d_v=[None, None, None, 12]), ps.E_ALIGN),
    (dict(d_k=[None, None, 0, None]), ps.E_RANGE), (dict(work=None), ps.E_NULLPTR), (dict(work=AT + 16384 + 16), ps.E_ALIGN),
    (dict(work_bytes=8), ps.E_RANGE)])
def test_attention_backward_refuses(change, code):
    assert attention(True, **change) == code


def test_attention_forward_refuses_a_short_work_buffer():
    """Few queries over many keys are cut into chunks, whose results need room; other shapes need none."""
    need = ps.Context.attention_forward_bytes(2, 4, 5000, 4, 2, 8)
    assert need > 0 and ps.Context.attention_forward_bytes(2, 4, 4, 4, 2, 8) == 0
    assert attention(k_len=5000, work=None) == ps.E_NULLPTR
    assert attention(k_len=5000, work_bytes=need - 1) == ps.E_RANGE
    assert attention(k_len=5000, work=AT + 16384 + 64, work_bytes=need) == ps.E_ALIGN


def test_attention_of_nothing_is_done():
    assert attention(batch=0) == ps.OK and attention(True, batch=0) == ps.OK
    assert attention(q_len=0) == ps.OK and attention(True, q_len=0, k_len=0) == ps.OK


# ---- the binding's own checks: what the library cannot see

@pytest.fixture
def ctx():
    c = ps.Context.__new__(ps.Context)
    c.torch_device, c.device, c.stream, c._h = torch.device("cpu"), -1, None, None     # a host tensor's device is -1
    return c


def refused(code, call, *args, **kw):
    with pytest.raises(ps.PsError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_binding_refuses_shapes_types_and_strides(ctx):
    x = torch.zeros(4, 8)
    refused(ps.E_RANGE, ctx.dropout_into, x, torch.zeros(4, 7), 0.1, 1)
    refused(ps.E_RANGE, ctx.dropout_into, x, x.half(), 0.1, 1)
    refused(ps.E_RANGE, ctx.dropout_into, x.int(), x.int(), 0.1, 1)
    refused(ps.E_RANGE, ctx.dropout_into, x[0], x[0], 0.1, 1)
    refused(ps.E_ALIGN, ctx.dropout_into, x.t(), x.t(), 0.1, 1)
    refused(ps.E_RANGE, ctx.dropout_into, x, x, 0.1, -1)
    refused(ps.E_RANGE, ctx.dropout_into, x, x, 0.1, 1, first=-4)
    ctx.device = 0                                                  # and another device's tensor is refused
    refused(ps.E_RANGE, ctx.dropout_into, x, x.clone(), 0.1, 1)
    ctx.device = -1
    tokens = torch.zeros(3, dtype=torch.int64)
    refused(ps.E_RANGE, ctx.embed_forward_into, x, tokens.short(), torch.zeros(3, 8))
    refused(ps.E_RANGE, ctx.embed_forward_into, x, tokens, torch.zeros(4, 8))
    refused(ps.E_ALIGN, ctx.embed_forward_into, x, torch.zeros(6, dtype=torch.int64)[::2], torch.zeros(3, 8))
    refused(ps.E_RANGE, ctx.embed_forward_into, x, tokens.reshape(3, 1), torch.zeros(3, 8))
    refused(ps.E_RANGE, ctx.embed_forward_into, x, tokens, torch.zeros(3, 8), first_row=-1)
    refused(ps.E_RANGE, ctx.embed_backward_into, torch.zeros(4, 8), tokens, x)
    q, k = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16), torch.zeros(2, 6, 2, 16, dtype=torch.bfloat16)
    lse = torch.zeros(2, 4, 5)
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k[:, :5], q, lse)
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k.half(), q, lse)
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k, q, lse.double())
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k, q, lse[:, :, :4])
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k, q, lse, q_lens=torch.zeros(2))
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k, q, lse, k_lens=torch.zeros(3, dtype=torch.int32))
    refused(ps.E_ALIGN, ctx.attention_forward_into, q, k, k, torch.zeros(2, 5, 4, 32, dtype=torch.bfloat16)[..., ::2], lse)


@pytest.mark.parametrize("scale", [1e39, -1e39, math.inf, math.nan])
def test_binding_refuses_a_scale_that_is_no_float(ctx, scale):
    q, k = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16), torch.zeros(2, 6, 2, 16, dtype=torch.bfloat16)
    refused(ps.E_RANGE, ctx.attention_forward_into, q, k, k, q, torch.zeros(2, 4, 5), scale=scale)
    refused(ps.E_RANGE, ctx.attention_backward_into, q, k, k, q, torch.zeros(2, 4, 5), q, q, k, k, scale=scale)
