"""The operators of a training step on the GPU, against their definitions in 64 bits.

Bounds are counted, not measured.  u = eps / 2 of a type is the largest relative error of one
rounding to it (subnormals: half of the smallest one); f = 2^-24 is that of float32.  A sum of n terms in
float32, in any order, is off by at most n f times the sum of the terms' magnitudes.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ps():
    import paper_2601_02311_b200.ps as m
    return m


@pytest.fixture(scope="module")
def ctx(ps):
    return ps.Context(0)


def u_of(dtype):
    return torch.finfo(dtype).eps / 2


def tiny_of(dtype):
    """Half of the smallest subnormal: the largest error of a rounding that ends among the subnormals."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def within(got, want, bound, what=""):
    got = got.double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= bound) & ~((got == want))
    assert not bad.any(), (what, int(bad.sum()), (got - want)[bad][:3], bound.expand_as(want)[bad][:3], torch.nonzero(bad)[:3])


def normal(gen, *shape, dtype=torch.float32, size=1.0):
    return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, size, generator=gen)


# ------------------------------------------------------------------ dropout

def words(index, stream, seed):
    """Philox4x32-10's word for each of some element indices, in Python integers."""
    m = (1 << 32) - 1
    out = []
    for g in index:
        c = [g // 4 & m, g // 4 >> 32, stream & m, stream >> 32]
        k0, k1 = seed & m, seed >> 32
        for _ in range(10):
            p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(q >> 32) ^ c[1] ^ k0, q & m, (p >> 32) ^ c[3] ^ k1, p & m]
            k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
        out.append(c[g % 4])
    return out


def test_generator_gives_the_published_words():
    # the known answers that the generator's authors publish, for counters and keys of zeros, ones and pi
    def block(counter, key):
        g = 4 * (counter[0] | counter[1] << 32)
        return words([g, g + 1, g + 2, g + 3], counter[2] | counter[3] << 32, key[0] | key[1] << 32)
    assert block([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert block([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert block([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def dropout_want(x, p, seed, stream, residual, first, pitch):
    rows, cols = x.shape
    index = [first + r * pitch + c for r in range(rows) for c in range(cols)]
    kept = torch.tensor(words(index, stream, seed), dtype=torch.int64).view(rows, cols).to(x.device) >= round(p * 2 ** 32)
    y = torch.where(kept, x.double() / (1 - p) if p < 1 else 0.0, 0.0)
    size = y.abs()
    if residual is not None:
        y, size = y + residual.double(), size + residual.double().abs()
    # the scale, the product and the sum are each rounded to float32, the result to its type
    return y, kept, u_of(x.dtype) * y.abs() + tiny_of(x.dtype) + 4 * F * size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols, first, pitch, p", [
    (1, 1, 0, 1, 0.5), (1, 3, 5, 3, 0.5), (7, 129, 0, 129, 0.1), (5, 256, 0, 256, 0.1), (3, 264, 4, 1056, 0.25),
    (4, 250, 1, 1000, 0.1), (2, 31, (1 << 40) + 2, 1 << 41, 0.3), (33, 8, 0, 8, 0.0), (9, 16, 3, 16, 1.0), (2, 2049, 7, 2049, 0.1)])
def test_dropout(ctx, dtype, rows, cols, first, pitch, p):
    gen = torch.Generator("cuda").manual_seed(rows * 7919 + cols)
    x, res = normal(gen, rows, cols, dtype=TYPES[dtype]), normal(gen, rows, cols, dtype=TYPES[dtype])
    seed, stream = 0xA4093822299F31D0, (3 << 32) + 77
    for residual in (None, res):
        want, _, bound = dropout_want(x, p, seed, stream, residual, first, pitch)
        got = ctx.dropout(x, p, seed, stream, residual, first, pitch)
        ctx.check_status()
        within(got, want, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset, stride", [(0, 200), (1, 201), (8, 136), (3, 160)])
def test_dropout_of_rows_in_a_larger_tensor(ctx, dtype, offset, stride):
    """Columns of wider rows, at any alignment; what lies between them stays as it was."""
    gen = torch.Generator("cuda").manual_seed(stride)
    x, res, y = (normal(gen, 6, stride + 16, dtype=TYPES[dtype]) for _ in range(3))
    part = [t[:, offset:offset + 130] for t in (x, res, y)]
    before = y.clone()
    want, _, bound = dropout_want(part[0], 0.2, 5, 0, part[1], 0, 130)
    ctx.dropout_into(part[0], part[2], 0.2, 5, residual=part[1])
    ctx.check_status()
    within(part[2], want, bound)
    assert torch.equal(y[:, :offset], before[:, :offset]) and torch.equal(y[:, offset + 130:], before[:, offset + 130:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nth", [0, 1, 2])
@pytest.mark.parametrize("offset, stride, cols", [(32, 96, 64), (16, 80, 64), (48, 96, 48), (32, 96, 40), (4, 96, 64)])
def test_dropout_at_every_alignment_of_one_tensor(ctx, dtype, nth, offset, stride, cols):
    """Rows of one of the three tensors begin `offset` bytes behind a multiple of 64, `stride` elements apart: accesses of 32 bytes, of
    16 or of an element."""
    gen = torch.Generator("cuda").manual_seed(offset + cols)
    whole = [normal(gen, 5, 128, dtype=TYPES[dtype]) for _ in range(3)]
    at = offset // whole[0].element_size()
    part = [t.view(-1).as_strided((5, cols), (stride if i == nth else 128, 1), at if i == nth else 0) for i, t in enumerate(whole)]
    before = whole[2].clone()
    want, _, bound = dropout_want(part[0], 0.2, 5, 1, part[1], 4, 96)
    ctx.dropout_into(part[0], part[2], 0.2, 5, stream=1, residual=part[1], first=4, pitch=96)
    ctx.check_status()
    within(part[2], want, bound)
    # what lies around y's rows is as it was
    rest = torch.ones(5 * 128, dtype=torch.bool, device="cuda")
    rest.as_strided((5, cols), part[2].stride(), part[2].storage_offset()).zero_()
    assert torch.equal(whole[2].view(-1)[rest], before.view(-1)[rest])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("cols, first, offset", [(1, 0, 1), (2, 3, 3), (15, 1, 7), (127, 2, 0), (505, 1, 3), (508, 0, 1), (509, 3, 0), (1013, 2, 5), (1531, 1, 6),
                                                 (2040, 3, 2)])
def test_dropout_of_rows_that_begin_anywhere(ctx, dtype, alike, cols, first, offset):
    """Rows at every distance from a multiple of 16 bytes, the same in all tensors or another in the residual."""
    gen = torch.Generator("cuda").manual_seed(cols)
    stride = cols + 9 - cols % 2
    whole = [normal(gen, 6 * stride + 32, dtype=TYPES[dtype]) for _ in range(3)]
    part = [t.as_strided((6, cols), (stride, 1), offset + (0 if alike or i != 1 else 3)) for i, t in enumerate(whole)]
    before = whole[2].clone()
    want, _, bound = dropout_want(part[0], 0.3, 11, 2, part[1], first, 4 * cols + 1)
    ctx.dropout_into(part[0], part[2], 0.3, 11, stream=2, residual=part[1], first=first, pitch=4 * cols + 1)
    ctx.check_status()
    within(part[2], want, bound)
    rest = torch.ones_like(whole[2], dtype=torch.bool)
    rest.as_strided((6, cols), (stride, 1), offset).zero_()
    assert torch.equal(whole[2][rest], before[rest])
    ctx.dropout_into(part[0], part[0], 0.3, 11, stream=2, residual=part[1], first=first, pitch=4 * cols + 1)
    assert torch.equal(part[0], part[2])


def test_dropout_in_place_and_of_broadcast_rows(ctx):
    gen = torch.Generator("cuda").manual_seed(1)
    x, res = normal(gen, 10, 72, dtype=torch.bfloat16), normal(gen, 10, 72, dtype=torch.bfloat16)
    want = ctx.dropout(x, 0.3, 9, residual=res)
    a, b = x.clone(), res.clone()
    ctx.dropout_into(a, a, 0.3, 9, residual=res)
    ctx.dropout_into(x, b, 0.3, 9, residual=b)
    assert torch.equal(a, want) and torch.equal(b, want)
    row = x[:1].expand(10, 72)
    assert torch.equal(ctx.dropout(row, 0.3, 9), ctx.dropout(row.contiguous(), 0.3, 9))
    ctx.check_status()


def test_dropped_elements_are_not_looked_at(ctx):
    gen = torch.Generator("cuda").manual_seed(2)
    x = normal(gen, 16, 100)
    _, kept, _ = dropout_want(x, 0.5, 11, 0, None, 0, 100)
    bad = torch.where(kept, x, torch.tensor([math.nan, math.inf], device="cuda").repeat(50))
    assert torch.equal(ctx.dropout(bad, 0.5, 11), ctx.dropout(x, 0.5, 11))
    assert ctx.dropout(torch.full_like(x, math.nan), 1.0, 11).eq(0).all()


def test_dropout_of_shards_is_the_whole_tensors(ctx):
    gen = torch.Generator("cuda").manual_seed(3)
    x = normal(gen, 24, 1000, dtype=torch.bfloat16)
    whole = ctx.dropout(x, 0.1, 17, stream=4)
    for begin, end in ((0, 5), (5, 24)):                # rows of a data axis
        assert torch.equal(ctx.dropout(x[begin:end], 0.1, 17, stream=4, first=begin * 1000), whole[begin:end])
    for begin, end in ((0, 334), (334, 667), (667, 1000)):    # columns of a tensor axis
        assert torch.equal(ctx.dropout(x[:, begin:end], 0.1, 17, stream=4, first=begin, pitch=1000), whole[:, begin:end])


def test_dropout_drops_its_share_and_streams_differ(ctx):
    x = torch.ones(1 << 20, 4, device="cuda")
    masks = [ctx.dropout(x, 0.1, seed, stream) == 0 for seed, stream in ((1, 0), (1, 1), (2, 0))]
    n = x.numel()
    for m in masks:                                     # six deviations of a binomial count
        assert abs(int(m.sum()) - 0.1 * n) < 6 * math.sqrt(0.09 * n)
    for a, b in ((0, 1), (0, 2), (1, 2)):
        assert abs(int((masks[a] & masks[b]).sum()) - 0.01 * n) < 6 * math.sqrt(0.0099 * n)


def test_dropout_behind_two_to_the_32_elements(ctx):
    """Offsets that pass 32 bits: the last rows of a tensor of 2^32 + elements, in bytes and in elements."""
    cols = 1 << 14
    rows = (1 << 18) + 3
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-2:] = 1.0
    y = ctx.dropout(x, 0.25, 3)
    assert torch.equal(y[-2:], ctx.dropout(x[-2:].clone(), 0.25, 3, first=(rows - 2) * cols, pitch=cols))
    assert y[:-2].eq(0).all()


# ------------------------------------------------------------------ embedding

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("token_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("tokens, rows, dim, first_row", [(1, 1, 1, 0), (7, 5, 3, 0), (300, 50, 129, 20), (64, 1000, 768, 0),
                                                         (1000, 3, 264, 1), (5, 4, 2050, 0)])
def test_lookup(ctx, dtype, token_type, tokens, rows, dim, first_row):
    gen = torch.Generator("cuda").manual_seed(tokens + dim)
    table = normal(gen, rows, dim, dtype=TYPES[dtype])
    ids = torch.randint(-2, first_row + rows + 3, (tokens,), device="cuda", generator=gen).to(token_type)
    held = (ids >= first_row) & (ids < first_row + rows)
    want = table[(ids.long() - first_row).clamp(0, rows - 1)].double() * 1.7 * held[:, None]
    got = ctx.embed_forward(table, ids, 1.7, first_row)
    ctx.check_status()
    # the scale and the product rounded to float32, the result to its type
    within(got, want, u_of(table.dtype) * want.abs() + tiny_of(table.dtype) + 3 * F * want.abs())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("of_table", [False, True])
@pytest.mark.parametrize("offset, stride, dim", [(32, 160, 128), (16, 160, 128), (32, 136, 128), (32, 160, 72), (64, 1088, 1040), (4, 160, 128)])
def test_lookup_at_every_alignment(ctx, dtype, of_table, offset, stride, dim):
    """The table's or the result's rows begin `offset` bytes behind a multiple of 64: accesses of 32 bytes, of 16 or of an element."""
    gen = torch.Generator("cuda").manual_seed(offset + dim)
    table, out = normal(gen, 40, 1152, dtype=TYPES[dtype]), normal(gen, 60, 1152, dtype=TYPES[dtype])
    at = offset // table.element_size()
    t = table.view(-1).as_strided((40, dim), (stride if of_table else 1152, 1), at if of_table else 0)
    o = out.view(-1).as_strided((60, dim), (1152 if of_table else stride, 1), 0 if of_table else at)
    ids = torch.randint(-1, 42, (60,), device="cuda", generator=gen)
    held = (ids >= 0) & (ids < 40)
    want = t[ids.clamp(0, 39)].double() * 1.7 * held[:, None]
    before = out.clone()
    ctx.embed_forward_into(t, ids, o, 1.7)
    ctx.check_status()
    within(o, want, u_of(table.dtype) * want.abs() + tiny_of(table.dtype) + 3 * F * want.abs())
    rest = torch.ones(60 * 1152, dtype=torch.bool, device="cuda")
    rest.as_strided((60, dim), o.stride(), o.storage_offset()).zero_()
    assert torch.equal(out.view(-1)[rest], before.view(-1)[rest])


def gradient_want(d_out, ids, rows, scale, first_row, dtype):
    held = (ids >= first_row) & (ids < first_row + rows)
    at = (ids.long() - first_row)[held]
    terms = d_out[held].double() * scale
    want = torch.zeros(rows, d_out.shape[1], device="cuda", dtype=torch.float64).index_add_(0, at, terms)
    size = torch.zeros_like(want).index_add_(0, at, terms.abs())
    n = torch.zeros(rows, device="cuda", dtype=torch.float64).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    return want, u_of(dtype) * want.abs() + tiny_of(dtype) + (n[:, None] + 3) * F * size


@pytest.mark.parametrize("dtype, grad", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens, rows, dim, spread", [
    (0, 4, 8, 1), (1, 1, 1, 1), (1, 300, 8, 1), (40, 7, 3, 1), (513, 2000, 130, 1), (4096, 40, 264, 3), (5000, 1, 72, 1),
    (3000, 70001, 16, 2), (20000, 257, 8, 6), (2500, 5, 1030, 1),
    (8192, 300, 24, 2), (8193, 300, 24, 2), (20000, 300001, 8, 5), (33000, 2, 40, 1)])
def test_table_gradient(ctx, dtype, grad, tokens, rows, dim, spread):
    gen = torch.Generator("cuda").manual_seed(tokens + dim)
    d_out = normal(gen, tokens, dim, dtype=TYPES[dtype])
    ids = (torch.rand(tokens, device="cuda", generator=gen) ** spread * (rows + 2)).long() - 1     # some outside
    want, bound = gradient_want(d_out, ids, rows, 0.7, 0, TYPES[grad])
    got = ctx.embed_backward(d_out, ids, rows, 0.7, dtype=TYPES[grad])
    ctx.check_status()
    within(got, want, bound)
    again = ctx.embed_backward(d_out, ids.int(), rows, 0.7, dtype=TYPES[grad])
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", TYPES)
def test_table_gradient_added_to_what_is_there(ctx, dtype):
    gen = torch.Generator("cuda").manual_seed(4)
    t = TYPES[dtype]
    d_out, there = normal(gen, 700, 40, dtype=t), normal(gen, 300, 40, dtype=t)
    ids = torch.randint(0, 150, (700,), device="cuda", generator=gen) * 2          # every other row
    want, bound = gradient_want(d_out, ids, 300, 1.3, 0, t)
    want = want + there.double()
    got = there.clone()
    ctx.embed_backward_into(d_out, ids, got, 1.3, accumulate=True)
    ctx.check_status()
    within(got, want, bound + u_of(t) * want.abs() + 2 * F * (want.abs() + there.double().abs()))
    assert torch.equal(got[1::2], there[1::2])


@pytest.mark.parametrize("first", [0, 1, 4])
def test_table_gradient_of_rows_in_a_larger_tensor(ctx, first):
    gen = torch.Generator("cuda").manual_seed(first)
    wide, table = normal(gen, 900, 96, dtype=torch.bfloat16), normal(gen, 50, 88)
    d_out, d_table = wide[:, first:first + 70], table[:, first:first + 70]
    before = table.clone()
    ids = torch.randint(0, 50, (900,), device="cuda", generator=gen)
    want, bound = gradient_want(d_out, ids, 50, 1.0, 0, torch.float32)
    ctx.embed_backward_into(d_out, ids, d_table)
    ctx.check_status()
    within(d_table, want, bound)
    assert torch.equal(table[:, :first], before[:, :first]) and torch.equal(table[:, first + 70:], before[:, first + 70:])


def test_table_gradient_of_shards_is_the_whole_tables(ctx):
    """Vocabulary rows of a tensor axis: each shard has the very rows of the single device."""
    gen = torch.Generator("cuda").manual_seed(6)
    d_out = normal(gen, 3000, 64, dtype=torch.bfloat16)
    ids = (torch.rand(3000, device="cuda", generator=gen) ** 3 * 1000).long()
    whole = ctx.embed_backward(d_out, ids, 1000)
    for begin, end in ((0, 1), (1, 400), (400, 1000)):
        assert torch.equal(ctx.embed_backward(d_out, ids, end - begin, first_row=begin), whole[begin:end])
    ctx.check_status()


def test_embedding_rows_behind_two_to_the_32_bytes(ctx):
    """Offsets that pass 32 bits, in elements and bytes, on both sides."""
    rows, dim = 70000, 1 << 16                          # 4.6e9 elements
    table = torch.zeros(rows, dim, device="cuda", dtype=torch.bfloat16)
    table[-3:] = 2.0
    ids = torch.tensor([rows - 1, 0, rows - 3, -1], device="cuda")
    out = ctx.embed_forward(table, ids)
    assert out.amin(1).tolist() == [2.0, 0.0, 2.0, 0.0] and out.amax(1).tolist() == [2.0, 0.0, 2.0, 0.0]
    ids = torch.tensor([rows - 1, rows - 1, rows - 2], device="cuda")
    ctx.embed_backward_into(torch.ones(3, dim, device="cuda", dtype=torch.bfloat16), ids, table)
    ctx.check_status()
    assert table[-3:].amin(1).tolist() == [0.0, 1.0, 2.0] and table[-3:].amax(1).tolist() == [0.0, 1.0, 2.0]
    assert not table[:-3].any()


def test_table_gradient_agrees_with_differences(ctx):
    """<d_out, lookup(E + h D)> - <d_out, lookup(E - h D)> over 2 h is <dE, D>: the lookup is linear."""
    gen = torch.Generator("cuda").manual_seed(8)
    table, step, d_out = normal(gen, 60, 40), normal(gen, 60, 40), normal(gen, 500, 40)
    ids = torch.randint(-1, 60, (500,), device="cuda", generator=gen)
    up, down = (ctx.embed_forward(table + h * step, ids, 0.5).double() for h in (1.0, -1.0))
    change = ((up - down) * d_out.double()).sum() / 2
    inner = (ctx.embed_backward(d_out, ids, 60, 0.5).double() * step.double()).sum()
    size = (up.abs() + down.abs()).mul(d_out.double().abs()).sum()
    assert abs(change - inner) <= 500 * F * size


# ------------------------------------------------------------------ attention

def seen_of(batch, q_len, k_len, causal, q_lens, k_lens):
    i, j = torch.arange(q_len, device="cuda"), torch.arange(k_len, device="cuda")
    n = torch.full((batch,), q_len, device="cuda") if q_lens is None else q_lens.long().clamp(0, q_len)
    m = torch.full((batch,), k_len, device="cuda") if k_lens is None else k_lens.long().clamp(0, k_len)
    seen = (i < n[:, None])[:, :, None] & (j < m[:, None])[:, None]
    if causal:
        seen = seen & (j <= i[:, None] + (m - n)[:, None, None])
    return seen[:, None]                                 # [batch, 1, q, k]


def per_head(x, heads):
    """[batch, len, h, dim] in 64 bits as [batch, heads, len, dim], shared heads repeated."""
    return x.double().permute(0, 2, 1, 3).repeat_interleave(heads // x.shape[2], 1)


def no_padding(x, lens, length):
    """Padding takes no part: zeros, whatever it holds."""
    if lens is None:
        return x
    pad = torch.arange(length, device="cuda") >= lens.long().clamp(0, length)[:, None]
    return x.masked_fill(pad[:, :, None, None], 0.0)


def attention_want(q, k, v, scale, causal, q_lens, k_lens):
    heads = q.shape[2]
    seen = seen_of(q.shape[0], q.shape[1], k.shape[1], causal, q_lens, k_lens)
    q, k, v = no_padding(q, q_lens, q.shape[1]), no_padding(k, k_lens, k.shape[1]), no_padding(v, k_lens, k.shape[1])
    qh, kh, vh = (per_head(x, heads) for x in (q, k, v))
    s = (qh @ kh.transpose(-1, -2) * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
    # how far a score in float32 may be off: the product's dim terms, the scale, the exponent's range reduction
    off = ((q.shape[3] + 8) * F * (qh.abs() @ kh.abs().transpose(-1, -2)) * abs(scale)).masked_fill(~seen, 0.0)
    return seen, qh, kh, vh, p, lse, off


# the exponential's own error, the sums of up to k_len terms and the division, relative
def sums(n):
    return (n + 16) * F + 2.0 ** -21


def check_forward(ctx, q, k, v, scale, causal, q_lens=None, k_lens=None):
    out, lse = ctx.attention_forward(q, k, v, scale, causal, q_lens, k_lens)
    ctx.check_status()
    scale = q.shape[3] ** -0.5 if scale is None else scale
    _, _, _, vh, p, want_lse, off = attention_want(q, k, v, scale, causal, q_lens, k_lens)
    u, t, n = u_of(q.dtype), tiny_of(q.dtype), k.shape[1]
    most = off.amax(-1) if n else torch.zeros_like(want_lse)
    want = p @ vh
    # a probability is off by its score's error, twice (its own and the sum's); rounded to the type relative to the row's
    # largest, which is at least 1 / 256 of the largest number the kernel may hold; the sum of n of them in float32
    rel = u + sums(n) + 2 * most[..., None]
    bound = u * want.abs() + t + rel * (p @ vh.abs()) + 256 * t * vh.abs().sum(-2, keepdim=True)
    within(out.permute(0, 2, 1, 3), want, bound, "out")
    finite = want_lse != -math.inf
    assert torch.equal(lse == -math.inf, ~finite)
    within(lse[finite], want_lse[finite], (most + sums(n) + 4 * F * want_lse.abs())[finite], "lse")
    return out, lse


def check_backward(ctx, q, k, v, d_out, scale, causal, q_lens=None, k_lens=None):
    out, lse = ctx.attention_forward(q, k, v, scale, causal, q_lens, k_lens)
    got = ctx.attention_backward(q, k, v, out, lse, d_out, scale, causal, q_lens, k_lens)
    ctx.check_status()
    scale = q.shape[3] ** -0.5 if scale is None else scale
    seen, qh, kh, vh, p, _, off = attention_want(q, k, v, scale, causal, q_lens, k_lens)
    heads, kv_heads = q.shape[2], k.shape[2]
    gh, oh = per_head(no_padding(d_out, q_lens, q.shape[1]), heads), per_head(out, heads)
    # the gradient's definition with the log-sum-exp and output that it is given
    s = (qh @ kh.transpose(-1, -2) * scale).masked_fill(~seen, -math.inf)
    lse = lse.double()
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
    delta, dp = (gh * oh).sum(-1, keepdim=True), gh @ vh.transpose(-1, -2)
    size = gh.abs() @ vh.abs().transpose(-1, -2) + (gh * oh).abs().sum(-1, keepdim=True)
    ds = p * (dp - delta)
    u, t, d = u_of(q.dtype), tiny_of(q.dtype), q.shape[3]
    rel = sums(8) + off + 4 * F * lse.masked_fill(lse == -math.inf, 0.0).abs()[..., None]    # of a probability
    # P is rounded to the type (a type with subnormals holds it 2^12 as large), dS as well (there it is
    # scaled so that the bound of |dP - delta| of a key head's queries, at most |d_out| (|v| + |out|), is a large number of the type)
    p_off = (u + rel) * p + t / 4096 * seen
    largest = (gh.norm(dim=-1).amax() if gh.numel() else 0.0) * (vh.norm(dim=-1).amax() if vh.numel() else 0.0)
    ds_off = u * ds.abs() + (rel + (d + 4) * F) * p * size + 2 * t * largest * 2.0 ** -12 * seen

    def shared(x):
        return x.unflatten(1, (kv_heads, heads // kv_heads)).sum(2)
    n_k, n_q = k.shape[1], q.shape[1] * (heads // kv_heads)
    want = [ds @ kh * scale, shared(ds.transpose(-1, -2) @ qh) * scale, shared(p.transpose(-1, -2) @ gh)]
    bound = [(ds_off + n_k * F * ds.abs()) @ kh.abs() * abs(scale),
             shared((ds_off + n_q * F * ds.abs()).transpose(-1, -2) @ qh.abs()) * abs(scale),
             shared((p_off + n_q * F * p).transpose(-1, -2) @ gh.abs())]
    for name, g, w, b in zip(("d_q", "d_k", "d_v"), got, want, bound):
        within(g.permute(0, 2, 1, 3), w, b * (1 + u) + (u + 4 * F) * w.abs() + t, name)
    return got


def tensors(seed, batch, q_len, k_len, heads, kv_heads, dim, dtype, size=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)
    t = TYPES[dtype]
    return (normal(gen, batch, q_len, heads, dim, dtype=t), normal(gen, batch, k_len, kv_heads, dim, dtype=t),
            normal(gen, batch, k_len, kv_heads, dim, dtype=t), normal(gen, batch, q_len, heads, dim, dtype=t, size=size))


SHAPES = [(1, 1, 1, 1, 1, 128), (2, 1, 1, 3, 3, 8), (1, 1, 300, 4, 2, 128), (1, 300, 1, 2, 1, 64), (2, 127, 129, 2, 2, 128),
          (1, 128, 128, 4, 1, 128), (1, 256, 256, 2, 2, 64), (1, 257, 255, 3, 1, 128), (2, 200, 333, 4, 2, 80), (1, 333, 200, 6, 2, 40),
          (1, 640, 640, 7, 1, 96), (3, 65, 513, 2, 1, 16), (1, 513, 1025, 2, 2, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_forward(ctx, dtype, causal, shape):
    q, k, v, _ = tensors(1, *shape, dtype)
    check_forward(ctx, q, k, v, None, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_backward(ctx, dtype, causal, shape):
    q, k, v, d_out = tensors(2, *shape, dtype)
    check_backward(ctx, q, k, v, d_out, None, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens, k_lens", [([300, 0, 1, 129], [300, 300, 300, 300]), ([300, 200, 5, 128], [17, 0, 1, 257]),
                                            ([128, 256, 300, 7], [128, 256, 300, 7]), ([999, -5, 3, 300], [999, 4, -1, 2]),
                                            (None, [1, 64, 128, 0]), ([1, 64, 128, 0], None)])
def test_attention_of_padded_sequences(ctx, dtype, causal, q_lens, k_lens):
    """Padding holds NaN and infinities: nothing of it is used, and zeros are written for it."""
    q, k, v, d_out = tensors(3, 4, 300, 300, 4, 2, 64, dtype)
    lens = [None if n is None else torch.tensor(n, device="cuda", dtype=torch.int32) for n in (q_lens, k_lens)]
    for x, n in ((q, lens[0]), (d_out, lens[0]), (k, lens[1]), (v, lens[1])):
        if n is not None:
            for b in range(4):
                x[b, max(0, int(n[b])):] = math.nan
                x[b, max(0, int(n[b])) + 1:] = math.inf
    check_forward(ctx, q, k, v, None, causal, *lens)
    check_backward(ctx, q, k, v, d_out, None, causal, *lens)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 4097, 2, 1, 128), (2, 250, 6000, 4, 2, 64), (1, 256, 4300, 3, 3, 96), (3, 5, 9000, 2, 2, 40),
                                   (1, 4500, 256, 2, 1, 128), (2, 6001, 3, 4, 2, 64)])
def test_attention_of_few_rows_and_a_long_axis(ctx, dtype, causal, shape):
    """Chunks of the long axis, joined: with lengths that leave chunks, and whole sequences, without keys or queries."""
    q, k, v, d_out = tensors(16, *shape, dtype)
    check_forward(ctx, q, k, v, None, causal)
    check_backward(ctx, q, k, v, d_out, None, causal)
    batch, q_len, k_len = shape[:3]
    lens = [torch.tensor([n, n // 3, 0][:batch], device="cuda", dtype=torch.int32) for n in (q_len, k_len)]
    for x, n, length in ((q, lens[0], q_len), (d_out, lens[0], q_len), (k, lens[1], k_len), (v, lens[1], k_len)):
        for b in range(batch):
            x[b, int(n[b]):] = math.nan
    check_forward(ctx, q, k, v, None, causal, *lens)
    check_backward(ctx, q, k, v, d_out, None, causal, *lens)


def test_attention_gradients_of_the_most_heads_before_a_long_axis(ctx):
    """One key, so that every probability is 1: dV is the sum of dO, dK nothing but rounding, and so is dQ."""
    q, k, v, d_out = tensors(17, 1, 4097, 1, 32768, 32768, 8, "bf16")
    out, lse = ctx.attention_forward(q, k, v, None, False)
    d_q, d_k, d_v = ctx.attention_backward(q, k, v, out, lse, d_out, None, False)
    ctx.check_status()
    assert torch.equal(out, v.expand_as(out))
    # P in 32 bits is off by less than 2^-9, so that it is rounded to 1; 4097 terms in 32 bits, one rounding
    want, sizes = d_out.double().sum(1, keepdim=True), d_out.double().abs().sum(1, keepdim=True)
    u = u_of(torch.bfloat16)
    within(d_v, want, 4097 * F * sizes + u * want.abs())
    # dO V^T and delta are sums of the same 8 products, each off by at most 8 roundings; dS by twice that and its own
    ds = 2 * 10 * F * (d_out.double().abs() * v.double().abs()).sum(-1, keepdim=True)
    scale = 8 ** -0.5
    within(d_q, torch.zeros_like(d_q).double(), ds * k.double().abs() * scale * (1 + 4 * u))
    within(d_k, torch.zeros_like(d_k).double(), (ds * q.double().abs()).sum(1, keepdim=True) * scale * (1 + 4 * u))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 4.0])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_scales(ctx, dtype, scale):
    """No scores at all, negative ones, and ones so far apart that a row has one key."""
    q, k, v, d_out = tensors(4, 1, 200, 260, 2, 1, 128, dtype)
    check_forward(ctx, q, k, v, scale, True)
    check_backward(ctx, q, k, v, d_out, scale, True)


@pytest.mark.parametrize("size", [1e-7, 1e-3, 300.0])
def test_attention_gradients_of_any_size_in_half_precision(ctx, size):
    q, k, v, d_out = tensors(5, 1, 150, 150, 2, 2, 64, "f16", size=size)
    check_backward(ctx, q, k, v, d_out, None, True)


def test_attention_growing_scores(ctx):
    """Every block of keys beats the last one's largest score by far, then falls: the running maximum moves."""
    q, k, v, d_out = tensors(6, 1, 140, 1100, 2, 2, 128, "bf16")
    ramp = torch.cat([torch.linspace(0, 6, 700), torch.linspace(6, -6, 400)]).to("cuda")
    k = (k * 0.2 + ramp[None, :, None, None] * 0.3).bfloat16()
    q = (q * 0.2 + 0.3).bfloat16()
    check_forward(ctx, q, k, v, 0.5, False)
    check_backward(ctx, q, k, v, d_out, 0.5, False)


@pytest.mark.parametrize("order", [(0, 2, 1, 3), (2, 0, 1, 3), (1, 2, 0, 3)])
def test_attention_of_any_strides(ctx, order):
    """[batch, len, heads, dim] as views of other orders, of wider rows and of one tensor that holds all three."""
    gen = torch.Generator("cuda").manual_seed(7)
    back = [order.index(i) for i in range(4)]

    def view(n, heads):
        shape = [2, n, heads, 64]
        return normal(gen, *[shape[i] for i in order], dtype=torch.bfloat16).permute(back)
    q, k, v, d_out = view(150, 4), view(200, 2), view(200, 2), view(150, 4)
    plain = [x.contiguous() for x in (q, k, v, d_out)]
    out, lse = ctx.attention_forward(q, k, v)
    want, want_lse = ctx.attention_forward(*plain[:3])
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    grads = [torch.empty_like(x) for x in (q, k, v)]        # the views' own strides
    assert grads[0].stride() == q.stride()
    ctx.attention_backward_into(q, k, v, out, lse, d_out, *grads)
    for g, w in zip(grads, ctx.attention_backward(*plain[:3], out, lse, plain[3])):
        assert torch.equal(g, w)
    qkv = normal(gen, 2, 130, 8, 72, dtype=torch.bfloat16)
    q, k, v = qkv[:, :, :4, :64], qkv[:, :, 4:6, :64], qkv[:, :, 6:, 8:]
    assert torch.equal(ctx.attention_forward(q, k, v)[0], ctx.attention_forward(*[x.contiguous() for x in (q, k, v)])[0])
    ctx.check_status()


def test_attention_of_strides_behind_two_to_the_31(ctx):
    """Tokens 2^29 elements apart and sequences 2^31: a view of a few rows of a very large tensor."""
    q, k, v, d_out = tensors(17, 2, 4, 4, 1, 1, 64, "bf16")
    hold = torch.zeros((1 << 32) + 256, device="cuda", dtype=torch.bfloat16)
    far = [hold.as_strided((2, 4, 1, 64), (1 << 31, 1 << 29, 64, 1), 64 * i) for i in range(4)]
    for f, x in zip(far, (q, k, v, d_out)):
        f.copy_(x)
    out, lse = ctx.attention_forward(*far[:3])
    want = ctx.attention_forward(q, k, v)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    grads = ctx.attention_backward(*far[:3], out, lse, far[3])
    for g, w in zip(grads, ctx.attention_backward(q, k, v, out, lse, d_out)):
        assert torch.equal(g, w)
    ctx.check_status()


def test_attention_leaves_what_lies_around_its_results(ctx):
    q, k, v, d_out = tensors(8, 2, 130, 140, 2, 1, 40, "bf16")
    out, lse = ctx.attention_forward(q, k, v)
    hold = [torch.full((2, n + 2, h + 1, 56), 7.0, device="cuda", dtype=torch.bfloat16) for n, h in ((130, 2), (130, 2), (140, 1), (140, 1))]
    part = [x[:, 1:-1, :-1, 8:48] for x in hold]
    ctx.attention_forward_into(q, k, v, part[0], lse)
    ctx.attention_backward_into(q, k, v, out, lse, d_out, *part[1:])
    want = (out,) + ctx.attention_backward(q, k, v, out, lse, d_out)
    for x, p, w in zip(hold, part, want):
        assert torch.equal(p, w)
        p.fill_(7.0)
        assert x.eq(7.0).all()


def test_attention_of_shards_is_the_whole_batchs(ctx):
    """Sequences of a data axis and key heads of a tensor axis have the single device's bits, on every run."""
    q, k, v, d_out = tensors(9, 3, 270, 270, 8, 4, 128, "bf16")
    out, lse = ctx.attention_forward(q, k, v)
    grads = ctx.attention_backward(q, k, v, out, lse, d_out)
    assert all(torch.equal(a, b) for a, b in zip(grads, ctx.attention_backward(q, k, v, out, lse, d_out)))
    for b in range(3):
        o, l = ctx.attention_forward(q[b:b + 1], k[b:b + 1], v[b:b + 1])
        g = ctx.attention_backward(q[b:b + 1], k[b:b + 1], v[b:b + 1], o, l, d_out[b:b + 1])
        assert torch.equal(o, out[b:b + 1]) and all(torch.equal(x, y[b:b + 1]) for x, y in zip(g, grads))
    for h in (0, 2):
        part = [q[:, :, 2 * h:2 * h + 4], k[:, :, h:h + 2], v[:, :, h:h + 2]]
        o, l = ctx.attention_forward(*part)
        g = ctx.attention_backward(*part, o, l, d_out[:, :, 2 * h:2 * h + 4])
        assert torch.equal(o, out[:, :, 2 * h:2 * h + 4])
        assert torch.equal(g[0], grads[0][:, :, 2 * h:2 * h + 4]) and torch.equal(g[1], grads[1][:, :, h:h + 2])
        assert torch.equal(g[2], grads[2][:, :, h:h + 2])


def test_attention_gradients_agree_with_differences(ctx):
    """A step h D of q, k or v changes <d_out, out> by 2 h <gradient, D> + O(h^3), out taken from the definition in 64 bits."""
    q, k, v, d_out = tensors(10, 1, 70, 90, 2, 1, 64, "f16")
    out, lse = ctx.attention_forward(q, k, v)
    grads = ctx.attention_backward(q, k, v, out, lse, d_out)
    gen = torch.Generator("cuda").manual_seed(11)
    for at, grad in enumerate(grads):
        d = normal(gen, *grad.shape).double()
        h = 1e-4
        values = []
        for sign in (1, -1):
            x = [t.double() for t in (q, k, v)]
            x[at] = x[at] + sign * h * d
            _, _, _, vh, p, _, _ = attention_want(*x, 0.125, True, None, None)
            values.append(((p @ vh).permute(0, 2, 1, 3) * d_out.double()).sum())
        change, inner = (values[0] - values[1]) / (2 * h), (grad.double() * d).sum()
        # each element of the gradient has a few roundings of u of its terms; their signs are independent of D's
        size = (grad.double().abs() * d.abs()).sum() + d_out.double().abs().sum()
        assert abs(change - inner) <= 8 * u_of(torch.float16) * size


def test_attention_long_in_one_call(ctx):
    """A long axis on both sides, against the definition of a few rows."""
    q, k, v, d_out = tensors(12, 1, 5000, 9001, 2, 1, 128, "bf16")
    out, lse = ctx.attention_forward(q, k, v)
    rows = [0, 127, 128, 2500, 4999]
    s = torch.einsum("ihd,jd->hij", q[0, rows].double(), k[0, :, 0].double()) * 128 ** -0.5
    hide = torch.arange(9001, device="cuda") > torch.tensor(rows, device="cuda")[:, None] + 4001
    s = s.masked_fill(hide, -math.inf)
    p = torch.softmax(s, -1)
    want = p @ v[0, :, 0].double()
    bound = u_of(torch.bfloat16) * (want.abs() + 1.1 * (p @ v[0, :, 0].double().abs())) + 1e-5
    within(out[0, rows].permute(1, 0, 2), want, bound)
    within(lse[0, :, rows], torch.logsumexp(s, -1), torch.full_like(lse[0, :, rows], 1e-4).double())
    d_q, _, _ = ctx.attention_backward(q, k, v, out, lse, d_out)
    g = d_out[0, rows].double().permute(1, 0, 2)
    dp = g @ v[0, :, 0].double().t()
    ds = p * (dp - (g * out[0, rows].double().permute(1, 0, 2)).sum(-1, keepdim=True))
    want = ds @ k[0, :, 0].double() * 128 ** -0.5
    size = ((ds.abs() * 1.1 * u_of(torch.bfloat16) + p * 1e-4) @ k[0, :, 0].double().abs()) * 128 ** -0.5
    within(d_q[0, rows].permute(1, 0, 2), want, size + u_of(torch.bfloat16) * want.abs())


# ------------------------------------------------------------------ together

def step(ctx, table, tokens, weights, shape, seed, first_row_of_batch=0):
    """One training step's run of the operators on some sequences: embed, dropout, attention, dropout with residual; and back."""
    batch, length, heads, kv_heads, dim = shape
    hidden = heads * dim
    flat = tokens.reshape(-1)
    x = ctx.embed_forward(table, flat, scale=2.0)
    first = first_row_of_batch * hidden
    h = ctx.dropout(x, 0.1, seed, stream=0, first=first)
    q = h.view(batch, length, heads, dim)
    k, v = q[:, :, :kv_heads], q[:, :, kv_heads:2 * kv_heads]
    out, lse = ctx.attention_forward(q, k, v)
    y = ctx.dropout(out.view(-1, hidden), 0.2, seed, stream=1, residual=h, first=first)
    g = weights.reshape(-1, hidden)                     # the loss is <weights, y>
    d_attn = ctx.dropout(g, 0.2, seed, stream=1, first=first)
    d_q, d_k, d_v = ctx.attention_backward(q, k, v, out, lse, d_attn.view_as(q))
    d_h = g.float().view(batch, length, heads, dim) + d_q.float()
    d_h[:, :, :kv_heads] += d_k.float()
    d_h[:, :, kv_heads:2 * kv_heads] += d_v.float()
    d_x = ctx.dropout(d_h.view(-1, hidden), 0.1, seed, stream=0, first=first)
    return y, d_x


def test_a_step_on_shards_is_the_single_devices(ctx):
    """The verification protocol on these operators: two logical devices with half of the batch each."""
    gen = torch.Generator("cuda").manual_seed(13)
    shape, vocab = (4, 150, 6, 2, 64), 500
    table = normal(gen, vocab, 384, dtype=torch.bfloat16)
    tokens = torch.randint(0, vocab, (4, 150), device="cuda", generator=gen)
    weights = normal(gen, 4, 150, 384, dtype=torch.bfloat16)
    y, d_x = step(ctx, table, tokens, weights, shape, 99)
    grad = ctx.embed_backward(d_x, tokens.reshape(-1), vocab, scale=2.0, dtype=torch.float32)
    total = None
    for b in (0, 2):
        part = step(ctx, table, tokens[b:b + 2], weights[b:b + 2], (2,) + shape[1:], 99, first_row_of_batch=b * 150)
        rows = slice(b * 150, (b + 2) * 150)
        assert torch.equal(part[0], y[rows]) and torch.equal(part[1], d_x[rows])
        share = ctx.embed_backward(part[1], tokens[b:b + 2].reshape(-1), vocab, scale=2.0, dtype=torch.float32)
        total = share if total is None else total + share
    assert (total - grad).norm() <= 1e-5 * grad.norm()          # the protocol's own bound
    # and the gradient is the loss's: autograd of the same step in 64 bits, masks taken from the operators
    e = table.double().requires_grad_()
    ones = torch.ones(600, 384, device="cuda")
    h = e[tokens.reshape(-1)] * 2.0 * ctx.dropout(ones, 0.1, 99, stream=0).double()
    q = h.view(4, 150, 6, 64)
    _, _, _, vh, p, _, _ = attention_want(q, q[:, :, :2], q[:, :, 2:4], 0.125, True, None, None)
    out = (p @ vh).permute(0, 2, 1, 3).reshape(600, 384)
    (out * ctx.dropout(ones, 0.2, 99, stream=1).double() + h).mul(weights.reshape(600, 384).double()).sum().backward()
    # a chain of half a dozen roundings to bfloat16, each relative to what it rounds
    assert (grad.double() - e.grad).norm() <= 6 * u_of(torch.bfloat16) * e.grad.norm()
    ctx.check_status()


def test_operators_on_two_streams_at_once(ps):
    """Two contexts whose calls overlap on the device: no work space is shared."""
    contexts = [ps.Context(0, torch.cuda.Stream()) for _ in range(2)]
    gen = torch.Generator("cuda").manual_seed(18)
    inputs = []
    for i in range(2):
        q, k, v, d_out = tensors(19 + i, 2, 700, 900, 8, 4, 128 if i else 64, "f16" if i else "bf16")
        rows = normal(gen, 9000 + i, 256, dtype=torch.bfloat16)
        inputs.append((q, k, v, d_out, rows, torch.randint(0, 50, (9000 + i,), device="cuda", generator=gen)))

    def every(ctx, q, k, v, d_out, rows, ids):
        out, lse = ctx.attention_forward(q, k, v)
        return (out, lse) + ctx.attention_backward(q, k, v, out, lse, d_out) + (
            ctx.embed_backward(rows, ids, 60), ctx.dropout(rows, 0.3, 5))
    torch.cuda.synchronize()
    want = []
    for ctx, x in zip(contexts, inputs):
        want.append(every(ctx, *x))
        torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for _ in range(3):
            got = [every(ctx, *x) for ctx, x in zip(contexts, inputs)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))
    for ctx in contexts:
        ctx.check_status()


def test_operators_on_other_streams_and_in_graphs(ps):
    """A context of its own stream, and every operator captured once and replayed on new data, two graphs in turn."""
    side = torch.cuda.Stream()
    ctx = ps.Context(0, side)
    gen = torch.Generator("cuda").manual_seed(14)
    q, k, v, d_out = tensors(15, 2, 140, 140, 4, 2, 64, "bf16")
    qh, kh, vh, gh = tensors(16, 1, 9, 5000, 2, 1, 128, "f16")       # (with norms and chunks)
    table = normal(gen, 90, 256, dtype=torch.bfloat16)
    tokens = torch.randint(0, 90, (280,), device="cuda", generator=gen)
    rows = normal(gen, 280, 256, dtype=torch.bfloat16)

    def every():
        out, lse = ctx.attention_forward(q, k, v)
        half = ctx.attention_forward(qh, kh, vh)
        return (out, lse) + half + ctx.attention_backward(qh, kh, vh, *half, gh) + ctx.attention_backward(q, k, v, out, lse, d_out) + (
            ctx.embed_forward(table, tokens), ctx.embed_backward(rows, tokens, 90), ctx.dropout(rows, 0.1, 3, residual=rows))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = every()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = every()
            graphs.append((graph, got))
        for graph, got in graphs + graphs[::-1]:
            for t in got:
                t.fill_(1.0)
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        for t in (q, rows):
            t.mul_(-0.5)
        tokens.copy_((tokens + 17) % 90)
        want = every()
        for graph, got in graphs:
            graph.replay()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    side.synchronize()
    ctx.check_status()
    del graphs, graph, got
