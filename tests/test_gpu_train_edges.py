"""Operators of a training step where sizes, types or the order of calls are at an edge, against their definitions
in 64 bits.  Bounds are counted as in test_gpu_train_operators.py."""
import math

import pytest
import torch

from test_gpu_train_operators import F, TYPES, gradient_want, normal, tensors, tiny_of, u_of, within

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


def far_keys(n, at, below, dim, heads, seed, spread):
    """One query whose key `at` has a value of zero and whose other keys' scores lie `below` (and up to `spread` more) under
    that one's, in numbers that half precision holds."""
    gen = torch.Generator("cuda").manual_seed(seed)
    q = torch.zeros(1, 1, heads, dim, device="cuda", dtype=torch.float16)
    q[..., 0] = 1.0
    k = torch.zeros(1, n, heads, dim, device="cuda", dtype=torch.float16)
    k[..., 0] = -below - spread * torch.rand(1, n, heads, device="cuda", generator=gen)
    k[:, at, :, 0] = 0.0
    v = torch.rand(1, n, heads, dim, device="cuda", generator=gen).add_(0.5).half()
    v[:, at] = 0.0
    return q, k, v


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("below, spread", [(9.0, 0.0), (14.0, 0.0), (14.0, 1.0), (16.5, 0.0), (16.5, 1.0)])
@pytest.mark.parametrize("n, at", [(2000, 0), (2000, 1990), (2000, 700), (8192, 5), (8192, 8191)])
def test_half_precision_keeps_small_probabilities(ctx, dim, below, spread, n, at):
    """All of the output comes from keys far below the row's largest."""
    q, k, v = far_keys(n, at, below, dim, 2, n + at, spread)
    out, lse = ctx.attention_forward(q, k, v, 1.0, False)
    ctx.check_status()
    s = k[0, :, :, 0].double().t()                              # [head, key]: q is a unit vector
    want = (torch.softmax(s, -1)[:, None] @ v[0].double().transpose(0, 1))[:, 0]
    # A probability: rounded to half, relative; where that is subnormal, by half of 2^-24, of a number that is held 2^7 as large (the
    # row's largest number is at least 2^7, so is the sum that divides it); the exponent in float32, off by 4 roundings of
    # numbers up to (below + spread) log2 e + 7; the exponential itself; n terms summed twice and divided.
    u, exponent = u_of(torch.float16), 4 * F * ((below + spread) * 1.4427 + 7)
    bound = (2 * u + exponent + (2 * n + 16) * F + 2.0 ** -21) * want + 2.0 ** -32 * v[0].double().sum(0)
    within(out[0, 0], want, bound, "out")
    within(lse[0, :, 0], torch.logsumexp(s, -1), torch.full_like(lse[0, :, 0], 1e-5 + (n + 16) * F).double(), "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("step", [0.7, 1.0, 2.0, 3.0, 8.0, 20.0])
def test_attention_whose_largest_score_moves_with_every_block(ctx, dtype, step):
    """Blocks of 128 keys with equal scores, each `step` above the last one's and by that much heavier: whether the sums
    are rescaled or not, no weight leaves the type's range."""
    blocks, heads, dim = 12, 2, 64
    gen = torch.Generator("cuda").manual_seed(int(step * 10))
    q = torch.zeros(1, 300, heads, dim, device="cuda", dtype=TYPES[dtype])
    q[..., 0] = 1.0
    k = torch.zeros(1, 128 * blocks, heads, dim, device="cuda", dtype=TYPES[dtype])
    k[..., 0] = (torch.arange(blocks, device="cuda") * step).repeat_interleave(128)[None, :, None]
    v = normal(gen, 1, 128 * blocks, heads, dim, dtype=TYPES[dtype])
    out, lse = ctx.attention_forward(q, k, v, 1.0, False)
    ctx.check_status()
    s = k[0, :, 0, 0].double()
    p = torch.softmax(s, -1)
    want, size = (torch.einsum("j,jhd->hd", p, x) for x in (v[0].double(), v[0].double().abs()))
    u, n = u_of(TYPES[dtype]), 128 * blocks
    most = float(s.abs().max()) * 1.4427 + 7
    bound = u * want.abs() + tiny_of(TYPES[dtype]) + (u + 4 * F * most + (2 * n + 16) * F + 2.0 ** -21) * size + 2.0 ** -32 * v[0].double().abs().sum(0)
    within(out[0], want.expand(300, heads, dim), bound, "out")
    within(lse[0], torch.logsumexp(s, -1).expand(heads, 300), torch.full((heads, 300), (n + 16) * F + 8 * F * most, device="cuda").double(), "lse")


@pytest.mark.parametrize("size", [100.0, 700.0, 1000.0, 1500.0, 2000.0])
@pytest.mark.parametrize("at", [0, 130, 511])
def test_half_precision_with_scores_of_millions(ctx, size, at):
    """One key far above the others, at scores (up to 5e8) of which float32 holds whole numbers only: its value is the output."""
    q = torch.full((1, 200, 1, 128), size, device="cuda", dtype=torch.float16)
    k = torch.full((1, 512, 1, 128), 0.5 * size, device="cuda", dtype=torch.float16)
    k[:, at] = size
    v = normal(torch.Generator("cuda").manual_seed(at), 1, 512, 1, 128, dtype=torch.float16)
    out, lse = ctx.attention_forward(q, k, v, None, False)
    ctx.check_status()
    # the one weight cancels but for its own rounding to half and the division's; the others are zero
    want = v[0, at].double().expand(200, 1, 128)
    within(out[0], want, 2 * u_of(torch.float16) * want.abs() + 4 * F * want.abs() + tiny_of(torch.float16))
    score = size * size * 128 * 128 ** -0.5
    within(lse[0, 0], torch.full((200,), score, device="cuda").double(), torch.full((200,), (128 + 8) * F * score, device="cuda").double())


@pytest.mark.parametrize("dtype, dim, q_len, k_len, causal", [("bf16", 64, 700, 700, True), ("f16", 64, 700, 700, True), ("bf16", 128, 500, 900, False),
                                                             ("f16", 128, 900, 500, True), ("bf16", 64, 3, 4500, True), ("f16", 128, 4500, 3, False)])
def test_attention_gradients_with_whatever_the_work_buffer_holds(ctx, ps, dtype, dim, q_len, k_len, causal):
    """One buffer for calls in a row on operands that differ, and between them bytes of all sorts in it: the rows that a call reads are its own."""
    cases = []
    for seed in (22, 23):
        q, k, v, d_out = tensors(seed, 2, q_len, k_len, 4, 2, dim, dtype)
        out, lse = ctx.attention_forward(q, k, v, None, causal)
        cases.append(((q, k, v, out, lse, d_out), ctx.attention_backward(q, k, v, out, lse, d_out, None, causal)))
    work = torch.empty(ps.Context.attention_backward_bytes(2, q_len, k_len, 4, 2, dim), dtype=torch.uint8, device="cuda")
    results = []
    for turn in range(12):
        if turn % 4 < 3:
            work.fill_((0, 1, 255)[turn % 4])                       # (zeros, whole numbers that are not zero, NaN)
        operands, want = cases[turn % 2]
        grads = [torch.empty_like(t) for t in operands[:3]]
        ctx.attention_backward_into(*operands, *grads, causal=causal, work=work)
        results.append((grads, want))
    ctx.check_status()
    for grads, want in results:
        assert all(torch.equal(g, w) for g, w in zip(grads, want))


# ------------------------------------------------------------------ the table's gradient from more than 8192 tokens

def some_ids(gen, tokens, rows, spread):
    """Low rows are frequent (lists of thousands), most rows have none, some tokens name no row."""
    return (torch.rand(tokens, device="cuda", generator=gen) ** spread * (rows + 2)).long() - 1


# what is compiled: packs of 16 bytes or single elements, one or two of them a lane (above 2^25 elements of the table); columns in
# one part or several; pieces of 32 in one wave or many; lists with and without pieces of 1024; a sort's block with one tile or more
LARGE = [(9000, 300, 130, 2), (9000, 300, 1030, 2), (9000, 5, 1032, 1), (20000, 40000, 1024, 5), (9000, 40000, 901, 4), (8193, 33000, 1040, 1),
         (20000, 9000, 4100, 3), (12000, 260, 4096, 2)]


@pytest.mark.parametrize("dtype, grad", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("tokens, rows, dim, spread", LARGE)
def test_table_gradient_of_many_tokens(ctx, dtype, grad, tokens, rows, dim, spread):
    gen = torch.Generator("cuda").manual_seed(tokens + dim)
    d_out = normal(gen, tokens, dim, dtype=TYPES[dtype])
    ids = some_ids(gen, tokens, rows, spread)
    want, bound = gradient_want(d_out, ids, rows, 0.7, 0, TYPES[grad])
    got = ctx.embed_backward(d_out, ids, rows, 0.7, dtype=TYPES[grad])
    ctx.check_status()
    within(got, want, bound)
    assert torch.equal(got, ctx.embed_backward(d_out, ids.int(), rows, 0.7, dtype=TYPES[grad]))


@pytest.mark.parametrize("tokens, rows, dim, spread", [(303104, 1000, 8, 1), (303105, 1000, 8, 1), (310000, 300001, 5, 3), (700001, 30, 3, 2), (650000, 128000, 16, 4)])
def test_table_gradient_with_several_tiles_a_block_of_the_sort(ctx, tokens, rows, dim, spread):
    gen = torch.Generator("cuda").manual_seed(tokens)
    d_out = normal(gen, tokens, dim, dtype=torch.bfloat16)
    ids = some_ids(gen, tokens, rows, spread)
    want, bound = gradient_want(d_out, ids, rows, 1.0, 0, torch.float32)
    got = ctx.embed_backward(d_out, ids, rows, dtype=torch.float32)
    ctx.check_status()
    within(got, want, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, rows, dim", [(0, 50, 24), (9000, 300, 40), (9000, 300, 131), (9000, 40000, 1024), (20000, 40000, 901)])
def test_table_gradient_of_many_tokens_added_to_what_is_there(ctx, dtype, tokens, rows, dim):
    gen = torch.Generator("cuda").manual_seed(tokens + rows)
    t = TYPES[dtype]
    d_out, there = normal(gen, tokens, dim, dtype=t), normal(gen, rows, dim, dtype=t)
    ids = (torch.rand(tokens, device="cuda", generator=gen) ** 3 * (rows // 2)).long() * 2              # every other row
    want, bound = gradient_want(d_out, ids, rows, 1.3, 0, t)
    want = want + there.double()
    got = there.clone()
    ctx.embed_backward_into(d_out, ids, got, 1.3, accumulate=True)
    ctx.check_status()
    within(got, want, bound + u_of(t) * want.abs() + 2 * F * (want.abs() + there.double().abs()))
    assert torch.equal(got[1::2], there[1::2])


@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("rows, dim, first, stride", [(50, 70, 0, 88), (50, 72, 8, 88), (50, 70, 1, 89), (50, 264, 4, 280), (30000, 1120, 8, 1144), (30000, 1121, 3, 1127)])
def test_table_gradient_of_many_tokens_into_rows_of_a_larger_tensor(ctx, grad, rows, dim, first, stride):
    gen = torch.Generator("cuda").manual_seed(first + dim)
    wide, table = normal(gen, 9000, stride, dtype=torch.bfloat16), normal(gen, rows, stride, dtype=TYPES[grad])
    d_out, d_table = wide[:, first:first + dim], table[:, first:first + dim]
    before = table.clone()
    ids = some_ids(gen, 9000, rows, 2)
    want, bound = gradient_want(d_out, ids, rows, 1.0, 0, TYPES[grad])
    ctx.embed_backward_into(d_out, ids, d_table)
    ctx.check_status()
    within(d_table, want, bound)
    assert torch.equal(table[:, :first], before[:, :first]) and torch.equal(table[:, first + dim:], before[:, first + dim:])


@pytest.mark.parametrize("rows, dim, begins", [(1000, 64, (0, 1, 400)), (1000, 65, (0, 999)), (45000, 1024, (0, 7, 40000))])
def test_table_gradient_of_many_tokens_on_shards_is_the_whole_tables(ctx, rows, dim, begins):
    """A shard of the vocabulary has the very rows of the single device, also where the two take another number of packs a lane."""
    gen = torch.Generator("cuda").manual_seed(6)
    d_out = normal(gen, 12000, dim, dtype=torch.bfloat16)
    ids = some_ids(gen, 12000, rows, 3)
    whole = ctx.embed_backward(d_out, ids, rows)
    for begin, end in zip(begins, begins[1:] + (rows,)):
        assert torch.equal(ctx.embed_backward(d_out, ids, end - begin, first_row=begin), whole[begin:end])
    ctx.check_status()


# ------------------------------------------------------------------ streams

def all_operators(ctx, x):
    q, k, v, d_out, rows, ids = x
    out, lse = ctx.attention_forward(q, k, v)
    into = torch.empty_like(rows)
    ctx.dropout_into(rows, into, 0.2, 9)
    few = ctx.attention_forward(q[:, :1], k, v)                     # (in chunks, with a work buffer)
    return (out, lse, into) + few + ctx.attention_backward(q, k, v, out, lse, d_out) + (
        ctx.embed_forward(rows, ids), ctx.embed_backward(rows, ids, 50), ctx.dropout(rows, 0.3, 5, residual=rows))


def operands(seed):
    q, k, v, d_out = tensors(seed, 1, 300, 4200, 4, 2, 64, "f16")
    gen = torch.Generator("cuda").manual_seed(seed)
    return q, k, v, d_out, normal(gen, 400, 256, dtype=torch.bfloat16), torch.randint(0, 50, (400,), device="cuda", generator=gen)


@pytest.mark.parametrize("own, current", [(True, False), (True, True), (False, True)])
def test_operators_in_the_order_of_another_stream(ps, own, current):
    """A context's stream is not the current one: operands still in the making, temporaries freed and their memory filled at once, results
    used at once."""
    torch.cuda.synchronize()
    ctx = ps.Context(0, torch.cuda.Stream() if own else None)
    with torch.cuda.stream(torch.cuda.Stream() if current else torch.cuda.default_stream()):
        plain = ps.Context(0, torch.cuda.current_stream() if current else None)
        sources = [operands(seed) for seed in (31, 32, 33)]
        want = [all_operators(plain, x) for x in sources]
        torch.cuda.synchronize()
        held = [torch.zeros_like(t) for t in sources[0]]
        for turn in range(6):
            torch.cuda._sleep(10_000_000)                           # (a few milliseconds)
            for h, t in zip(held, sources[turn % 3]):
                h.copy_(t)
            got = all_operators(ctx, [h.clone() for h in held])
            seen = [g.clone() for g in got]
            for h in held:
                h.zero_()
            del got
            junk = [torch.full_like(s, 3.0) for s in seen + held]
            for s, w in zip(seen, want[turn % 3]):
                assert torch.equal(s, w)
            del junk
        torch.cuda.current_stream().synchronize()
    ctx.check_status()


def test_operators_of_another_stream_in_a_capture(ps):
    """A capture of the current stream takes in the calls of a context with a stream of its own."""
    ctx = ps.Context(0, torch.cuda.Stream())
    side = torch.cuda.Stream()
    first, second = operands(34), operands(35)
    held = [t.clone() for t in first]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = [all_operators(ctx, x) for x in (first, second)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = all_operators(ctx, held)
        for x, w in ((first, want[0]), (second, want[1]), (first, want[0])):
            for h, t in zip(held, x):
                h.copy_(t)
            for g in got:
                g.fill_(1.0)
            graph.replay()
            for g, t in zip(got, w):
                assert torch.equal(g, t)
        side.synchronize()
    ctx.check_status()
    del graph, got


def test_operators_of_contexts_on_their_own_streams_overlap(ps):
    """Each context's stream is current for its calls, so nothing orders the two: no work space is shared."""
    contexts = [ps.Context(0, torch.cuda.Stream()) for _ in range(2)]
    inputs = [operands(36), operands(37)]
    torch.cuda.synchronize()
    want = []
    for ctx, x in zip(contexts, inputs):
        with torch.cuda.stream(ctx.stream):
            want.append(all_operators(ctx, x))
        torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for _ in range(3):
            got = []
            for ctx, x in zip(contexts, inputs):
                with torch.cuda.stream(ctx.stream):
                    got.append(all_operators(ctx, x))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))
    for ctx in contexts:
        ctx.check_status()
