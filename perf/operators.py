"""The operators of a transformer's training step that the library offers, as cases that can be
timed and compared: dropout whose mask comes out of a counter, the embedding lookup with its
gradient, and attention with the backward pass that recomputes the probabilities.

A case is a dict of plain values.  Its "op" says which operator and direction it takes:

  dropout       y = dropout(x) + residual             (Context.dropout)
  dropout_grad  the same mask on the output's gradient (Context.dropout)
  embed         scaled rows of a table                (Context.embed_forward)
  embed_grad    the table's gradient                  (Context.embed_backward)
  attend        output and log-sum-exp                (Context.attention_forward)
  attend_grad   gradients of queries, keys and values (Context.attention_backward)

Sizes follow the shapes of paper_2601_02311_b200/synth.py: hidden sizes that are multiples of 128, heads of
128, vocabularies of 32000 to 256000, sequences of 2048 to 32768, 1 to 64 sequences a micro-batch.
"""
import functools
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}


def dropout(name, rows, cols, op="dropout", dtype="bf16", p=0.1, first=0, pitch=0):
    return dict(name=name, op=op, rows=rows, cols=cols, dtype=dtype, p=p, first=first, pitch=pitch or cols)


def embed(name, tokens, rows, dim, op="embed", dtype="bf16", wide=False, scale=1.0, absent=0.0):
    return dict(name=name, op=op, tokens=tokens, rows=rows, dim=dim, dtype=dtype, wide=wide, scale=scale, absent=absent)


def attend(name, batch, q_len, heads, dim, op="attend", kv_heads=0, k_len=0, dtype="bf16", causal=True, ragged=0):
    return dict(name=name, op=op, batch=batch, q_len=q_len, k_len=k_len or q_len, heads=heads, kv_heads=kv_heads or heads,
                dim=dim, dtype=dtype, causal=causal, ragged=ragged)


def listed():
    return [
        # after a sublayer of the smallest shape, one short sequence: what a call costs
        dropout("dropout_short", 2048, 768),
        # after a sublayer of a large shape: sixteen sequences of 4096
        dropout("dropout_large", 65536, 8192),
        # the gradient, of a shard whose columns start in the middle of a group of the generator's words
        dropout("dropout_grad_odd", 12301, 5003, op="dropout_grad", dtype="f32", p=0.15, first=1251, pitch=20012),
        # a short sequence's lookup in the smallest table
        embed("embed_short", 2048, 32000, 768, scale=27.7),
        # a large micro-batch in a large table
        embed("embed_large", 131072, 128000, 8192),
        # the gradient of the table for a short sequence: most rows have no token
        embed("embed_grad_short", 2048, 32000, 768, op="embed_grad", scale=27.7),
        # the gradient for a large micro-batch into the largest vocabulary; padding at the end of the sequences
        embed("embed_grad_large", 131072, 256000, 8192, op="embed_grad", absent=0.05),
        # the smallest shape's attention on a short sequence
        attend("attend_short", 1, 384, 6, 128),
        # a long sequence with four query heads to a key head
        attend("attend_long", 1, 8192, 32, 128, kv_heads=8),
        # the smallest shape's backward pass
        attend("attend_grad_short", 1, 384, 6, 128, op="attend_grad"),
        # sequences of different lengths, padded; heads of 64 in 16-bit IEEE floats
        attend("attend_grad_ragged", 6, 2047, 16, 64, op="attend_grad", kv_heads=4, dtype="f16", ragged=7),
        # a long sequence's backward pass
        attend("attend_grad_long", 1, 8192, 32, 128, op="attend_grad", kv_heads=8),
    ]


def between(rng, lo, hi):
    """A whole number, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["dropout", "dropout_grad", "embed", "embed_grad", "embed_grad", "attend", "attend", "attend_grad", "attend_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("dropout"):
        cols = rng.choice([between(rng, 1, 16384), 128 * rng.randint(6, 128)])
        rows = between(rng, 1, min(131072, 500_000_000 // cols))
        shard = rng.random() < 0.4
        case = dropout("", rows, cols, op, dtype, rng.choice([0.0, 0.05, 0.1, 0.5]), rng.randrange(1 << 40) if shard else 0,
                       cols * rng.randint(1, 8) if shard else cols)
    elif op.startswith("embed"):
        dim = rng.choice([between(rng, 1, 16384), 128 * rng.randint(6, 128)])
        rows = between(rng, 1000, min(256000, 1_000_000_000 // dim))
        tokens = between(rng, 1, min(131072, 400_000_000 // dim))
        case = embed("", tokens, rows, dim, op, dtype, op == "embed_grad" and rng.random() < 0.4, rng.choice([1.0, math.sqrt(dim)]),
                     rng.choice([0.0, 0.0, 0.1, 0.6]))
    else:
        dim = rng.choice([128, 128, 128, 64, 64, 32, 80, 96])
        kv_heads, group = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 1, 2, 4, 7])
        batch = rng.choice([1, 1, 2, 3, 8])
        pairs = 1_000_000_000 // (batch * kv_heads * group)
        q_len = rng.choice([between(rng, 1, min(32768, int(math.sqrt(pairs)))), 128 * between(rng, 1, max(1, min(256, int(math.sqrt(pairs)) // 128)))])
        k_len = q_len if rng.random() < 0.7 else between(rng, 1, min(32768, pairs // q_len))
        case = attend("", batch, q_len, kv_heads * group, dim, op, kv_heads, k_len, rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.7,
                      rng.choice([0, 0, rng.randrange(1, 1000)]))
    del case["name"]
    return case


def lengths(case):
    """Queries and keys of each sequence: all of them, or what the padding leaves."""
    if not case["ragged"]:
        return [case["q_len"]] * case["batch"], [case["k_len"]] * case["batch"]
    rng = random.Random(case["ragged"])
    share = [rng.uniform(0.2, 1.0) for _ in range(case["batch"])]
    return [max(1, int(s * case["q_len"])) for s in share], [max(1, int(s * case["k_len"])) for s in share]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, size=1.0):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, size, generator=gen)

    state = dict(case=case)
    if case["op"].startswith("dropout"):
        state["x"] = normal(case["rows"], case["cols"])
        state["residual"] = normal(case["rows"], case["cols"]) if case["op"] == "dropout" else None
        state["seed"], state["stream"] = seed * 0x9E3779B97F4A7C15 % (1 << 64), seed % 977
    elif case["op"].startswith("embed"):
        # words are as frequent as the reciprocal of their rank, and ranks lie anywhere in the table
        u = torch.rand(case["tokens"], device="cuda", dtype=torch.float64, generator=gen)
        rank = torch.exp(u * math.log(case["rows"])).long().clamp_(1, case["rows"]) - 1
        tokens = rank * 982451653 % case["rows"]
        if case["absent"]:
            tokens[torch.rand(case["tokens"], device="cuda", generator=gen) < case["absent"]] = -1
        state["tokens"] = tokens
        if case["op"] == "embed":
            state["table"] = normal(case["rows"], case["dim"], size=0.02)
        else:
            state["d_out"] = normal(case["tokens"], case["dim"], size=0.01)
    else:
        q_lens, k_lens = lengths(case)
        batch, heads, kv_heads, dim = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        state["q"] = normal(batch, case["q_len"], heads, dim)
        state["k"] = normal(batch, case["k_len"], kv_heads, dim)
        state["v"] = normal(batch, case["k_len"], kv_heads, dim)
        state["q_lens"] = state["k_lens"] = None
        if case["ragged"]:
            state["q_lens"], state["k_lens"] = (torch.tensor(n, device="cuda", dtype=torch.int32) for n in (q_lens, k_lens))
        if case["op"] == "attend_grad":
            state["d_out"] = normal(batch, case["q_len"], heads, dim, size=0.01)
            state["out"], state["lse"] = plain_attend(state)
    return state


# ---- the operators in their plain form

def philox(counter, stream, seed):
    """Four 32-bit words of the generator for every block counter: [..., 4], as int64."""
    low = 0xFFFFFFFF
    a, b = counter & low, counter >> 32 & low
    c, d = torch.full_like(a, stream & low), torch.full_like(a, stream >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = (q >> 32 & low) ^ b ^ k0, q & low, (p >> 32 & low) ^ d ^ k1, p & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack((a, b, c, d), -1)


def plain_dropout(s):
    case, x = s["case"], s["x"]
    begin = case["first"] + case["pitch"] * torch.arange(case["rows"], device=x.device)
    blocks = (begin >> 2)[:, None] + torch.arange(case["cols"] // 4 + 2, device=x.device)
    words = philox(blocks, s["stream"], s["seed"]).flatten(1)
    words = words.gather(1, (begin & 3)[:, None] + torch.arange(case["cols"], device=x.device))
    kept = words >= round(case["p"] * 2.0 ** 32)
    y = torch.where(kept, x.float() * (1.0 / (1.0 - case["p"])), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def plain_embed(s):
    held = s["tokens"] >= 0
    rows = s["table"][s["tokens"].clamp(min=0)].float() * s["case"]["scale"]
    return torch.where(held[:, None], rows, 0.0).to(s["table"].dtype)


def plain_embed_grad(s):
    case, held = s["case"], s["tokens"] >= 0
    grad = torch.zeros(case["rows"], case["dim"], device="cuda")
    grad.index_add_(0, s["tokens"].clamp(min=0), torch.where(held[:, None], s["d_out"].float(), 0.0))
    return (grad * case["scale"]).to(torch.float32 if case["wide"] else s["d_out"].dtype)


def plain_scores(s):
    """Scaled scores [batch, kv_heads, group, q, k] in 32 bits, and where a key may be seen."""
    case, q, k = s["case"], s["q"].float(), s["k"].float()
    batch, q_len, heads, dim = q.shape
    k_len, kv_heads = k.shape[1:3]
    q = q.view(batch, q_len, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4)
    scores = q @ k.permute(0, 2, 3, 1)[:, :, None] * dim ** -0.5
    q_lens, k_lens = (torch.full((batch,), n, device=q.device) if lens is None else lens.long()
                      for n, lens in ((q_len, s["q_lens"]), (k_len, s["k_lens"])))
    i, j = torch.arange(q_len, device=q.device), torch.arange(k_len, device=q.device)
    seen = (i < q_lens[:, None])[:, :, None] & (j < k_lens[:, None])[:, None, :]
    if case["causal"]:
        seen = seen & (j <= i[:, None] + (k_lens - q_lens)[:, None, None])
    return scores.masked_fill_(~seen[:, None, None], -math.inf)


def by_head(x, kv_heads):
    """[batch, len, heads, dim] as [batch, kv_heads, group, len, dim] in 32 bits."""
    batch, length, heads, dim = x.shape
    return x.float().view(batch, length, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4)


def by_token(x, dtype):
    batch, kv_heads, group, length, dim = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(batch, length, kv_heads * group, dim).to(dtype)


def plain_attend(s):
    kv_heads, scores = s["k"].shape[2], plain_scores(s)
    most = scores.amax(-1, keepdim=True).clamp_(min=-1e30)
    weights = torch.exp(scores.sub_(most))
    total = weights.sum(-1, keepdim=True)
    out = weights @ by_head(s["v"], kv_heads) / total.masked_fill(total == 0, 1.0)
    lse = (most + torch.log(total)).squeeze(-1)
    return by_token(out, s["q"].dtype), lse.flatten(1, 2)


def plain_attend_grad(s):
    kv_heads, dtype = s["k"].shape[2], s["q"].dtype
    scale = s["q"].shape[3] ** -0.5
    lse = s["lse"].view(s["lse"].shape[0], kv_heads, -1, s["lse"].shape[2], 1)
    weights = torch.exp(plain_scores(s).sub_(lse.masked_fill(lse == -math.inf, 0.0)))
    d_out = by_head(s["d_out"], kv_heads)
    d_v = (weights.transpose(-1, -2) @ d_out).sum(2, keepdim=True)
    d_weights = d_out @ by_head(s["v"], kv_heads).transpose(-1, -2)
    delta = (weights * d_weights).sum(-1, keepdim=True)
    d_scores = weights.mul_(d_weights.sub_(delta)).mul_(scale)
    d_q = d_scores @ by_head(s["k"], kv_heads)
    d_k = (d_scores.transpose(-1, -2) @ by_head(s["q"], kv_heads)).sum(2, keepdim=True)
    return {"d_q": by_token(d_q, dtype), "d_k": by_token(d_k, dtype), "d_v": by_token(d_v, dtype)}


PLAIN = dict(dropout=plain_dropout, dropout_grad=plain_dropout, embed=plain_embed, embed_grad=plain_embed_grad,
             attend=plain_attend, attend_grad=plain_attend_grad)


# ---- the library's calls

@functools.lru_cache(maxsize=None)
def context(device, stream):
    from paper_2601_02311_b200 import ps
    return ps.Context(device, torch.cuda.ExternalStream(stream, device) if stream else None)


def run(state):
    case = state["case"]
    if not own:
        return PLAIN[case["op"]](state)
    device = torch.cuda.current_device()
    ctx = context(device, torch.cuda.current_stream().cuda_stream)
    if case["op"].startswith("dropout"):
        return ctx.dropout(state["x"], case["p"], state["seed"], stream=state["stream"], residual=state["residual"],
                           first=case["first"], pitch=case["pitch"])
    if case["op"] == "embed":
        return ctx.embed_forward(state["table"], state["tokens"], scale=case["scale"])
    if case["op"] == "embed_grad":
        return ctx.embed_backward(state["d_out"], state["tokens"], case["rows"], scale=case["scale"],
                                  dtype=torch.float32 if case["wide"] else None)
    if case["op"] == "attend":
        return ctx.attention_forward(state["q"], state["k"], state["v"], causal=case["causal"], q_lens=state["q_lens"],
                                     k_lens=state["k_lens"])
    d_q, d_k, d_v = ctx.attention_backward(state["q"], state["k"], state["v"], state["out"], state["lse"], state["d_out"],
                                           causal=case["causal"], q_lens=state["q_lens"], k_lens=state["k_lens"])
    return {"d_q": d_q, "d_k": d_k, "d_v": d_v}


# ---- what a pass cannot do without

def work(case):
    w = WIDTH[case["dtype"]]
    if case["op"].startswith("dropout"):
        n = case["rows"] * case["cols"]
        arrays = 3 if case["op"] == "dropout" else 2
        return {"bytes": arrays * n * w, "flops": arrays * n}
    if case["op"].startswith("embed"):
        held = case["tokens"] * (1.0 - case["absent"])
        # a lookup reads each row that occurs once: of rows as frequent as 1 / rank, so many occur
        rate = held / math.log(case["rows"])
        occurring = rate * math.log1p(case["rows"] / max(rate, 1.0)) + min(rate, case["rows"])
        occurring = min(occurring, held, case["rows"])
        if case["op"] == "embed":
            return {"bytes": int(8 * case["tokens"] + (case["tokens"] + occurring) * case["dim"] * w), "flops": int(held * case["dim"])}
        return {"bytes": int(8 * case["tokens"] + held * case["dim"] * w + case["rows"] * case["dim"] * (4 if case["wide"] else w)),
                "flops": int(held * case["dim"])}
    pairs = 0
    for n, m in zip(*lengths(case)):
        if not case["causal"]:
            pairs += n * m
        elif n <= m:
            pairs += n * m - n * (n - 1) // 2
        else:
            pairs += m * (m + 1) // 2
    q, k = case["batch"] * case["q_len"] * case["heads"], case["batch"] * case["k_len"] * case["kv_heads"]
    d, grad = case["dim"], case["op"] == "attend_grad"
    arrays = (4 * q + 4 * k if grad else 2 * q + 2 * k) * d * w + 4 * q
    return {"bytes": arrays, "flops": (10 if grad else 4) * d * pairs * case["heads"]}


# ---- the definitions in 64 bits

def exact_words(case, seed, rows):
    """The generator's word of every element of some rows, out of products of 16-bit halves."""
    g = case["first"] + rows[:, None] * case["pitch"] + torch.arange(case["cols"], device="cuda")
    block, mask = torch.div(g, 4, rounding_mode="floor"), (1 << 32) - 1

    def product(x, m):
        lo, hi = x % 65536 * m, torch.div(x, 65536, rounding_mode="floor") * m
        low = (lo + hi % 65536 * 65536) % (1 << 32)
        return torch.div(lo + hi % 65536 * 65536, 1 << 32, rounding_mode="floor") + torch.div(hi, 65536, rounding_mode="floor"), low

    key, stream = seed * 0x9E3779B97F4A7C15 % (1 << 64), seed % 977
    x = [block % (1 << 32), torch.div(block, 1 << 32, rounding_mode="floor"), torch.full_like(block, stream), torch.zeros_like(block)]
    for n in range(10):
        k0, k1 = (key % (1 << 32) + n * 0x9E3779B9) & mask, (key // (1 << 32) + n * 0xBB67AE85) & mask
        (h0, l0), (h1, l1) = product(x[0], 0xD2511F53), product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
    which = g % 4
    return torch.where(which < 2, torch.where(which == 0, x[0], x[1]), torch.where(which == 2, x[2], x[3]))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("dropout"):
        y = torch.empty(case["rows"], case["cols"], device="cuda", dtype=torch.float64)
        step = max(1, 30_000_000 // case["cols"])
        for at in range(0, case["rows"], step):
            rows = torch.arange(at, min(at + step, case["rows"]), device="cuda")
            part = s["x"][rows].double() / (1.0 - case["p"])
            part[exact_words(case, seed, rows) < round(case["p"] * 2.0 ** 32)] = 0.0
            y[rows] = part if s["residual"] is None else part + s["residual"][rows].double()
        return y
    if case["op"] == "embed":
        y = torch.zeros(case["tokens"], case["dim"], device="cuda", dtype=torch.float64)
        at = torch.nonzero(s["tokens"] >= 0).flatten()
        y[at] = s["table"][s["tokens"][at]].double() * case["scale"]
        return y
    if case["op"] == "embed_grad":
        grad = torch.zeros(case["rows"], case["dim"], device="cuda", dtype=torch.float64)
        at = torch.nonzero(s["tokens"] >= 0).flatten()
        grad.index_put_((s["tokens"][at],), s["d_out"][at].double() * case["scale"], accumulate=True)
        return grad
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    q, k, v = (s[n].double() for n in "qkv")
    out, lse = torch.zeros_like(q), torch.full((case["batch"], case["heads"], case["q_len"]), -math.inf, device="cuda", dtype=torch.float64)
    d_q, d_k, d_v = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b, (n, m) in enumerate(zip(*lengths(case))):
        for h in range(case["heads"]):
            kh = h // group
            scores = torch.einsum("id,jd->ij", q[b, :n, h], k[b, :m, kh]) * scale
            if case["causal"]:
                scores += torch.full_like(scores, -math.inf).triu_(m - n + 1)
            begin = max(0, n - m) if case["causal"] else 0  # rows before it see nothing
            scores = scores[begin:]
            lse[b, h, begin:n] = torch.logsumexp(scores, 1)
            weights = torch.softmax(scores, 1)
            if case["op"] == "attend":
                out[b, begin:n, h] = torch.einsum("ij,jd->id", weights, v[b, :m, kh])
                continue
            d_out = s["d_out"][b, begin:n, h].double()
            d_v[b, :m, kh] += torch.einsum("ij,id->jd", weights, d_out)
            d_weights = torch.einsum("id,jd->ij", d_out, v[b, :m, kh])
            d_scores = weights * (d_weights - torch.einsum("ij,ij->i", weights, d_weights)[:, None]) * scale
            d_q[b, begin:n, h] = torch.einsum("ij,jd->id", d_scores, k[b, :m, kh])
            d_k[b, :m, kh] += torch.einsum("ij,id->jd", d_scores, q[b, begin:n, h])
    return (out, lse) if case["op"] == "attend" else {"d_q": d_q, "d_k": d_k, "d_v": d_v}
