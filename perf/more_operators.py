"""Cases of the operators around a vocabulary-parallel model's two ends, through the
package's public entry points.

One step of speculative decoding and of training such a model passes through

* ``quantise``: a matrix in blocks of 32 values with a shared power of two and 4-bit
  floating-point elements, and the values those stand for (``MX4Matrix.quantise``);
* ``product``: hidden states quantised that way times a rank's shard of such weights,
  stored into every slot of the heap with arrival counters (``GatheredOutput.run_mx4``);
* ``verify``: drafted tokens accepted or replaced by the target's probabilities, from
  given random numbers (``DraftVerification``);
* ``embed``: a rank's share of the lookup of tokens in a vocabulary-parallel table, scaled
  and stored into every slot (``GatheredRows``);
* ``embed_grad``: the gradient of the rank's shard of the table (``EmbeddingGrad``).

The layer sizes are this repository's own workloads (8192 x 3584 on 8 ranks, 28672 columns
gathered; 4096 x 1024 on 8 ranks); the other sizes are generic: odd vocabularies whose rows
start at any alignment, masked columns at -inf, drafts of different lengths.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _quantise(rows, K, dtype, name=None):
    c = {"kind": "quantise", "rows": rows, "K": K, "dtype": dtype}
    return c if name is None else dict(c, name=name)


def _product(M, K, N, world, rank, dtype, name=None):
    c = {"kind": "product", "M": M, "K": K, "N": N, "world": world, "rank": rank, "dtype": dtype}
    return c if name is None else dict(c, name=name)


def _verify(sequences, drafted, vocab, dtype, mode="draft", scale=1.0, pad=0, masked=0, name=None):
    """``mode``: "draft" (the drafting model's logits are there), "tokens" (tokens alone, as
    from a lookup in the text so far) or "greedy".  ``pad``: columns between a row's end and
    the next row; ``masked``: columns at the end of the vocabulary that are -inf."""
    c = {"kind": "verify", "sequences": sequences, "drafted": drafted, "vocab": vocab,
         "dtype": dtype, "mode": mode, "scale": scale, "pad": pad, "masked": masked}
    return c if name is None else dict(c, name=name)


def _embed(tokens, D, vocab, world, rank, dtype, scale=1.0, name=None):
    """``vocab``: rows of the rank's shard."""
    c = {"kind": "embed", "tokens": tokens, "D": D, "vocab": vocab, "world": world, "rank": rank,
         "dtype": dtype, "scale": scale}
    return c if name is None else dict(c, name=name)


def _embed_grad(tokens, D, vocab, world, rank, dtype, table="f32", scale=1.0, accumulate=False,
                name=None):
    """``table``: type of the table's gradient; ``accumulate``: added to what it holds (that
    of an output head that shares the table)."""
    c = {"kind": "embed_grad", "tokens": tokens, "D": D, "vocab": vocab, "world": world,
         "rank": rank, "dtype": dtype, "table": table, "scale": scale, "accumulate": accumulate}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the hidden states of a decode batch
        _quantise(64, 8192, "bf16", name="quantise_64rows"),
        # the weights of the whole head, from 32 bits
        _quantise(28672, 8192, "f32", name="quantise_weights"),
        # a single token through the large layer's shard
        _product(1, 8192, 3584, 8, 3, "bf16", name="product_1token_large"),
        # what a decode batch of drafts puts through the large layer's shard
        _product(64, 8192, 3584, 8, 0, "bf16", name="product_64tokens_large"),
        # prompts: the large layer's shard, gathered on 8 ranks
        _product(4096, 8192, 3584, 8, 5, "bf16", name="product_4096tokens_large"),
        # prompts or a training step through the whole head on one rank
        _product(4096, 8192, 28672, 1, 0, "f16", name="product_4096tokens_whole"),
        # one sequence with 4 drafted tokens: latency
        _verify(1, 4, 28672, "bf16", name="verify_1sequence"),
        # a decode batch over an odd vocabulary, rows at any alignment, tokens masked
        _verify(64, 5, 50001, "f16", scale=1.25, pad=3, masked=2000, name="verify_64sequences"),
        # the accepted tokens of a decode batch
        _embed(64, 8192, 3584, 8, 2, "bf16", scale=1.5, name="embed_64tokens"),
        # a batch of prompts
        _embed(8192, 8192, 3584, 8, 0, "bf16", name="embed_8192tokens"),
        # a small training step: every row of the shard's gradient is written
        _embed_grad(2048, 4096, 1024, 8, 1, "bf16", scale=2.0, name="embed_grad_2048tokens"),
        # a batch of long sequences, added to the output head's gradient
        _embed_grad(32768, 4096, 28672, 1, 0, "bf16", accumulate=True,
                    name="embed_grad_32768tokens"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.random()
    dtype = rng.choice(("bf16", "bf16", "f16"))
    world = rng.choice((1, 2, 4, 8, 8))
    if what < 0.15:
        K = 32 * _log_int(rng, 1, 256)
        return _quantise(_log_int(rng, 1, 28672), K, rng.choice(("bf16", "f16", "f32")))
    if what < 0.45:
        M = rng.choice((1, 2, 5, 16, 37, 64, _log_int(rng, 65, 4096), _log_int(rng, 65, 4096)))
        K = 32 * _log_int(rng, 8, 256)
        N = 8 * _log_int(rng, 16, 1024)
        return _product(M, K, N, world, rng.randrange(world), dtype)
    if what < 0.7:
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        sequences, drafted = _log_int(rng, 1, 64), rng.choice((0, 1, 2, 3, 4, 5, 7, 8))
        vocab = _log_int(rng, 1000, 131072)
        if rng.random() < 0.5:
            vocab = min(vocab // 128 * 128 + 128, 131072)
        while sequences * (2 * drafted + 1) * vocab * DTYPES[dtype].itemsize > 64 * 11 * 50001 * 2:
            sequences = max(1, sequences // 2)
            vocab = vocab if sequences > 1 else vocab // 2
        return _verify(sequences, drafted, vocab, dtype, rng.choice(("draft", "draft", "tokens", "greedy")),
                       rng.choice((1.0, 1.0, 0.7, 1.25)), rng.choice((0, 0, 1, 8, 64)),
                       rng.choice((0, 0, vocab // 50, vocab // 3)))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    D = 8 * _log_int(rng, 16, 1024)
    if what < 0.85:
        return _embed(_log_int(rng, 1, 4096), D, _log_int(rng, 100, 32000), world,
                      rng.randrange(world), dtype, rng.choice((1.0, 1.0, 0.5, math.sqrt(D))))
    D = min(D, 4096)
    return _embed_grad(_log_int(rng, 1, 32768), D, _log_int(rng, 100, 28672), world,
                       rng.randrange(world), dtype, rng.choice(("f32", "f32", dtype)),
                       rng.choice((1.0, 1.0, 0.5, math.sqrt(D))), rng.random() < 0.5)


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _values(rows, K, gen, dtype):
    """Rows of spread like hidden states', a few channels many times the others."""
    x = torch.randn((rows, K), generator=gen, device="cuda")
    x *= torch.rand((K,), generator=gen, device="cuda").pow_(-0.25)
    return x.to(dtype)


def _product_inputs(case, seed):
    gen = _generator(seed)
    M, K, N = case["M"], case["K"], case["N"]
    X = _values(M, K, gen, DTYPES[case["dtype"]])
    q = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    # weights of a spread of about 1 / sqrt(K)
    around = 127 - int(round(math.log2(2.9 * math.sqrt(K))))
    scales = torch.randint(around - 1, around + 2, (N, K // 32), generator=gen, device="cuda",
                           dtype=torch.uint8)
    return X, q, scales


def _logits(rows, vocab, pad, masked, gen, dtype):
    """Spread like a head's logits, in half the rows one token far ahead; the masked columns
    -inf.  In 32 bits, and as a [rows, vocab] view of rows that are vocab + pad apart."""
    x = torch.randn((rows, vocab + pad), generator=gen, device="cuda").mul_(2.5)
    ahead = torch.randint(0, vocab - masked, (rows,), generator=gen, device="cuda")
    lift = torch.rand((rows,), generator=gen, device="cuda").sub_(0.5).clamp_(min=0).mul_(28.0)
    x[torch.arange(rows, device="cuda"), ahead] += lift
    x[:, vocab - masked:vocab] = -math.inf
    return x, x.to(dtype)[:, :vocab]


def _verify_inputs(case, seed):
    gen = _generator(seed)
    B, k, vocab, pad = case["sequences"], case["drafted"], case["vocab"], case["pad"]
    dt = DTYPES[case["dtype"]]
    x, logits = _logits(B * (k + 1), vocab, pad, case["masked"], gen, dt)
    # the drafting model is near the target, and the drafted tokens are drawn from it
    near = x.view(B, k + 1, vocab + pad)[:, :k].reshape(B * k, vocab + pad)
    near = torch.randn(near.shape, generator=gen, device="cuda").mul_(0.5).add_(near)
    draft = near.to(dt)[:, :vocab]
    race = torch.rand((B * k, vocab), generator=gen, device="cuda").clamp_(min=1e-7)
    race = race.log_().neg_().log_().neg_()
    if case["mode"] == "greedy":
        race *= 0.3
    ids = (draft.float() * case["scale"] + race).argmax(1).view(B, k) if k else \
        torch.empty((B, 0), dtype=torch.int64, device="cuda")
    # drafts that end early, and sequences without one
    length = torch.randint(0, 3 * k + 1, (B, 1), generator=gen, device="cuda")
    if B == 1:
        length.fill_(k)
    ids = torch.where(torch.arange(k, device="cuda") < length, ids, -1)
    uniforms = torch.rand((B, k), generator=gen, device="cuda")
    noise = torch.rand((B, vocab), generator=gen, device="cuda")
    noise = torch.log1p(noise.neg_()).neg_().clamp_(min=1e-20)
    return logits, ids, uniforms, noise, draft


def _tokens(case, gen):
    """Every world-th token is the shard's, in an order of chance; frequent and rare ones (the
    k-th token's share is about 1 / k), and a few positions of padding."""
    T, vocab, world, rank = case["tokens"], case["vocab"], case["world"], case["rank"]
    u = torch.rand((T,), generator=gen, device="cuda", dtype=torch.float64)
    kth = ((u * math.log(vocab + 1)).exp() - 1).to(torch.int64).clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device="cuda")[kth]
    shard = torch.randperm(T, generator=gen, device="cuda") + rank
    ids = ids + shard % world * vocab
    padding = torch.rand((T,), generator=gen, device="cuda") < 0.02
    return torch.where(padding, -1, ids) if T > 64 else ids


def _embed_inputs(case, seed):
    gen = _generator(seed)
    table = torch.randn((case["vocab"], case["D"]), generator=gen, device="cuda")
    return _tokens(case, gen), table.mul_(0.05).to(DTYPES[case["dtype"]])


def _embed_grad_inputs(case, seed):
    gen = _generator(seed)
    tokens = _tokens(case, gen)
    drows = torch.randn((case["tokens"], case["D"]), generator=gen, device="cuda")
    held = torch.zeros((0,), device="cuda")
    if case["accumulate"]:
        held = torch.randn((case["vocab"], case["D"]), generator=gen, device="cuda")
    return tokens, drows.to(DTYPES[case["dtype"]]), held.to(DTYPES[case["table"]])


def prepare(case, seed):
    s = {"case": case}
    kind = case["kind"]
    if kind == "quantise":
        s["x"] = _values(case["rows"], case["K"], _generator(seed), DTYPES[case["dtype"]])
    elif kind == "product":
        s["X"], s["q"], s["scales"] = _product_inputs(case, seed)
    elif kind == "verify":
        s["logits"], s["ids"], s["uniforms"], s["noise"], s["draft"] = _verify_inputs(case, seed)
    elif kind == "embed":
        s["tokens"], s["table"] = _embed_inputs(case, seed)
    else:
        s["tokens"], s["drows"], held = _embed_grad_inputs(case, seed)
        s["dtable"] = held if case["accumulate"] else \
            torch.empty((case["vocab"], case["D"]), dtype=held.dtype, device="cuda")
    _keep_own(s, case) if own else _keep_plain(s, case)
    return s


def _keep_own(s, case):
    import paper_2511_12500_amd as sym
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "quantise":
        s["to"] = sym.MX4Matrix.empty(case["rows"], case["K"])
        s["values"] = torch.empty_like(s["x"])
    elif kind == "product":
        M, N, w, r = case["M"], case["N"], case["world"], case["rank"]
        tiles = -(-M // sym.MX4_TILE_M) * -(-N // sym.MX4_TILE_N)
        heap = sym.Heap(w, M * w * N * 2 + w * tiles * 4 + 4096)
        out = sym.GatheredOutput(heap, M, N, dt, sym.MX4_TILE_M, sym.MX4_TILE_N)
        s["out"], s["block"] = out, out.C_all()[:, :, r * N:(r + 1) * N]
        s["X4"] = sym.MX4Matrix.empty(M, case["K"])
        s["weight"] = sym.MX4Matrix(s["q"], s["scales"])
    elif kind == "verify":
        s["op"] = sym.DraftVerification(case["sequences"], case["drafted"], case["vocab"], dt,
                                        scale=case["scale"], draft_scale=case["scale"])
    elif kind == "embed":
        T, D, w = case["tokens"], case["D"], case["world"]
        heap = sym.Heap(w, T * D * dt.itemsize + w * T * 4 + w * D * 4 + (1 << 16))
        s["out"] = sym.GatheredRows(heap, T, D, dt)
        s["rows"] = s["out"].rows_all()
    else:
        s["op"] = sym.EmbeddingGrad(case["tokens"], case["D"], dt)


def _keep_plain(s, case):
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "product":
        M, N, w, r = case["M"], case["N"], case["world"], case["rank"]
        C = torch.zeros((w, M, w * N), dtype=dt, device="cuda")
        s["block"] = C[:, :, r * N:(r + 1) * N]
    elif case["kind"] == "embed":
        s["rows"] = torch.zeros((case["world"], case["tokens"], case["D"]), dtype=dt,
                                device="cuda")


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"quantise": _own_quantise, "product": _own_product, "verify": _own_verify,
                "embed": _own_embed, "embed_grad": _own_embed_grad}[kind](state)
    return {"quantise": _plain_quantise, "product": _plain_product, "verify": _plain_verify,
            "embed": _plain_embed, "embed_grad": _plain_embed_grad}[kind](state)


def _own_quantise(s):
    s["to"].quantise(s["x"], values=s["values"])
    return {"values": s["values"]}


def _own_product(s):
    s["X4"].quantise(s["X"])
    s["out"].run_mx4(s["X4"], s["weight"], s["case"]["rank"])
    return {"block": s["block"]}


def _own_verify(s):
    op, mode = s["op"], s["case"]["mode"]
    if mode == "greedy":
        op.run(s["logits"], s["ids"])
    else:
        op.run(s["logits"], s["ids"], s["uniforms"], s["noise"],
               s["draft"] if mode == "draft" else None)
    return {"tokens": op.tokens, "accepted": op.accepted, "logprob": op.logprob}


def _own_embed(s):
    s["out"].run(s["tokens"], s["table"], s["case"]["rank"], scale=s["case"]["scale"])
    return {"rows": s["rows"]}


def _own_embed_grad(s):
    case = s["case"]
    s["op"].run(s["tokens"], s["drows"], s["dtable"], first=case["rank"] * case["vocab"],
                scale=case["scale"], accumulate=case["accumulate"])
    return {"dtable": s["dtable"]}


def _in_blocks(x):
    """The values that x, in blocks of 32 with a shared power of two, stands for in 4 bits."""
    b = x.float().view(x.shape[0], -1, 32)
    _, e = torch.frexp(b.abs().amax(2, keepdim=True))
    e = (e - 3).clamp(min=-127)
    v = torch.ldexp(b, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = ((a / step).round() * step).clamp(max=6.0)
    return torch.ldexp(torch.copysign(a, v), e).view(x.shape)


def _plain_quantise(s):
    return {"values": _in_blocks(s["x"]).to(s["x"].dtype)}


def _plain_product(s):
    q, scales = s["q"], s["scales"]
    code = torch.stack((q & 15, q >> 4), dim=2).view(q.shape[0], s["case"]["K"]).long()
    steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device)
    w = torch.cat((steps, -steps))[code]
    w = torch.ldexp(w.view(q.shape[0], -1, 32), scales.int()[:, :, None] - 127).view(w.shape)
    y = _in_blocks(s["X"]) @ w.t()
    s["block"].copy_(y.to(s["X"].dtype).expand_as(s["block"]))
    return {"block": s["block"]}


def _plain_verify(s):
    """In 64 bits: an accepted token and a drawn one lie next to a border."""
    case, ids, u = s["case"], s["ids"], s["uniforms"]
    B, k, V = case["sequences"], case["drafted"], case["vocab"]
    greedy, at = case["mode"] == "greedy", ids.clamp(min=0)
    z = s["logits"].double().reshape(B, k + 1, V) * case["scale"]
    z = z - z.amax(2, keepdim=True)
    logp = z - z.exp().sum(2, keepdim=True).log()
    p = logp.exp()
    every = torch.arange(V, device=ids.device)
    if greedy:
        best = torch.where(z == 0, every, V).amin(2)
        good = ids == best[:, :k]
    else:
        if case["mode"] == "draft":
            y = s["draft"].double().reshape(B, k, V) * case["scale"]
            y = (y - y.amax(2, keepdim=True)).exp() if k else y
            q = y / y.sum(2, keepdim=True)
        else:
            q = (every == ids[:, :, None]).double()
        p_of = p[:, :k].gather(2, at[:, :, None])[:, :, 0]
        q_of = q.gather(2, at[:, :, None])[:, :, 0]
        good = (ids >= 0) & (u.double() * q_of < p_of)
    accepted = good.long().cumprod(1).sum(1)
    row = torch.arange(B, device=ids.device)
    drafted = (ids >= 0).long().cumprod(1).sum(1)
    p_a = p[row, accepted]
    if greedy:
        last = best[row, accepted]
    else:
        w = p_a
        if k:
            q_a = q[row, accepted.clamp(max=k - 1)]
            w = torch.where((accepted < drafted)[:, None], (p_a - q_a).clamp(min=0), p_a)
            w = torch.where((w > 0).any(1)[:, None], w, p_a)
        score = w / s["noise"].double()
        last = torch.where(score == score.amax(1, keepdim=True), every, V).amin(1)
    place = torch.arange(k + 1, device=ids.device)
    tokens = torch.cat((at, at.new_zeros(B, 1)), 1)
    tokens = torch.where(place == accepted[:, None], last[:, None], tokens)
    logprob = logp.gather(2, tokens[:, :, None])[:, :, 0]
    used = place <= accepted[:, None]
    return {"tokens": torch.where(used, tokens, -1), "accepted": accepted,
            "logprob": torch.where(used, logprob, 0.0).float()}


def _plain_embed(s):
    case, tokens = s["case"], s["tokens"]
    first = case["rank"] * case["vocab"]
    at = ((tokens >= first) & (tokens < first + case["vocab"])).nonzero()[:, 0]
    got = s["table"][tokens[at] - first].float() * case["scale"]
    s["rows"][:, at] = got.to(s["table"].dtype)
    if case["rank"] == 0:
        s["rows"][:, (tokens < 0).nonzero()[:, 0]] = 0.0
    return {"rows": s["rows"]}


def _plain_embed_grad(s):
    case, tokens, dtable = s["case"], s["tokens"], s["dtable"]
    first = case["rank"] * case["vocab"]
    at = ((tokens >= first) & (tokens < first + case["vocab"])).nonzero()[:, 0]
    got = torch.zeros(dtable.shape, device=dtable.device)
    got.index_add_(0, tokens[at] - first, s["drows"][at].float())
    got *= case["scale"]
    dtable.copy_((got + dtable.float() if case["accumulate"] else got).to(dtable.dtype))
    return {"dtable": dtable}


def exact(case, seed):
    kind = case["kind"]
    if kind == "quantise":
        x = _values(case["rows"], case["K"], _generator(seed), DTYPES[case["dtype"]])
        return {"values": torch.cat([_exact_blocks(x[i:i + 4096])
                                     for i in range(0, case["rows"], 4096)])}
    if kind == "product":
        return _exact_product(case, seed)
    if kind == "verify":
        return _exact_verify(case, seed)
    if kind == "embed":
        return _exact_embed(case, seed)
    return _exact_embed_grad(case, seed)


def _exact_blocks(x):
    """The nearest of the 15 values, of two as near the one whose last bit is 0, to each
    element over its block's power of two: two below the one that the largest begins with."""
    d = x.double().reshape(x.shape[0], -1, 32)
    top = d.abs().max(dim=2).values.clamp(min=2.0 ** -149)
    unit = torch.exp2(torch.floor(torch.log2(top)) - 2.0).clamp(min=2.0 ** -127)[:, :, None]
    a = d.abs() / unit
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    r = torch.zeros_like(a)
    for j in range(1, 8):
        border = (grid[j - 1] + grid[j]) / 2
        r = torch.where(a >= border if j % 2 == 0 else a > border, grid[j], r)
    return (r * d.sign() * unit).reshape(x.shape)


def _exact_product(case, seed):
    X, q, scales = _product_inputs(case, seed)
    x = _exact_blocks(X)
    N, K = case["N"], case["K"]
    y = torch.empty((case["M"], N), dtype=torch.float64, device="cuda")
    for n in range(0, N, 4096):
        code = torch.empty((q[n:n + 4096].shape[0], K), dtype=torch.int64, device="cuda")
        code[:, 0::2] = q[n:n + 4096] % 16
        code[:, 1::2] = q[n:n + 4096] // 16
        # sign, two bits of exponent, one of fraction; no exponent: halves
        e, f = code // 2 % 4, (code % 2).double()
        w = torch.where(e == 0, f * 0.5, (1.0 + 0.5 * f) * torch.exp2(e - 1.0))
        w = torch.where(code >= 8, -w, w).view(-1, K // 32, 32)
        w = (w * torch.exp2(scales[n:n + 4096].double() - 127.0)[:, :, None]).view(-1, K)
        y[:, n:n + 4096] = x @ w.t()
    return {"block": y.expand(case["world"], -1, -1)}


def _exact_verify(case, seed):
    """log p of the accepted tokens and of the drawn one, a sequence at a time."""
    logits, ids, uniforms, noise, draft = _verify_inputs(case, seed)
    k = case["drafted"]
    got = torch.zeros((case["sequences"], k + 1), dtype=torch.float64, device="cuda")
    for b in range(case["sequences"]):
        rows = logits[b * (k + 1):(b + 1) * (k + 1)].double() * case["scale"]
        lp = torch.log_softmax(rows, dim=1)
        i = 0
        while i < k and int(ids[b, i]) >= 0:
            d = int(ids[b, i])
            if case["mode"] == "greedy":
                if d != int((rows[i] == rows[i].max()).nonzero()[0, 0]):
                    break
            else:
                q_d = 1.0
                if case["mode"] == "draft":
                    q = torch.softmax(draft[b * k + i].double() * case["scale"], dim=0)
                    q_d = float(q[d])
                if not float(uniforms[b, i]) * q_d < math.exp(float(lp[i, d])):
                    break
            got[b, i] = lp[i, d]
            i += 1
        if case["mode"] == "greedy":
            got[b, i] = lp[i].max()
            continue
        w = lp[i].exp()
        if i < k and int(ids[b, i]) >= 0:
            less = torch.zeros_like(w)
            less[int(ids[b, i])] = 1.0
            less = torch.relu(w - (q if case["mode"] == "draft" else less))
            w = less if float(less.max()) > 0 else w
        got[b, i] = lp[i, int((w / noise[b].double()).argmax())]
    return {"tokens": None, "accepted": None, "logprob": got}


def _exact_embed(case, seed):
    tokens, table = _embed_inputs(case, seed)
    local = tokens - case["rank"] * case["vocab"]
    mine = (local >= 0) & (local < case["vocab"]) & (tokens >= 0)
    rows = torch.zeros((case["tokens"], case["D"]), dtype=torch.float64, device="cuda")
    rows[mine] = table.double()[local[mine]] * case["scale"]
    return {"rows": rows.expand(case["world"], -1, -1)}


def _exact_embed_grad(case, seed):
    tokens, drows, held = _embed_grad_inputs(case, seed)
    local = tokens - case["rank"] * case["vocab"]
    mine = ((local >= 0) & (local < case["vocab"]) & (tokens >= 0)).nonzero()[:, 0]
    got = torch.zeros((case["vocab"], case["D"]), dtype=torch.float64, device="cuda")
    got = got.index_put_((local[mine],), drows[mine].double() * case["scale"], accumulate=True)
    return {"dtable": got + held.double() if case["accumulate"] else got}


def _distinct(n, vocab):
    """How many different tokens n draws of _tokens hold on average."""
    j = torch.arange(1, vocab + 1, dtype=torch.float64)
    share = torch.log1p(1.0 / j) / math.log(vocab + 1)
    return float((1.0 - (1.0 - share).pow(n)).sum())


def work(case):
    kind, esize = case["kind"], DTYPES[case["dtype"]].itemsize
    if kind == "quantise":
        n = case["rows"] * case["K"]
        return {"bytes": n * (2 * esize + 17 / 32), "flops": 4 * n}
    if kind == "product":
        M, K, N, w = case["M"], case["K"], case["N"], case["world"]
        return {"bytes": 2 * M * K + N * K * 17 / 32 + 2 * w * M * N, "flops": 2 * M * K * N}
    if kind == "verify":
        B, k, V = case["sequences"], case["drafted"], case["vocab"]
        rows = B * (k + 1) + (B * k if case["mode"] == "draft" else 0)
        race = 0 if case["mode"] == "greedy" else B * V * 4
        return {"bytes": rows * V * esize + race + B * (k + 1) * 24,
                "flops": rows * V * 4 + race}
    T, D, w = case["tokens"], case["D"], case["world"]
    mine = -(-T // w)
    if kind == "embed":
        return {"bytes": 8 * T + mine * D * esize * (1 + w), "flops": mine * D}
    out = DTYPES[case["table"]].itemsize * D
    rows = 2 * _distinct(mine, case["vocab"]) if case["accumulate"] else case["vocab"]
    return {"bytes": 8 * T + mine * D * esize + rows * out, "flops": mine * D}
