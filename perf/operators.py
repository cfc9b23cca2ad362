"""Cases of the output head's operators, through the package's public entry points.

A vocabulary-parallel head is a column-parallel layer: every rank's product with
its shard of the vocabulary is stored into its column block of the gathered
logits in every slot.  What runs around it:

* ``w4``: the product of a few tokens with a rank's shard of 4-bit weights
  (group scales), stored into every slot with arrival counters
  (``GatheredOutput.run_w4``);
* ``logprobs``: log probabilities of given tokens, entropies and the top
  alternatives of rows of logits, and the gradient (``TokenLogprobs``);
* ``distill``: the loss against a teacher's top entries and its gradient
  (``TopDistillation``).

The layer sizes are this repository's own workloads (8192 x 3584 on 8 ranks,
28672 columns gathered; 4096 x 1024 on 8 ranks, 8192 gathered); the other
vocabularies are generic: a power of two, odd ones whose rows start at any
alignment, and 2000 columns of padding or of masked tokens at -inf.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _logprobs(rows, vocab, dtype, top=0, scale=1.0, pad=0, masked=0, grad="none", name=None):
    """``pad``: columns between a row's end and the next row; ``masked``: columns at the end
    of the vocabulary that are -inf.  ``grad``: "step" (the weights of the loss are known
    before the call, as in cross entropy: values and gradient from one call) or "after" (they
    follow from the values, as in a policy update: a call for each)."""
    c = {"kind": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top,
         "scale": scale, "pad": pad, "masked": masked, "grad": grad}
    return c if name is None else dict(c, name=name)


def _distill(rows, vocab, k, dtype, values="f32", scale=1.0, rest=False, pad=0, masked=0,
             train=True, name=None):
    """``rest``: the teacher's remaining mass is one more class."""
    c = {"kind": "distill", "rows": rows, "vocab": vocab, "k": k, "dtype": dtype,
         "values": values, "scale": scale, "rest": rest, "pad": pad, "masked": masked,
         "train": train}
    return c if name is None else dict(c, name=name)


def _w4(M, K, N, world, rank, dtype, group=128, zeros=False, name=None):
    c = {"kind": "w4", "M": M, "K": K, "N": N, "world": world, "rank": rank, "dtype": dtype,
         "group": group, "zeros": zeros}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one sequence's next token: latency, a row split over the chip
        _logprobs(1, 28672, "bf16", top=20, name="logprobs_1row_top20"),
        # a decode batch with alternatives for each token
        _logprobs(64, 28672, "bf16", top=20, scale=0.8, masked=2000, name="logprobs_64rows_top20"),
        # cross entropy over a batch of sequences, with entropy and log-sum terms
        _logprobs(4096, 28672, "bf16", grad="step", name="logprobs_4096rows_step"),
        # a policy update: what the gradient is weighted with follows from the log probabilities
        _logprobs(2048, 32000, "f16", grad="after", name="logprobs_2048rows_after"),
        # scoring with many alternatives; an odd vocabulary in 32 bits, rows at any alignment
        _logprobs(333, 100003, "f32", top=64, scale=1.25, name="logprobs_ragged_f32_top64"),
        # an evaluation's loss, no gradient
        _distill(64, 8192, 16, "f16", values="f16", train=False, name="distill_64rows_eval"),
        # a training step over a batch of sequences: loss and gradient
        _distill(4096, 28672, 64, "bf16", rest=True, name="distill_4096rows_rest"),
        # a row of 256 KiB
        _distill(1024, 131072, 32, "bf16", scale=0.5, name="distill_large_vocab"),
        # an odd vocabulary in 32 bits, a padded one, an odd number of entries
        _distill(1000, 50001, 99, "f32", scale=0.7, pad=3, masked=2000, name="distill_ragged_f32"),
        # a single token through the large layer's shard
        _w4(1, 8192, 3584, 8, 3, "bf16", name="w4_1token_large"),
        # a decode batch through the large layer's shard
        _w4(64, 8192, 3584, 8, 0, "bf16", zeros=True, name="w4_64tokens_large"),
        # the whole head on one rank, a small batch
        _w4(16, 8192, 28672, 1, 0, "f16", group=64, name="w4_16tokens_whole"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.random()
    if what < 0.3:
        group = rng.choice((32, 64, 128, 128))
        K = max(group, _log_int(rng, 512, 8192) // group * group)
        N = _log_int(rng, 256, 8192) // 8 * 8
        if rng.random() < 0.3:      # K ends inside a group
            K = max(32, K - 32)
        world = rng.choice((1, 2, 4, 8, 8))
        return _w4(rng.choice((1, 1, 2, 3, 4, 8, 13, 16, 24, 32, 47, 64)), K, N, world,
                   rng.randrange(world), rng.choice(("bf16", "bf16", "f16")), group,
                   rng.random() < 0.5)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    rows = _log_int(rng, 1, 4096)
    vocab = _log_int(rng, 1000, 131072)
    if rng.random() < 0.5:
        vocab = vocab // 128 * 128 + 128
    vocab = min(vocab, 131072)
    while rows * vocab * DTYPES[dtype].itemsize > 4096 * 28672 * 2:
        rows //= 2
    pad = rng.choice((0, 0, 0, 1, 8, 64))
    masked = rng.choice((0, 0, vocab // 50, vocab // 3))
    scale = rng.choice((1.0, 1.0, 0.7, 1.25))
    if what < 0.65:
        grad = rng.choice(("none", "none", "none", "step", "after"))
        top = rng.choice((0, 1, 5, 20, 20, 64, 100) if grad == "none" else (0, 0, 1, 5))
        return _logprobs(rows, vocab, dtype, top, scale, pad, masked, grad)
    return _distill(rows, vocab, rng.choice((1, 8, 16, 32, 50, 64, 100, 128)), dtype,
                    rng.choice(("f32", "f32", "bf16", "f16")), scale, rng.random() < 0.4, pad,
                    masked, rng.random() < 0.8)


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _logits(case, gen):
    """[rows, vocab] view of rows that are vocab + pad apart: spread like a head's logits, in
    half the rows one token far ahead; the masked columns -inf."""
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn((rows, vocab + case["pad"]), generator=gen, device="cuda").mul_(2.0)
    ahead = torch.randint(0, vocab - case["masked"], (rows,), generator=gen, device="cuda")
    lift = torch.rand((rows,), generator=gen, device="cuda").sub_(0.5).clamp_(min=0).mul_(24.0)
    x[torch.arange(rows, device="cuda"), ahead] += lift
    x = x.to(DTYPES[case["dtype"]])[:, :vocab]
    if case["masked"]:
        x[:, vocab - case["masked"]:] = -math.inf
    return x, ahead


def _logprobs_inputs(case, seed):
    gen = _generator(seed)
    rows = case["rows"]
    x, ahead = _logits(case, gen)
    other = torch.randint(0, case["vocab"] - case["masked"], (rows,), generator=gen, device="cuda")
    u = torch.rand((rows,), generator=gen, device="cuda")
    targets = torch.where(u < 0.6, ahead, other)
    targets = torch.where(u > 0.95, -1, targets) if rows > 1 else targets   # no token asked for
    grads = torch.randn((3, rows), generator=gen, device="cuda")
    return x, targets, grads


def _distill_inputs(case, seed):
    gen = _generator(seed)
    rows, k = case["rows"], case["k"]
    x, _ = _logits(case, gen)
    t = torch.randn(x.shape, generator=gen, device="cuda").mul_(0.7).add_(x)
    values, ids = t.topk(k, dim=1)
    values = (values - t.logsumexp(1, keepdim=True)).to(DTYPES[case["values"]])
    # lists of fewer entries, and rows without any
    length = torch.randint(1, 4 * k + 1, (rows, 1), generator=gen, device="cuda")
    length = torch.where(torch.rand((rows, 1), generator=gen, device="cuda") < 0.03, 0, length)
    if rows == 1:
        length.fill_(k)
    ids = torch.where(torch.arange(k, device="cuda") < length, ids, -1)
    weight = torch.rand((rows,), generator=gen, device="cuda").add_(0.5)
    return x, ids, values, weight


def _w4_inputs(case, seed):
    gen = _generator(seed)
    M, K, N = case["M"], case["K"], case["N"]
    dt = DTYPES[case["dtype"]]
    groups = -(-K // case["group"])
    X = torch.randn((M, K), generator=gen, device="cuda").to(dt)
    q = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.rand((N, groups), generator=gen, device="cuda").add_(0.5)
    scales = (scales * (0.2 / math.sqrt(K))).to(dt)
    zeros = None
    if case["zeros"]:
        zeros = torch.randint(5, 11, (N, groups), generator=gen, device="cuda", dtype=torch.uint8)
    return X, q, scales, zeros


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] == "w4":
        M, N, w, r = case["M"], case["N"], case["world"], case["rank"]
        s["X"], s["q"], s["scales"], s["zeros"] = _w4_inputs(case, seed)
        tiles = -(-N // 16)
        if own:
            import paper_2511_12500_amd as sym
            heap = sym.Heap(w, M * w * N * 2 + w * tiles * 4 + 4096)
            out = sym.GatheredOutput(heap, M, N, DTYPES[case["dtype"]], sym.W4_TILE_M,
                                     sym.W4_TILE_N)
            C, arrived = out.C_all(), out.arrived_all().view(w, w, tiles)
            s["out"] = out
            s["weight"] = sym.W4Weight(s["q"], s["scales"], s["zeros"], case["group"])
        else:
            C = torch.zeros((w, M, w * N), dtype=DTYPES[case["dtype"]], device="cuda")
            arrived = torch.zeros((w, w, tiles), dtype=torch.int32, device="cuda")
        s["block"], s["arrived"] = C[:, :, r * N:(r + 1) * N], arrived[:, r]
        return s
    rows, vocab, dt = case["rows"], case["vocab"], DTYPES[case["dtype"]]
    if case["kind"] == "logprobs":
        s["logits"], s["targets"], s["grads"] = _logprobs_inputs(case, seed)
    else:
        s["logits"], s["ids"], s["values"], s["weight"] = _distill_inputs(case, seed)
    if own:
        import paper_2511_12500_amd as sym
        s["op"] = (sym.TokenLogprobs(rows, vocab, dt, top=case["top"], scale=case["scale"])
                   if case["kind"] == "logprobs" else
                   sym.TopDistillation(rows, vocab, dt, case["k"], scale=case["scale"],
                                       rest=case["rest"]))
        s["dlogits"] = torch.empty((rows, vocab), dtype=dt, device="cuda")
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"logprobs": _own_logprobs, "distill": _own_distill, "w4": _own_w4}[kind](state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill, "w4": _plain_w4}[kind](state)


def _own_logprobs(s):
    op, grad, g = s["op"], s["case"]["grad"], s["grads"]
    got = {"logprob": op.logprob, "entropy": op.entropy, "top_ids": op.top_ids,
           "top_logprobs": op.top_logprobs}
    if grad == "step":
        op.run(s["logits"], s["targets"], s["dlogits"], g[0], g[1], g[2])
    else:
        op.run(s["logits"], s["targets"])
    if grad == "after":
        op.backward(s["logits"], s["targets"], s["dlogits"], g[0], g[1], g[2])
    if grad != "none":
        got["dlogits"] = s["dlogits"]
    return got


def _own_distill(s):
    op = s["op"]
    if not s["case"]["train"]:
        op.run(s["logits"], s["ids"], s["values"])
        return {"loss": op.loss}
    op.run(s["logits"], s["ids"], s["values"], s["weight"], s["dlogits"])
    return {"loss": op.loss, "dlogits": s["dlogits"]}


def _own_w4(s):
    s["out"].run_w4(s["X"], s["weight"], s["case"]["rank"])
    return {"block": s["block"], "arrived": s["arrived"]}


def _plain_logprobs(s):
    case, logits, targets, g = s["case"], s["logits"], s["targets"], s["grads"]
    x = logits.float()
    z = (x - x.amax(1, keepdim=True)) * case["scale"]
    e = z.exp()
    log_sum = e.sum(1, keepdim=True).log()
    logp = z - log_sum
    p = logp.exp()
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1)
    asked = (targets >= 0)
    at = targets.clamp(min=0)[:, None]
    logprob = torch.where(asked, logp.gather(1, at)[:, 0], 0.0)
    # the order of the floats as whole numbers, then the lower index first
    top_ids = torch.empty((x.shape[0], 0), dtype=torch.int64, device=x.device)
    top_logprobs = torch.empty((x.shape[0], 0), dtype=torch.float32, device=x.device)
    if case["top"]:
        b = (x + 0.0).view(torch.int32)
        key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).to(torch.int64) * (1 << 32)
        key = key + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
        top_ids = key.topk(case["top"], dim=1).indices
        top_logprobs = logp.gather(1, top_ids)
    got = {"logprob": logprob, "entropy": entropy, "top_ids": top_ids,
           "top_logprobs": top_logprobs}
    if case["grad"] != "none":
        gl = torch.where(asked, g[0], 0.0)
        d = p * (g[2] - gl)[:, None] - (plogp + p * entropy[:, None]) * g[1][:, None]
        d.scatter_add_(1, at, gl[:, None])
        got["dlogits"] = (d * case["scale"]).to(logits.dtype)
    return got


def _plain_distill(s):
    case, logits, ids = s["case"], s["logits"], s["ids"]
    x = logits.float()
    z = (x - x.amax(1, keepdim=True)) * case["scale"]
    e = z.exp()
    total = e.sum(1, keepdim=True)
    valid = ids >= 0
    some = valid.any(1)
    at = ids.clamp(min=0)
    v = s["values"].float()
    if case["rest"]:
        q = torch.where(valid, v.exp(), 0.0)
        logq = v
        q_rest = torch.where(some, (1.0 - q.sum(1)).clamp(min=0.0), 0.0)
    else:
        v = torch.where(valid, v * case["scale"], -math.inf)
        v = v - torch.where(some, v.amax(1), 0.0)[:, None]
        q = v.exp()
        sum_q = q.sum(1, keepdim=True).clamp(min=1e-30)
        q, logq = q / sum_q, v - sum_q.log()
        q_rest = torch.zeros_like(q[:, 0])
    logp = z.gather(1, at) - total.log()
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    # the classes outside the list
    outside = torch.ones(x.shape, dtype=torch.int32, device=x.device)
    outside.scatter_add_(1, at, -valid.to(torch.int32))
    outside = outside > 0
    rest = torch.where(outside, e, 0.0).sum(1)
    has = (q_rest > 0) & (rest > 0)
    term = q_rest * (q_rest.clamp(min=1e-30).log() - (rest / total[:, 0]).clamp(min=1e-38).log())
    loss = loss + torch.where(has, term, 0.0)
    if not case["train"]:
        return {"loss": loss}
    q_rest = torch.where(has, q_rest, 0.0)
    in_all = (q.sum(1) + q_rest)[:, None] / total
    of_rest = (q_rest / rest.clamp(min=1e-38))[:, None]
    d = e * in_all - torch.where(outside, e, 0.0) * of_rest
    d.scatter_add_(1, at, -q)
    d = d * (s["weight"] * case["scale"])[:, None]
    return {"loss": loss, "dlogits": d.to(logits.dtype)}


def _plain_w4(s):
    case, q = s["case"], s["q"]
    K = case["K"]
    w = torch.stack((q & 15, q >> 4), dim=2).view(q.shape[0], K).float()
    z = s["zeros"].float() if s["zeros"] is not None else torch.full_like(s["scales"], 8.0).float()
    spread = torch.arange(K, device=q.device) // case["group"]
    w = (w - z[:, spread]) * s["scales"].float()[:, spread]
    y = s["X"].float() @ w.t()
    s["block"].copy_(y.to(s["X"].dtype).expand_as(s["block"]))
    s["arrived"].add_(1)
    return {"block": s["block"], "arrived": s["arrived"]}


def exact(case, seed):
    if case["kind"] == "w4":
        X, q, scales, zeros = _w4_inputs(case, seed)
        W = torch.empty((q.shape[0], case["K"]), dtype=torch.float64, device="cuda")
        W[:, 0::2] = (q % 16).double()
        W[:, 1::2] = (q // 16).double()
        for g in range(scales.shape[1]):
            part = W[:, g * case["group"]:(g + 1) * case["group"]]
            part -= 8.0 if zeros is None else zeros[:, g:g + 1].double()
            part *= scales[:, g:g + 1].double()
        return {"block": (W @ X.double().t()).t().expand(case["world"], -1, -1), "arrived": None}
    if case["kind"] == "logprobs":
        x, targets, g = _logprobs_inputs(case, seed)
        parts = [_exact_logprobs(case, x[i:i + 512], targets[i:i + 512], g[:, i:i + 512])
                 for i in range(0, case["rows"], 512)]
    else:
        x, ids, values, weight = _distill_inputs(case, seed)
        parts = [_exact_distill(case, x[i:i + 512], ids[i:i + 512], values[i:i + 512],
                                weight[i:i + 512]) for i in range(0, case["rows"], 512)]
    got = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if case["kind"] == "logprobs":
        got["top_ids"] = None
    return got


def _exact_logprobs(case, x, targets, g):
    """log softmax y; dy_t/dx_v = [v = t] - p_v, dH/dx_v = -p_v (y_v + H), dlse/dx_v = p_v,
    each times the scale."""
    y = torch.log_softmax(x.double() * case["scale"], dim=1)
    p = y.exp()
    H = -torch.special.xlogy(p, p).sum(1)
    r = torch.arange(x.shape[0], device=x.device)
    use = targets >= 0
    got = {"logprob": torch.zeros_like(H), "entropy": H}
    got["logprob"][use] = y[r[use], targets[use]]
    got["top_logprobs"] = y.topk(case["top"], dim=1).values
    if case["grad"] != "none":
        g = g.double()
        d = p * g[2][:, None]
        d -= (torch.special.xlogy(p, p) + p * H[:, None]) * g[1][:, None]
        d[use] -= p[use] * g[0][use][:, None]
        d[r[use], targets[use]] += g[0][use]
        got["dlogits"] = d * case["scale"]
    return got


def _exact_distill(case, x, ids, values, weight):
    """sum_j q_j (log q_j - y_j), and with the rest q_R (log q_R - log p_R); d/dx_v is
    (sum q) p_v - q_v, for v outside the list with q_R p_v / p_R for q_v, times the scale."""
    y = torch.log_softmax(x.double() * case["scale"], dim=1)
    r, j = (ids >= 0).nonzero(as_tuple=True)
    t = torch.full(ids.shape, -math.inf, dtype=torch.float64, device=x.device)
    t[r, j] = values[r, j].double() * (1.0 if case["rest"] else case["scale"])
    if not case["rest"]:
        t = torch.nan_to_num(torch.log_softmax(t, dim=1), nan=-math.inf)
    q = t.exp()
    Q = torch.zeros_like(y)
    Q[r, ids[r, j]] = q[r, j]
    listed_ = torch.zeros(y.shape, dtype=torch.bool, device=x.device)
    listed_[r, ids[r, j]] = True
    loss = torch.special.xlogy(Q, Q).sum(1) - torch.where(Q > 0, Q * y, 0.0).sum(1)
    p = y.exp()
    qR = torch.zeros_like(loss)
    if case["rest"]:
        pR = torch.where(listed_, 0.0, p).sum(1)
        qR = torch.where((ids >= 0).any(1) & (pR > 0), (1.0 - q.sum(1)).clamp(min=0.0), 0.0)
        loss = loss + torch.where(qR > 0, torch.special.xlogy(qR, qR / pR), 0.0)
        Q = torch.where(listed_, Q, p * (qR / pR.clamp(min=1e-300))[:, None])
    if not case["train"]:
        return {"loss": loss}
    d = p * (q.sum(1) + qR)[:, None] - Q
    return {"loss": loss, "dlogits": d * (weight.double() * case["scale"])[:, None]}


def work(case):
    if case["kind"] == "w4":
        M, K, N, w = case["M"], case["K"], case["N"], case["world"]
        groups, tiles = -(-K // case["group"]), -(-N // 16)
        weights = N * K // 2 + N * groups * (3 if case["zeros"] else 2)
        return {"bytes": weights + 2 * M * K + 2 * w * M * N + 4 * w * tiles,
                "flops": 2 * M * K * N}
    rows, n = case["rows"], case["rows"] * case["vocab"]
    esize = DTYPES[case["dtype"]].itemsize
    if case["kind"] == "logprobs":
        # with weights that follow from the values the logits are read once for those and once
        # for the gradient
        passes, grad = {"none": (1, 0), "step": (2, 1), "after": (3, 1)}[case["grad"]]
        return {"bytes": n * esize * passes + rows * (16 + 12 * case["top"] + 12 * grad),
                "flops": n * (6 + 10 * grad)}
    return {"bytes": n * esize * (2 if case["train"] else 1) +
            rows * (4 + case["k"] * (8 + DTYPES[case["values"]].itemsize) +
                    (4 if case["train"] else 0)),
            "flops": n * (9 if case["train"] else 4)}
