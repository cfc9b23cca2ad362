"""GPU tests of the verification of drafted tokens (DraftVerification) against the
definition in 64 bits.  A decision or a draw that lies within the fp32 error of its
border (tests/ends_oracle.py has the bounds) may go either way; the sequences compared
are counted, so that this cannot hide a wrong kernel."""
import math

import numpy as np
import pytest
import torch

from tests import ends_oracle as o
from tests.gpu_util import require_gpu, sym

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


def inputs(S, k, V, dtype, seed, mode="draft", masked=0, near=0.5, short=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((S, k + 1, V), generator=g) * 2.5
    ahead = torch.randint(0, V, (S, k + 1), generator=g)
    lift = (torch.rand((S, k + 1), generator=g) - 0.4).clamp(min=0) * 25
    x.scatter_add_(2, ahead[:, :, None], lift[:, :, None])
    y = x[:, :k] + near * torch.randn((S, k, V), generator=g)
    if masked:
        x[:, :, V - masked:] = -math.inf
        y[:, :, V - masked:] = -math.inf
    x, y = x.to(TD[dtype]), y.to(TD[dtype])
    race = -torch.log(-torch.log(torch.rand((S, k, V), generator=g).clamp(1e-7, 1 - 1e-7)))
    if mode == "greedy":
        race = race * 0.2
    ids = (y.float() + race).argmax(2) if k else torch.empty((S, 0), dtype=torch.int64)
    if short and k:
        length = torch.randint(0, 2 * k + 1, (S, 1), generator=g)
        ids = torch.where(torch.arange(k) < length, ids, -1)
    u = torch.rand((S, k), generator=g)
    e = (-torch.log1p(-torch.rand((S, V), generator=g))).clamp(min=1e-20)
    return x.view(S * (k + 1), V), ids, u, e, y.reshape(S * k, V)


def check(S, k, op, x, ids, u, e, y, scale, draft_scale, least=None):
    torch.cuda.synchronize()
    tokens, accepted, logprob = op.tokens.cpu().numpy(), op.accepted.cpu().numpy(), op.logprob.cpu().numpy()
    x = x.double().numpy().reshape(S, k + 1, -1)
    y = None if y is None else y.double().numpy().reshape(S, k, x.shape[2])
    certain = 0
    for b in range(S):
        v = o.verify(x[b], None if y is None else y[b], ids[b].numpy(), u[b].numpy() if u is not None else None,
                     None if e is None else e[b].numpy(), scale, draft_scale)
        n = len(v.tokens)
        assert tokens[b, :n].tolist() == v.tokens, (b, v.tokens, tokens[b])
        # logits of the type, (x - m) scale and its sum's logarithm, each rounded in fp32; the
        # sum has at most 200 roundings of half a step and exponentials of errors like those
        tol = lambda lp: 2e-5 + 4 * o.U * abs(lp)                                  # noqa: E731
        for i in range(n):
            assert abs(logprob[b, i] - v.logprob[i]) <= tol(v.logprob[i]), (b, i)
        if v.open:
            continue
        certain += len(v.last) == 1
        assert accepted[b] == n, (b, accepted[b], n)
        assert int(tokens[b, n]) in v.last, (b, tokens[b], v.last)
        lp = v.last[int(tokens[b, n])]
        assert abs(logprob[b, n] - lp) <= tol(lp), (b, logprob[b, n], lp)
        assert (tokens[b, n + 1:] == -1).all() and (logprob[b, n + 1:] == 0).all(), b
    # a border is met by one sequence in some thousand
    assert certain >= (S - 1 - S // 50 if least is None else least), certain


def call(S, k, V, dtype, t, mode, scale=1.0, draft_scale=1.0, pad=0, least=None, **kw):
    x, ids, u, e, y = t
    op = sym().DraftVerification(S, k, V, TD[dtype], scale, draft_scale)
    op.tokens.fill_(-77)
    op.accepted.fill_(-77)
    op.logprob.fill_(math.nan)

    def rows(m):
        wide = torch.full((m.shape[0], V + pad), math.nan, dtype=m.dtype, device="cuda")
        wide[:, :V] = m
        return wide[:, :V]
    if mode == "greedy":
        op.run(rows(x), ids.cuda(), **kw)
        check(S, k, op, x, ids, None, None, None, scale, draft_scale, least)
    else:
        op.run(rows(x), ids.cuda(), u.cuda(), rows(e), rows(y) if mode == "draft" else None, **kw)
        check(S, k, op, x, ids, u, e, y if mode == "draft" else None, scale, draft_scale, least)
    if op.ws is not None:
        assert int(op.ws[:65536].sum()) == 0      # the counters
    return op


SHAPES = [  # sequences, drafted, vocab, scale, draft scale, pad, masked
    (1, 0, 1, 1.0, 1.0, 0, 0), (1, 1, 1, 1.0, 1.0, 0, 0), (3, 2, 7, 1.0, 1.0, 0, 0), (40, 4, 100, 0.7, 0.9, 1, 20),
    (17, 3, 1000, 1.25, 1.0, 3, 0), (5, 8, 4097, 1.0, 1.0, 0, 100), (64, 1, 2051, 1.0, 0.5, 5, 0),
    (2, 32, 777, 1.0, 1.0, 0, 0), (1, 4, 28672, 1.0, 1.0, 0, 0), (6, 5, 50001, 0.8, 0.8, 3, 2000),
    (2, 1, 140001, 1.0, 1.0, 0, 0), (300, 1, 64, 1.0, 1.0, 0, 0), (3, 0, 32000, 1.0, 1.0, 8, 0),
    (9, 2, 2, 1.0, 1.0, 2, 0), (9, 3, 3, 1.0, 1.0, 0, 0), (9, 1, 5, 1.0, 1.0, 1, 1), (260, 1, 9001, 1.0, 1.0, 0, 0),
    (2, 2, 2097152, 1.0, 1.0, 0, 0), (3, 1, 2097147, 0.9, 1.0, 1, 1000)]


@pytest.mark.parametrize("mode", ["draft", "tokens", "greedy"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "s%d_k%d_v%d_%g_%g_p%d_m%d" % s)
def test_sequences(shape, dtype, mode):
    S, k, V, scale, draft_scale, pad, masked = shape
    t = inputs(S, k, V, dtype, S + k + V, mode, masked)
    call(S, k, V, dtype, t, mode, scale, draft_scale, pad)


@pytest.mark.parametrize("mode", ["draft", "tokens", "greedy"])
def test_full_drafts_of_a_near_model(mode):
    """Many positions accepted (without the draft's probabilities fewer: with p alone)."""
    S, k, V = 50, 5, 3000
    x, ids, u, e, y = inputs(S, k, V, "bf16", 11, "greedy", near=0.02, short=False)
    x = x + 0.0
    top = x.float().view(S, k + 1, V)[:, :k].argmax(2)
    ids = torch.where(torch.rand((S, k), generator=torch.Generator().manual_seed(1)) < 0.9, top, ids)
    op = call(S, k, V, "bf16", (x, ids, u * 0.5, e, y), mode)
    assert int((op.accepted == k).sum()) > 5 or mode == "tokens"


@pytest.mark.parametrize("mode", ["draft", "tokens", "greedy"])
@pytest.mark.parametrize("k", [1, 32])
def test_certain_tokens(mode, k):
    """Every position has a token of probability near one: all accepted but for the drafts
    that say otherwise, and the extra token follows.  (Another token than that is as unlikely
    to the drafting model as to the target, so that with its probabilities it may pass.)"""
    S, V = 9, 600
    x, ids, u, e, y = inputs(S, k, V, "f32", 12, "greedy", short=False)
    top = torch.randint(0, V, (S, k + 1), generator=torch.Generator().manual_seed(2))
    x.view(S, k + 1, V).scatter_(2, top[:, :, None], 60.0)
    y.view(S, k, V).scatter_(2, top[:, :k, None], 60.0)
    ids = top[:, :k].clone()
    if mode != "draft":
        ids[3, k - 1] = (ids[3, k - 1] + 1) % V
    ids[4, k // 2] = -1
    op = call(S, k, V, "f32", (x, ids, u, e, y), mode)
    want = torch.full((S,), k)
    want[3], want[4] = k if mode == "draft" else k - 1, k // 2
    assert op.accepted.cpu().tolist() == want.tolist()
    at = torch.arange(k + 1) <= want[:, None]
    assert torch.equal(op.tokens.cpu(), torch.where(at, top, -1))


@pytest.mark.parametrize("mode", ["draft", "tokens"])
def test_borders_of_the_random_numbers(mode):
    """u = 0 accepts what has p > 0 alone; p = q gives no residual and draws from p; a drafted
    token outside the vocabulary is never accepted; absent tokens inside a list end it."""
    V = 50
    x = torch.zeros((8 * 3, V))
    x[:, 7] = -math.inf
    x[:, 3] = 1.0
    y = x.view(8, 3, V)[:, :2].reshape(16, V).clone()
    ids = torch.tensor([[7, 1], [3, 7], [1, -1], [-1, 1], [V, 1], [1, V + 5], [2 ** 40, 0], [3, -5]])
    u = torch.zeros((8, 2))
    e = (-torch.log1p(-torch.rand((8, V), generator=torch.Generator().manual_seed(0)))).clamp(min=1e-20)
    op = call(8, 2, V, "f32", (x, ids, u, e, y), mode, least=0)
    assert op.accepted.tolist() == [0, 1, 1, 0, 0, 1, 0, 1]
    assert not bool((op.tokens == 7).any())
    # u beyond 1 rejects all; where the draft is the target nothing of the residual is left
    op = call(8, 2, V, "f32", (x, ids, u + 2.0, e, y), mode, least=0)
    assert op.accepted.tolist() == [0] * 8
    if mode == "draft":
        want = (torch.softmax(x[0].double(), 0) / e.double()).argmax(1)
        assert op.tokens[:, 0].cpu().tolist() == want.tolist()


@pytest.mark.parametrize("mode", ["draft", "tokens", "greedy"])
@pytest.mark.parametrize("V", [300, 40000])
def test_rows_without_a_distribution(mode, V):
    """A NaN, an infinity or nothing above -inf in the target's row: the position is not
    accepted and has no token; in the draft's row: not accepted, drawn from the target."""
    S, k = 6, 2
    x, ids, u, e, y = inputs(S, k, V, "f32", 3, "greedy", short=False)
    x = x.view(S, k + 1, V)
    ids = x[:, :k].argmax(2)
    u.zero_()
    x[0, 0, 5] = math.nan
    x[1, 1, V - 1] = math.inf
    x[2, 2] = -math.inf
    x[3, 0] = -math.inf
    y = y.view(S, k, V)
    y[4, 1, 0] = math.nan
    y[5, 0] = -math.inf
    op = call(S, k, V, "f32", (x.reshape(-1, V), ids, u, e, y.reshape(-1, V)), mode, least=0)
    assert op.accepted[:4].tolist() == [0, 1, 2, 0]
    assert op.tokens[[0, 1, 2, 3], [0, 1, 2, 0]].tolist() == [-1] * 4
    if mode == "draft":
        assert op.accepted[4:].tolist() == [1, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [4, 6, 1001, 1002, 1003, 8195, 50001])
def test_tokens_at_the_end(V, dtype):
    """All but the last four tokens masked: each of them is drawn with its own noise."""
    S, k = 64, 1
    x, ids, u, e, y = inputs(S, k, V, dtype, V, "tokens", short=False)
    x[:, :V - 4] = -math.inf
    y[:, :V - 4] = -math.inf
    ids = V - 1 - torch.randint(0, 4, (S, k), generator=torch.Generator().manual_seed(V))
    op = call(S, k, V, dtype, (x, ids, u, e, y), "draft", pad=V % 3)
    drawn = op.tokens.cpu()[torch.arange(S), op.accepted.cpu()]
    assert sorted(set(drawn.tolist())) == list(range(V - 4, V))


@pytest.mark.parametrize("low", [-1e4, -1e10, -3e38])
def test_masks_of_low_values(low):
    """Masked by a large negative number in place of -inf."""
    S, k, V = 8, 2, 5000
    x, ids, u, e, y = inputs(S, k, V, "f32", 5)
    x[:, 1000:], y[:, 1000:] = low, low
    ids = ids % 1000 * (ids >= 0) + ids * (ids < 0)
    call(S, k, V, "f32", (x, ids, u, e, y), "draft")
    call(S, k, V, "f32", (x + low, ids, u, e, y), "greedy")


def test_equal_largest_logits():
    """Greedy takes the lowest of equal ones, wherever they lie in the row."""
    V = 140000
    x = torch.zeros((4 * 2, V))
    for r, at in enumerate([0, 9, 4095, 32768, 70001, V - 1, 100000, 5]):
        x[r, at:] = 1.0
    ids = torch.tensor([[0], [4096], [70001], [99999]])
    op = call(4, 1, V, "bf16", (x.bfloat16(), ids, None, None, None), "greedy", least=4)
    assert op.accepted.tolist() == [1, 0, 1, 0]
    assert op.tokens[:, 0].tolist() == [0, 4095, 70001, 100000]


def test_many_sequences():
    """More than one launch's."""
    S, k, V = 16384 // 9 + 300, 4, 40
    t = inputs(S, k, V, "f32", 21)
    call(S, k, V, "f32", t, "draft")


def test_another_stream_and_shared_noise():
    """A call on another stream; one row of noise for all sequences, which would tie their
    draws together, is refused."""
    S, k, V = 4, 2, 1000
    x, ids, u, e, y = inputs(S, k, V, "f32", 9)
    s = torch.cuda.Stream()
    op = call(S, k, V, "f32", (x, ids, u, e, y), "draft")
    want = [op.tokens.clone(), op.accepted.clone(), op.logprob.clone()]
    args = [a.cuda() for a in (x, ids, u, e, y)]
    op.tokens.zero_()
    torch.cuda.synchronize()
    op.run(*args, stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (op.tokens, op.accepted, op.logprob)))
    with pytest.raises(ValueError, match="noise: rows must not overlap"):
        op.run(*args[:3], args[3][:1].expand(S, V), args[4])


@pytest.mark.parametrize("V", [3000, 50001])
def test_captured(V):
    """Two graphs on one object, replayed in turn with new inputs between eager calls."""
    S, k = 5, 3
    ts = [inputs(S, k, V, "bf16", s) for s in (1, 2, 3)]
    op = sym().DraftVerification(S, k, V, torch.bfloat16)
    x, ids, u, e, y = (a.cuda() for a in ts[0])
    op.run(x, ids, u, e, y)
    graphs = []
    for mode in ("draft", "greedy"):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            op.run(x, ids, u, e, y) if mode == "draft" else op.run(x, ids)
    for i in range(5):
        t = ts[i % 3]
        for to, of in zip((x, ids, u, e, y), t):
            to.copy_(of)
        graphs[0].replay()
        check(S, k, op, *t, 1.0, 1.0)
        graphs[1].replay()
        check(S, k, op, t[0], t[1], None, None, None, 1.0, 1.0)
        if i == 2:
            op.run(x, ids, u, e)
            check(S, k, op, *t[:4], None, 1.0, 1.0)


def test_refusals():
    pkg = sym()
    S, k, V = 2, 3, 100
    x, ids, u, e, y = (a.cuda() for a in inputs(S, k, V, "f32", 1))
    op = pkg.DraftVerification(S, k, V, torch.float32)
    for bad in ((x[:-1], ids), (x, ids[:, :2].contiguous()), (x, ids.t().contiguous().t()), (x, ids, u[:1], e),
                (x, ids, u, e[:, :50]), (x, ids, u, e, y[1:]), (x.cpu(), ids)):
        with pytest.raises(ValueError):
            op.run(*bad)
    for bad in ((x.half(), ids), (x, ids.int()), (x, ids, u.double(), e), (x, ids, u, e, y.half())):
        with pytest.raises(TypeError):
            op.run(*bad)
    for bad in ((x, ids, u), (x, ids, None, e), (x, ids, None, None, y)):
        with pytest.raises(pkg.SymtileError) as err:
            op.run(*bad)
        assert err.value.name == "EINVAL"
    for bad in ((0, -1, k, V, 3), (0, S, 33, V, 3), (0, S, -1, V, 3), (0, S, k, 0, 3), (0, S, k, (1 << 21) + 1, 3),
                (0, S, k, V, 9), (99, S, k, V, 3)):
        with pytest.raises(pkg.SymtileError) as err:
            pkg.symtile_verify_workspace_bytes(*bad)
        assert err.value.name == "EINVAL", bad
    pkg.DraftVerification(0, k, V, torch.float32).run(x[:0], ids[:0], u[:0], e[:0])
    with pytest.raises(pkg.SymtileError):
        bad = pkg.DraftVerification(S, k, V, torch.float32, scale=0.0)
        bad.run(x, ids, u, e)
