"""GPU tests of token log probabilities and of the distillation loss, with their
gradients, against the 64-bit definitions in tests/head_oracle.py.

Bounds are those of head_oracle (derived there for fp32 sums); ids are compared
exactly.  Inputs are exact in the tested type, so the oracle sees what the
kernels see."""
import math

import numpy as np
import pytest
import torch

from tests import head_oracle as O
from tests.gpu_util import require_gpu, sym

pytestmark = pytest.mark.gpu

INF = math.inf
TD = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LOW = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal_rows(rows, vocab, dtype, seed, spread=2.0):
    return (torch.randn((rows, vocab), generator=gen(seed)) * spread).to(TD[dtype])


def special_rows(vocab, dtype, seed):
    """Rows at which a kernel can go wrong: equal, empty and nearly empty ones, the type's lowest
    value, sorted either way, whole-number ties, signed zeros, one row far ahead of all others."""
    g = gen(seed)
    low = LOW[dtype]
    n = torch.arange(vocab, dtype=torch.float32)
    rnd = torch.randn((vocab,), generator=g)
    rows = [torch.full((vocab,), 1.5), torch.full((vocab,), -INF), torch.full((vocab,), low)]
    one = torch.full((vocab,), -INF)
    one[vocab // 2] = -3.0
    rows.append(one)
    one = torch.full((vocab,), low)
    one[vocab - 1] = 2.0
    rows.append(one)
    half = rnd.clone()
    half[torch.rand((vocab,), generator=g) < 0.5] = -INF
    rows.append(half)
    half = rnd.clone()
    half[torch.rand((vocab,), generator=g) < 0.5] = low
    rows.append(half)
    rows += [n / vocab * 8, (vocab - n) / vocab * 8]
    rows.append(torch.randint(-2, 3, (vocab,), generator=g).float())
    rows.append(torch.where(torch.rand((vocab,), generator=g) < 0.5, -0.0, 0.0))
    far = rnd.clone()
    far[vocab // 3] = 300.0
    rows.append(far)
    return torch.stack(rows).to(TD[dtype])


def place(x, pad, offset=0):
    """x on the GPU as a view of rows that are vocab + pad apart, the first one `offset`
    elements into its memory, and the memory (which holds a pattern elsewhere)."""
    rows, vocab = x.shape
    mem = torch.full((offset + rows * (vocab + pad) + 8,), 7.0, dtype=x.dtype, device="cuda")
    view = mem[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(x)
    return view, mem


def close(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    with np.errstate(over="ignore"):      # what is beyond the outputs' range is an infinity there
        want = np.where(np.isinf(want.astype(np.float32)), want.astype(np.float32), want)
    bound = np.broadcast_to(np.asarray(bound, np.float64), want.shape)
    fin = np.isfinite(want)
    same = np.where(np.isnan(want), np.isnan(got), got == want)
    with np.errstate(invalid="ignore"):
        ok = np.where(fin, np.abs(got - want) <= bound, same)
    if not ok.all():
        i = tuple(int(v) for v in np.argwhere(~ok)[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} off, first at {i}: got {got[i]!r}, "
                             f"want {want[i]!r}, bound {bound[i]:.3e}")


def check_logprobs(op, x, targets, scale, top):
    """All outputs of op for the rows x (CPU tensor)."""
    X = x.double().numpy()
    got = [t.cpu().numpy() for t in (op.logprob, op.entropy, op.stats, op.top_ids, op.top_logprobs)]
    for r in range(X.shape[0]):
        lp, H, (m, log_s), ids, tl = O.token_logprobs(X[r], int(targets[r]), scale, top)
        b = O.log_bound(X[r], scale)
        # the entropy is log s less a mean of exponents, each as exact as a log probability
        hb = b * (2 + abs(H)) + 8 * O.U * (abs(log_s) + abs(H))
        close(got[0][r], lp, O.value_bound(X[r], scale, lp), f"row {r} logprob")
        close(got[1][r], H, hb, f"row {r} entropy")
        close(got[2][r], [m, log_s], [0.0, b], f"row {r} stats")
        assert np.array_equal(got[3][r], ids), (r, got[3][r], ids)
        close(got[4][r], tl, [O.value_bound(X[r], scale, v) for v in tl], f"row {r} top")


def check_logprob_grad(got, x, targets, scale, g, dtype):
    X = x.double().numpy()
    got = got.double().cpu().numpy()
    for r in range(X.shape[0]):
        gl, ge, gs = (0.0 if t is None else float(t[r]) for t in g)
        want = O.token_logprobs_grad(X[r], int(targets[r]), scale, gl, ge, gs)
        m, log_s, p, logp = O.row_sums(X[r], scale)
        if m == -INF:
            close(got[r], want, 0.0, f"row {r} gradient")
            continue
        lb = O.log_bound(X[r], scale) + 8 * O.U
        pos = p > 0
        l = np.where(pos, np.where(pos, logp, 0.0), 0.0)
        H = -np.sum(p * l)
        # p is off by its exponent's error relatively, logp + H absolutely
        size = p * (abs(gl) + abs(gs)) + p * np.abs(l + H) * abs(ge)
        err = size * (lb + 6 * O.U * (1 + np.abs(l))) + p * abs(ge) * (
            lb * (3 + abs(H)) + 6 * O.U * (np.abs(l) + H + abs(log_s)))
        t = int(targets[r])
        if t >= 0:
            err[t] += 4 * O.U * abs(gl)
        close(got[r], want, err * scale + O.half_ulp(np.abs(want) + err * scale, dtype) + O.TINY,
              f"row {r} gradient")


VOCABS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 127, 255, 257, 511, 1000, 2048, 4097, 8191]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs_of_special_rows(dtype, vocab):
    pkg = sym()
    x = torch.cat([special_rows(vocab, dtype, vocab), normal_rows(3, vocab, dtype, vocab + 1)])
    rows = x.shape[0]
    targets = torch.randint(-1, vocab, (rows,), generator=gen(3))
    for scale, top, pad, offset in ((1.0, min(vocab, 5), 0, 0), (0.7, min(vocab, 128), 3, 1),
                                    (1.9, 0, 8, 3)):
        dx, mem = place(x, pad, offset)
        op = pkg.TokenLogprobs(rows, vocab, TD[dtype], top=top, scale=scale)
        op.run(dx, targets.cuda())
        check_logprobs(op, x, targets, np.float32(scale).item(), top)


@pytest.mark.parametrize("dtype,rows,vocab,top", [
    ("bf16", 1, 28672, 20), ("f16", 2, 50001, 64), ("f32", 3, 100003, 128), ("bf16", 1, 131072, 128),
    ("f16", 1, 300001, 7), ("f32", 1, 262147, 1), ("bf16", 5, 32768, 0), ("bf16", 300, 1031, 20),
    ("f32", 700, 130, 3), ("f16", 40, 16384, 33),
])
def test_logprobs_of_long_and_many_rows(dtype, rows, vocab, top):
    pkg = sym()
    x = normal_rows(rows, vocab, dtype, rows + vocab)
    targets = torch.randint(0, vocab, (rows,), generator=gen(1))
    op = pkg.TokenLogprobs(rows, vocab, TD[dtype], top=top, scale=0.9)
    dx, _ = place(x, 1)
    for _ in range(2):                 # the second call runs on what the first left behind
        op.run(dx, targets.cuda())
        check_logprobs(op, x, targets, np.float32(0.9).item(), top)


@pytest.mark.parametrize("dtype,vocab", [("f32", 1 << 21), ("bf16", 1 << 21), ("f32", 1300007)])
def test_the_longest_rows(dtype, vocab):
    """As many segments as a row can have: values, top entries, both gradients."""
    pkg = sym()
    x = normal_rows(2, vocab, dtype, 3)
    x[1, 5:] = -INF                                     # all but the first segment's are masked
    targets = torch.tensor([vocab - 1, 2])
    g = [torch.randn((2,), generator=gen(k)) for k in range(3)]
    op = pkg.TokenLogprobs(2, vocab, TD[dtype], top=128)
    dl = torch.empty((2, vocab), dtype=TD[dtype], device="cuda")
    op.run(x.cuda(), targets.cuda(), dl, *[t.cuda() for t in g])
    check_logprobs(op, x, targets, 1.0, 128)
    check_logprob_grad(dl, x, targets, 1.0, g, dtype)
    ids, values = op.top_ids.cpu(), op.top_logprobs.cpu()
    kd = pkg.TopDistillation(2, vocab, TD[dtype], 128, rest=True)
    kd.run(x.cuda(), ids.cuda(), values.cuda(), g[0].cuda(), dl)
    check_distill(kd.loss, dl, x, ids, values, 1.0, True, g[0], dtype)
    with pytest.raises(pkg.SymtileError):
        pkg.TokenLogprobs(1, (1 << 21) + 1, TD[dtype])


def test_rows_past_32_bits():
    """The third row starts 2^32 elements into its memory."""
    pkg = sym()
    ld, vocab = 1 << 31, 1000
    mem = torch.empty(2 * ld + vocab, dtype=torch.bfloat16, device="cuda")
    dx = mem.as_strided((3, vocab), (ld, 1))
    x = normal_rows(3, vocab, "bf16", 3)
    dx.copy_(x)
    targets = torch.tensor([5, 999, 0])
    g = [torch.randn((3,), generator=gen(k)) for k in range(3)]
    op = pkg.TokenLogprobs(3, vocab, torch.bfloat16, top=7)
    dl = torch.empty((3, vocab), dtype=torch.bfloat16, device="cuda")
    op.run(dx, targets.cuda(), dl, *[t.cuda() for t in g])
    check_logprobs(op, x, targets, 1.0, 7)
    check_logprob_grad(dl, x, targets, 1.0, g, "bf16")
    op.backward(dx, targets.cuda(), dx, *[t.cuda() for t in g])          # in place
    check_logprob_grad(dx, x, targets, 1.0, g, "bf16")
    dx.copy_(x)
    ids, values = teacher_list(x, 9, 4, False)
    kd = pkg.TopDistillation(3, vocab, torch.bfloat16, 9)
    kd.run(dx, ids.cuda(), values.cuda(), g[0].cuda(), dx)
    check_distill(kd.loss, dx, x, ids, values, 1.0, False, g[0], "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [40000, 70000])
def test_long_special_rows(dtype, vocab):
    """Rows of ties, sorted rows and masks where a row is long or split."""
    pkg = sym()
    x = special_rows(vocab, dtype, 5)
    targets = torch.randint(-1, vocab, (x.shape[0],), generator=gen(3))
    for top in (20, 128):
        op = pkg.TokenLogprobs(x.shape[0], vocab, TD[dtype], top=top)
        op.run(x.cuda(), targets.cuda())
        check_logprobs(op, x, targets, 1.0, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 700, 9001])
def test_rows_with_nan_and_infinity(dtype, vocab):
    pkg = sym()
    x = normal_rows(4, vocab, dtype, 2)
    x[0, vocab // 2] = math.nan
    x[1, vocab - 1] = INF
    x[2] = math.nan
    op = pkg.TokenLogprobs(4, vocab, TD[dtype], top=min(vocab, 9))
    op.run(x.cuda(), torch.zeros(4, dtype=torch.int64, device="cuda"))
    lp, H, ids = op.logprob.cpu(), op.entropy.cpu(), op.top_ids.cpu().numpy()
    assert lp[0].isnan() and lp[2].isnan() and H[:3].isnan().all()
    for r in range(3):
        assert np.array_equal(ids[r], O.top_order(x[r].double().numpy())[:min(vocab, 9)]), r
    check = pkg.TokenLogprobs(1, vocab, TD[dtype], top=min(vocab, 9))   # the fourth row is untouched
    check.run(x[3:].cuda(), torch.zeros(1, dtype=torch.int64, device="cuda"))
    close(op.logprob[3].cpu(), check.logprob[0].cpu(), O.log_bound(x[3].double().numpy(), 1.0) * 2, "row 3")


GRADS = [  # which of grad_logprob, grad_entropy, grad_lse are there
    (1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab", [1, 7, 65, 1000, 4097, 28672, 70001])
def test_logprob_gradients(dtype, vocab):
    pkg = sym()
    x = torch.cat([special_rows(vocab, dtype, vocab + 7), normal_rows(2, vocab, dtype, vocab + 1)])
    rows = x.shape[0]
    targets = torch.randint(-1, vocab, (rows,), generator=gen(4))
    scale = np.float32(0.8).item()
    for i, there in enumerate(GRADS):
        g = [torch.randn((rows,), generator=gen(i + k)) if t else None for k, t in enumerate(there)]
        dg = [None if t is None else t.cuda() for t in g]
        dx, _ = place(x, i, i)
        op = pkg.TokenLogprobs(rows, vocab, TD[dtype], top=min(vocab, 4) if i == 1 else 0, scale=scale)
        dl, mem = place(torch.zeros_like(x), 2 * i, 5)
        op.run(dx, targets.cuda(), dl, *dg)                          # with the values
        check_logprob_grad(dl, x, targets, scale, g, dtype)
        check_logprobs(op, x, targets, scale, op.top)
        assert bool((mem[:5] == 7).all()), "written before the first row"
        if i:
            around = mem[5:5 + rows * (vocab + 2 * i)].view(rows, -1)[:, vocab:]
            assert bool((around == 7).all()), "written between the rows"
        assert bool((mem[5 + rows * (vocab + 2 * i):] == 7).all()), "written after the last row"
        apart = torch.full((rows, vocab), 5.0, dtype=TD[dtype], device="cuda")
        op.backward(dx, targets.cuda(), apart, *dg)                  # alone
        check_logprob_grad(apart, x, targets, scale, g, dtype)
        assert torch.equal(dx.cpu().float().nan_to_num(), x.float().nan_to_num())


def test_gradients_without_targets():
    pkg = sym()
    x = normal_rows(3, 777, "f32", 1)
    g = torch.randn((3,), generator=gen(5))
    op = pkg.TokenLogprobs(3, 777, torch.float32)
    dl = torch.empty((3, 777), device="cuda")
    op.run(x.cuda(), None, dl, None, g.cuda())
    check_logprob_grad(dl, x, [-1] * 3, 1.0, (None, g, None), "f32")


@pytest.mark.parametrize("dtype,rows,vocab", [("bf16", 30, 28672), ("f32", 2, 100001), ("f16", 5, 333)])
def test_gradient_in_place(dtype, rows, vocab):
    """dlogits may be the logits themselves, in one call or two."""
    pkg = sym()
    x = normal_rows(rows, vocab, dtype, 9)
    targets = torch.randint(-1, vocab, (rows,), generator=gen(4)).cuda()
    g = [torch.randn((rows,), generator=gen(k)).cuda() for k in range(3)]
    op = pkg.TokenLogprobs(rows, vocab, TD[dtype], top=3)
    want = torch.empty((rows, vocab), dtype=TD[dtype], device="cuda")
    op.run(x.cuda(), targets, want, *g)
    for two in (False, True):
        y, _ = place(x, 5)
        if two:
            op.run(y, targets)
            op.backward(y, targets, y, *g)
            check_logprob_grad(y, x, targets.cpu(), 1.0, [t.cpu() for t in g], dtype)
        else:
            op.run(y, targets, y, *g)
            assert torch.equal(y, want)
    ids = torch.randint(0, vocab, (rows, 8), generator=gen(6)).cuda()
    values = torch.randn((rows, 8), generator=gen(7)).cuda()
    kd = pkg.TopDistillation(rows, vocab, TD[dtype], 8)
    kd.run(x.cuda(), ids, values, g[0], want)
    y, _ = place(x, 5)
    kd.run(y, ids, values, g[0], y)
    assert torch.equal(y, want)


def test_gradients_are_differences_of_the_values():
    """fp32 logits moved by h either way: the kernel's gradient against its own values."""
    pkg = sym()
    rows, vocab, h = 40, 50, 1.0 / 64
    row = torch.randn((vocab,), generator=gen(1))
    x = row.repeat(rows, 1)
    up, down = x.clone(), x.clone()
    for r in range(rows):
        up[r, r] += h
        down[r, r] -= h
    targets = torch.full((rows,), 3, dtype=torch.int64, device="cuda")
    op = pkg.TokenLogprobs(rows, vocab, torch.float32)
    vals = []
    for t in (up, down):
        op.run(t.cuda(), targets)
        vals.append((0.5 * op.logprob.double() + 2.0 * op.entropy.double() - op.lse().double()).cpu())
    step = (up - down).double()[torch.arange(rows), torch.arange(rows)]
    dl = torch.empty((rows, vocab), device="cuda")
    op.run(x.cuda(), targets, dl, *[torch.full((rows,), v, device="cuda") for v in (0.5, 2.0, -1.0)])
    diff = (vals[0] - vals[1]) / step
    # third derivatives of these are below 40; the values' own error over the step
    tol = 40 * h * h / 6 + 8 * O.log_bound(row.numpy(), 1.0) / h
    assert float((diff - dl.cpu().double().diagonal()[:rows]).abs().max()) < tol


def test_targets_out_of_the_vocabulary():
    pkg = sym()
    x = normal_rows(3, 100, "f32", 1)
    op = pkg.TokenLogprobs(3, 100, torch.float32)
    dl = torch.empty((3, 100), device="cuda")
    one = torch.ones(3, device="cuda")
    op.run(x.cuda(), torch.tensor([100, -5, 1 << 40], device="cuda"), dl, one)
    assert op.logprob[0].isnan() and op.logprob[2].isnan() and op.logprob[1] == 0
    assert bool(dl[0].isnan().all()) and bool((dl[1] == 0).all())


# ---- distillation ------------------------------------------------------------------


def teacher_list(x, k, seed, rest, vdtype="f32"):
    """Lists as a teacher near x gives them: lengths differ, one row without entries."""
    g = gen(seed)
    rows, vocab = x.shape
    t = x.float().clamp(min=-50.0, max=50.0) + 0.7 * torch.randn(x.shape, generator=g)
    values, ids = t.topk(k, dim=1)
    values = (values - t.logsumexp(1, keepdim=True) - (0.05 if rest else 0.0)).to(TD[vdtype])
    ids = ids.clone()
    for r in range(rows):
        n = int(torch.randint(1, k + 1, (1,), generator=g)) if r % 3 == 0 else k
        ids[r, n:] = -1 - r
    if rows > 2:
        ids[2] = -1
    return ids, values


def check_distill(loss, grad, x, ids, values, scale, rest, row_grad, dtype):
    X, V, I = x.double().numpy(), values.double().numpy(), ids.numpy()
    loss = loss.cpu().numpy()
    grad = None if grad is None else grad.double().cpu().numpy()
    for r in range(X.shape[0]):
        want, wg = O.distill(X[r], I[r], V[r], scale, rest)
        m, log_s, p, logp = O.row_sums(X[r], scale)
        q, q_rest = O.teacher(I[r], V[r], scale, rest)
        lb = O.log_bound(X[r], scale) + 8 * O.U
        vmax = float(np.max(np.abs(np.where(I[r] >= 0, np.where(np.isfinite(V[r]), V[r], 0.0), 0.0)), initial=0.0))
        # q: its exponent's error, a sum of at most 128; the rest's is absolute
        qe = O.U * (4 * 2 * vmax * max(scale, 1.0) + 128 + 8)
        there = (I[r] >= 0) & (q > 0)
        lq = np.where(there, np.log(np.where(there, q, 1.0)), 0.0)
        lp = np.where(there, logp[np.clip(I[r], 0, len(X[r]) - 1)], 0.0)
        lp = np.where(np.isfinite(lp), lp, 0.0)
        b = float(np.sum(q * (qe * (2 + np.abs(lq - lp)) + lb + 8 * O.U * (np.abs(lq) + np.abs(lp)))))
        b += 128 * O.U * float(np.sum(q * np.abs(lq - lp)))
        if q_rest > 0:
            out = np.ones(len(p), dtype=bool)
            out[I[r][I[r] >= 0]] = False
            # log p_R from its own largest term: p itself may be below the smallest number
            top = float(np.max(logp[out], initial=-INF))
            log_pr = top + math.log(np.exp(logp[out] - top).sum()) if top > -INF else math.log(q_rest)
            ratio = abs(math.log(q_rest) - log_pr)
            b += (qe + 4 * O.U) * (2 + ratio + abs(math.log(q_rest))) + q_rest * (2 * lb + 16 * O.U * (1 + ratio))
        close(loss[r], want, b, f"row {r} loss")
        if grad is None:
            continue
        gr = float(row_grad[r])
        wg = wg * gr
        in_list = np.zeros(len(p))
        np.add.at(in_list, I[r][I[r] >= 0], q[I[r] >= 0])
        rel = lb + 6 * O.U * (2 + np.minimum(np.abs(np.where(p > 0, np.where(p > 0, logp, 0.0), 0.0)), 104.0))
        err = p * (rel * (1 + q.sum()) + qe) + in_list * (qe + 4 * O.U)
        if q_rest > 0:
            share = np.exp(np.where(out & np.isfinite(logp), logp - log_pr, -INF))
            err += np.where(out, share * (q_rest * 3 * rel + qe + 4 * O.U), 0.0)
        err *= abs(gr) * scale
        close(grad[r], wg, err + O.half_ulp(np.abs(wg) + err, dtype) + O.TINY, f"row {r} gradient")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("vocab,k", [(1, 1), (5, 5), (9, 3), (64, 64), (130, 128), (1000, 16),
                                     (4097, 99), (28672, 64), (70001, 128)])
def test_distillation(dtype, vocab, k, rest):
    pkg = sym()
    x = torch.cat([special_rows(vocab, dtype, vocab + 3), normal_rows(3, vocab, dtype, vocab)])
    rows = x.shape[0]
    ids, values = teacher_list(x, k, vocab + k, rest, {1: "bf16", 3: "f16"}.get(k, "f32"))
    g = torch.rand((rows,), generator=gen(1)) + 0.5
    g[rows - 1] = 0.0
    scale = np.float32(1.0 if rest else 0.75).item()
    kd = pkg.TopDistillation(rows, vocab, TD[dtype], k, scale=scale, rest=rest)
    dx, _ = place(x, 3, 1)
    kd.run(dx, ids.cuda(), values.cuda())                            # values alone
    check_distill(kd.loss, None, x, ids, values, scale, rest, g, dtype)
    alone = kd.loss.clone()
    dl, mem = place(torch.zeros_like(x), 1, 3)
    kd.run(dx, ids.cuda(), values.cuda(), g.cuda(), dl)
    check_distill(kd.loss, dl, x, ids, values, scale, rest, g, dtype)
    close(kd.loss.cpu(), alone.cpu(), 64 * O.U * (1 + alone.cpu().abs().nan_to_num(posinf=0)), "loss")
    assert bool((mem[:3] == 7).all())
    assert bool((mem[3:3 + rows * (vocab + 1)].view(rows, -1)[:, vocab] == 7).all())
    assert bool((mem[3 + rows * (vocab + 1):] == 7).all())
    back = torch.full((rows, vocab), 5.0, dtype=TD[dtype], device="cuda")
    kd.backward(dx, ids.cuda(), values.cuda(), g.cuda(), back)
    check_distill(kd.loss, back, x, ids, values, scale, rest, g, dtype)


@pytest.mark.parametrize("dtype,rows,vocab,k,rest", [
    ("bf16", 1, 131072, 32, False), ("f32", 2, 100003, 128, True), ("f16", 1, 300001, 7, True),
    ("bf16", 300, 1031, 20, True), ("f32", 600, 130, 3, False), ("f16", 33, 16384, 64, True)])
def test_distillation_of_long_and_many_rows(dtype, rows, vocab, k, rest):
    pkg = sym()
    x = normal_rows(rows, vocab, dtype, rows + vocab)
    ids, values = teacher_list(x, k, 3, rest)
    g = torch.rand((rows,), generator=gen(1)) + 0.5
    kd = pkg.TopDistillation(rows, vocab, TD[dtype], k, rest=rest)
    dl = torch.empty((rows, vocab), dtype=TD[dtype], device="cuda")
    for _ in range(2):
        kd.run(x.cuda(), ids.cuda(), values.cuda(), g.cuda(), dl)
        check_distill(kd.loss, dl, x, ids, values, 1.0, rest, g, dtype)


@pytest.mark.parametrize("rest", [False, True])
def test_lists_with_repeated_ids_and_infinite_values(rest):
    pkg = sym()
    vocab, k = 500, 12
    x = normal_rows(4, vocab, "f32", 8)
    ids = torch.randint(0, 40, (4, k), generator=gen(2))
    ids[0] = torch.tensor([7, 7, 7, 3, 3, -1, 7, 499, 0, 0, 3, 7])
    values = torch.log(torch.rand((4, k), generator=gen(3)) / k)
    values[1, 4] = -INF                        # a teacher's probability of zero
    values[0, 5] = math.nan                    # an absent entry's value is not read
    x[2, ids[2, 0]] = -INF                     # a listed token that the student has masked
    g = torch.ones(4)
    kd = pkg.TopDistillation(4, vocab, torch.float32, k, rest=rest)
    dl = torch.empty((4, vocab), device="cuda")
    kd.run(x.cuda(), ids.cuda(), values.cuda(), g.cuda(), dl)
    keep = [0, 1, 3]
    check_distill(kd.loss[keep], dl[keep], x[keep], ids[keep], values[keep], 1.0, rest, g[keep], "f32")
    assert float(kd.loss[2]) == INF
    _, want = O.distill(x[2].double().numpy(), ids[2].numpy(), values[2].double().numpy(), 1.0, rest)
    assert np.allclose(dl[2].cpu().numpy(), want, atol=1e-5)


def test_ids_out_of_the_vocabulary_give_nan():
    pkg = sym()
    x = normal_rows(3, 100, "bf16", 1)
    ids = torch.tensor([[1, 100], [1, 2], [-1, 1 << 40]], device="cuda")
    values = torch.zeros((3, 2), device="cuda")
    one = torch.ones(3, device="cuda")
    kd = pkg.TopDistillation(3, 100, torch.bfloat16, 2)
    dl = torch.zeros((3, 100), dtype=torch.bfloat16, device="cuda")
    kd.run(x.cuda(), ids, values, one, dl)
    assert kd.loss.isnan().tolist() == [True, False, True]
    assert dl.isnan().all(1).tolist() == [True, False, True] and not bool(dl[1].isnan().any())
    back = torch.zeros_like(dl)
    kd.backward(x.cuda(), ids, values, one, back)
    assert back.isnan().all(1).tolist() == [True, False, True]


# ---- streams, graphs, refusals -----------------------------------------------------


def test_other_streams_and_repeated_calls_give_the_same_bits():
    pkg = sym()
    for rows, vocab in ((1, 28672), (20, 4097)):
        x = normal_rows(rows, vocab, "bf16", 3).cuda()
        targets = torch.randint(0, vocab, (rows,), generator=gen(4)).cuda()
        op = pkg.TokenLogprobs(rows, vocab, torch.bfloat16, top=20)
        want = None
        side = torch.cuda.Stream()
        for i in range(4):
            for t in (op.logprob, op.entropy, op.stats, op.top_ids, op.top_logprobs):
                t.fill_(-1)
            if i % 2:
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    op.run(x, targets)
                torch.cuda.current_stream().wait_stream(side)
            else:
                op.run(x, targets)
            got = [t.clone() for t in (op.logprob, op.entropy, op.stats, op.top_ids, op.top_logprobs)]
            want = want or got
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows,vocab", [(2, 28672), (50, 1000), (3, 131072)])
def test_graph_replays(rows, vocab):
    pkg = sym()
    x = normal_rows(rows, vocab, "bf16", 3).cuda()
    targets = torch.randint(0, vocab, (rows,), generator=gen(4)).cuda()
    g = torch.ones(rows, device="cuda")
    op = pkg.TokenLogprobs(rows, vocab, torch.bfloat16, top=9)
    kd = pkg.TopDistillation(rows, vocab, torch.bfloat16, 9)
    dl, dk = torch.empty_like(x), torch.empty_like(x)

    def calls():
        op.run(x, targets, dl, g, g, g)
        kd.run(x, op.top_ids, op.top_logprobs, g, dk)

    outs = (op.logprob, op.entropy, op.top_ids, op.top_logprobs, dl, kd.loss, dk)
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        x.copy_(normal_rows(rows, vocab, "bf16", 30 + i))      # the program's own work between replays
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), i


def test_python_refusals():
    pkg = sym()
    x = torch.zeros((4, 100), dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    op = pkg.TokenLogprobs(4, 100, torch.bfloat16)
    for bad, err in ((x.float(), TypeError), (x[:3], ValueError), (x.cpu(), ValueError),
                     (x.t().contiguous().t(), ValueError), (x[:1].expand(4, 100), ValueError)):
        with pytest.raises(err):
            op.run(bad, t)
    for bad, err in ((t.int(), TypeError), (t[:3], ValueError), (t.cpu(), ValueError)):
        with pytest.raises(err):
            op.run(x, bad)
    with pytest.raises(TypeError):
        op.run(x, t, x, t)
    with pytest.raises(pkg.SymtileError):
        op.run(x, t, None, torch.ones(4, device="cuda"))          # gradients without dlogits
    with pytest.raises(TypeError):
        pkg.TokenLogprobs(4, 100, torch.float64)
    with pytest.raises(pkg.SymtileError):
        pkg.TokenLogprobs(4, 100, torch.bfloat16, top=101)
    with pytest.raises(pkg.SymtileError):
        pkg.TokenLogprobs(4, 100, torch.bfloat16, scale=0.0).run(x, t)
    kd = pkg.TopDistillation(4, 100, torch.bfloat16, 3)
    ids, values = torch.zeros((4, 3), dtype=torch.int64, device="cuda"), torch.zeros((4, 3), device="cuda")
    for a, b, err in ((ids.int(), values, TypeError), (ids[:, :2], values, ValueError),
                      (ids, values.double(), TypeError), (ids, values[:, :2], ValueError)):
        with pytest.raises(err):
            kd.run(x, a, b)
    mem = torch.zeros((8, 100), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pkg.SymtileError) as e:
        kd.run(mem[:4], ids, values, torch.ones(4, device="cuda"), mem[2:6])
    assert "overlaps" in str(e.value)
    with pytest.raises(pkg.SymtileError) as e:
        pkg.symtile_token_logprobs(99, x.data_ptr(), 4, 100, 0, pkg.BF16, 1.0, t.data_ptr(),
                                   op.logprob.data_ptr(), 0, 0)
    assert "device" in str(e.value)


def test_zero_rows():
    pkg = sym()
    op = pkg.TokenLogprobs(0, 100, torch.bfloat16, top=3)
    op.run(torch.empty((0, 100), dtype=torch.bfloat16, device="cuda"),
           torch.empty(0, dtype=torch.int64, device="cuda"))
    assert op.logprob.numel() == 0


# ---- large finite masks ------------------------------------------------------------

MASKS = [-1e8, -1e9, -1e10, -1e12, -1e20, -1e29, 1e10]


def masked_rows(vocab, dtype, mask, seed):
    """Rows of the mask alone, with its last third masked (the last segment of a row that is
    split, the first one's where it is the largest), with one token left, and without it."""
    x = normal_rows(4, vocab, dtype, seed).float()
    x[0] = mask
    x[1, vocab - vocab // 3:] = mask
    one = x[2, vocab // 2].clone()
    x[2] = mask
    x[2, vocab // 2] = one
    return x.to(TD[dtype])


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype,vocab", [("bf16", 1000), ("f32", 1001), ("bf16", 131072), ("f32", 70001)])
def test_rows_with_large_finite_masks(dtype, vocab, mask):
    pkg = sym()
    x = masked_rows(vocab, dtype, mask, 3)
    targets = torch.tensor([7, 11, vocab // 2, vocab - 1])
    g = [torch.randn((4,), generator=gen(k)) for k in range(3)]
    for scale in (1.0, np.float32(0.7).item(), 2.0):
        op = pkg.TokenLogprobs(4, vocab, TD[dtype], top=9, scale=scale)
        op.run(x.cuda(), targets.cuda())
        check_logprobs(op, x, targets, scale, 9)
        dl = torch.full((4, vocab), 5.0, dtype=TD[dtype], device="cuda")
        op.backward(x.cuda(), targets.cuda(), dl, *[t.cuda() for t in g])
        check_logprob_grad(dl, x, targets, scale, g, dtype)
        dl.fill_(5.0)
        op.run(x.cuda(), targets.cuda(), dl, *[t.cuda() for t in g])
        check_logprobs(op, x, targets, scale, 9)
        check_logprob_grad(dl, x, targets, scale, g, dtype)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype,vocab", [("bf16", 1000), ("f32", 1001), ("bf16", 131072), ("f32", 70001)])
def test_distillation_with_large_finite_masks(dtype, vocab, mask, rest):
    """As above, and with every token outside the list masked (the last row)."""
    pkg = sym()
    k = 16
    x = masked_rows(vocab, dtype, mask, 5)
    ids, values = teacher_list(x, k, 7, rest)
    ids = torch.where(ids < 0, torch.arange(k) * (vocab // k), ids)
    x = torch.cat([x, torch.full((1, vocab), mask).to(TD[dtype])])
    x[4, ids[3]] = normal_rows(1, k, dtype, 9)[0]
    ids, values = torch.cat([ids, ids[3:]]), torch.cat([values, values[3:]])
    g = torch.rand((5,), generator=gen(1)) + 0.5
    for scale in (1.0,) if rest else (1.0, np.float32(0.7).item(), 2.0):
        kd = pkg.TopDistillation(5, vocab, TD[dtype], k, scale=scale, rest=rest)
        kd.run(x.cuda(), ids.cuda(), values.cuda())
        check_distill(kd.loss, None, x, ids, values, scale, rest, g, dtype)
        back = torch.full((5, vocab), 5.0, dtype=TD[dtype], device="cuda")
        kd.backward(x.cuda(), ids.cuda(), values.cuda(), g.cuda(), back)
        check_distill(kd.loss, back, x, ids, values, scale, rest, g, dtype)
        back.fill_(5.0)
        kd.run(x.cuda(), ids.cuda(), values.cuda(), g.cuda(), back)
        check_distill(kd.loss, back, x, ids, values, scale, rest, g, dtype)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e30, 3e38])
def test_extreme_scales(scale):
    """Products of the scale that pass the range of fp32 either way."""
    pkg = sym()
    scale = np.float32(scale).item()
    x = torch.randn((3, 300), generator=gen(2)) * (1.0 if scale > 1 else 3e37)
    x[0] = 0.0
    x[1, 5:] = -1.0 if scale > 1 else -1e38
    targets = torch.tensor([3, 4, 5])
    op = pkg.TokenLogprobs(3, 300, torch.float32, top=5, scale=scale)
    op.run(x.cuda(), targets.cuda())
    check_logprobs(op, x, targets, scale, 5)
    ids, values = teacher_list(x, 5, 7, False)
    ids[2] = torch.arange(5)
    values = torch.zeros_like(values)
    kd = pkg.TopDistillation(3, 300, torch.float32, 5, scale=scale)
    kd.run(x.cuda(), ids.cuda(), values.cuda())
    check_distill(kd.loss, None, x, ids, values, scale, False, torch.ones(3), "f32")


# ---- workspaces --------------------------------------------------------------------


def c_logprobs(ws, x, targets, top, grad=None):
    """The C call on a workspace of the test's own; outputs filled with a pattern before."""
    pkg = sym()
    rows, vocab = x.shape
    new = lambda *s, dtype=torch.float32: torch.full(s, -7, dtype=dtype, device="cuda")  # noqa: E731
    out = [new(rows), new(rows), new(rows, 2), new(rows, top, dtype=torch.int64), new(rows, top)]
    dt = {torch.bfloat16: pkg.BF16, torch.float16: pkg.F16, torch.float32: pkg.F32}[x.dtype]
    pkg.symtile_token_logprobs(0, x.data_ptr(), rows, vocab, 0, dt, 1.0, targets.data_ptr(),
                               *[t.data_ptr() for t in out[:3]], top, out[3].data_ptr(),
                               out[4].data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel(),
                               stream=pkg.current_stream())

    class Outputs:
        logprob, entropy, stats, top_ids, top_logprobs = out
    return Outputs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_calls_of_all_sizes(dtype):
    """One row, many rows, other lengths, other operators, one after another."""
    pkg = sym()
    dt = {"bf16": pkg.BF16, "f32": pkg.F32}[dtype]
    sizes = [(1, 131072, 128), (128, 65544, 9), (1, 131072, 128), (300, 40000, 0), (2, 1 << 20, 100),
             (700, 33000, 3), (1, 131072, 0), (70, 131072, 1)]
    need = max(pkg.symtile_logits_workspace_bytes(0, r, v, dt, t) for r, v, t in sizes)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    for rows, vocab, top in sizes:
        x = normal_rows(rows, vocab, dtype, rows + vocab)
        targets = torch.randint(0, vocab, (rows,), generator=gen(1))
        got = c_logprobs(ws, x.cuda(), targets.cuda(), top)
        check_logprobs(got, x[:2], targets, 1.0, top) if rows < 3 else None
        own = pkg.TokenLogprobs(rows, vocab, TD[dtype], top=top)
        own.run(x.cuda(), targets.cuda())
        for name in ("logprob", "entropy", "stats", "top_ids", "top_logprobs"):
            assert torch.equal(getattr(got, name), getattr(own, name)), (rows, vocab, top, name)
        ids, values = torch.randint(0, vocab, (rows, 8), generator=gen(2)), torch.zeros(rows, 8)
        loss = torch.full((rows,), -7.0, device="cuda")
        dx, di, dv = x.cuda(), ids.cuda(), values.cuda()
        pkg.symtile_distill_topk(0, dx.data_ptr(), rows, vocab, 0, dt, 1.0, di.data_ptr(), dv.data_ptr(),
                                 pkg.F32, 8, pkg.DISTILL_RENORM, loss.data_ptr(), workspace=ws.data_ptr(),
                                 workspace_bytes=ws.numel(), stream=pkg.current_stream())
        kd = pkg.TopDistillation(rows, vocab, TD[dtype], 8)
        kd.run(dx, di, dv)
        assert torch.equal(loss, kd.loss), (rows, vocab)


def test_more_split_rows_than_counters():
    """Rows in several launches: every row is joined, and the counters end at zero."""
    pkg = sym()
    rows, vocab = 20001, 16400                     # fp32: 4100 vectors, two segments or more
    need = pkg.symtile_logits_workspace_bytes(0, rows, vocab, pkg.F32, 3)
    assert need > 0
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    row = torch.randn((vocab,), generator=gen(5))
    x = row.cuda().repeat(rows, 1)
    at = torch.arange(rows, device="cuda") % vocab
    x[torch.arange(rows, device="cuda"), at] = 9.0 + torch.arange(rows, device="cuda") / rows
    for _ in range(2):
        got = c_logprobs(ws, x, at, 3)
        assert torch.equal(got.top_ids[:, 0], at)
        want = torch.log_softmax(x[::997].double(), 1).gather(1, at[::997, None])[:, 0]
        assert float((got.logprob[::997].double() - want).abs().max()) < O.log_bound(row.numpy(), 1.0) + 64 * O.U
        assert bool((got.logprob == got.top_logprobs[:, 0]).all()) and bool((got.entropy > 0).all())


def test_the_first_call_on_another_stream():
    """stream= for the first call, right after the object was made while torch's current stream is
    busy and the memory of the workspace held other values before."""
    pkg = sym()
    rows, vocab = 3, 131072
    x = normal_rows(rows, vocab, "bf16", 3)
    targets = torch.randint(0, vocab, (rows,), generator=gen(4))
    ids, values = teacher_list(x, 9, 3, False)
    dx, dt, di, dv = x.cuda(), targets.cuda(), ids.cuda(), values.cuda()
    side = torch.cuda.Stream()
    for make in ("logprobs", "distill"):
        need = pkg.symtile_logits_workspace_bytes(0, rows, vocab, pkg.BF16, 9 if make == "logprobs" else 0)
        assert need > 0
        dirty = torch.full((need,), 3, dtype=torch.uint8, device="cuda")
        del dirty
        torch.cuda.synchronize()
        torch.cuda._sleep(200_000_000)
        if make == "logprobs":
            op = pkg.TokenLogprobs(rows, vocab, torch.bfloat16, top=9)
            op.run(dx, dt, stream=side.cuda_stream)
        else:
            op = pkg.TopDistillation(rows, vocab, torch.bfloat16, 9)
            op.run(dx, di, dv, stream=side.cuda_stream)
        torch.cuda.synchronize()
        if make == "logprobs":
            check_logprobs(op, x, targets, 1.0, 9)
        else:
            check_distill(op.loss, None, x, ids, values, 1.0, False, torch.ones(rows), "bf16")


def test_an_object_made_while_a_graph_is_captured():
    pkg = sym()
    x = normal_rows(2, 131072, "bf16", 3)
    dx, targets = x.cuda(), torch.tensor([5, 7])
    dt = targets.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op = pkg.TokenLogprobs(2, 131072, torch.bfloat16, top=3)
        op.run(dx, dt)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        check_logprobs(op, x, targets, 1.0, 3)


def test_a_device_that_does_not_exist_is_refused():
    """The size queries refuse it as the calls do, and leave nothing behind for the next call."""
    pkg = sym()
    for query in (lambda d: pkg.symtile_logits_workspace_bytes(d, 4, 131072, pkg.BF16, 5),
                  lambda d: pkg.symtile_w4_workspace_bytes(d, 64, 200, 8192, 64)):
        assert query(0) > 0
        for device in (99, -1):
            with pytest.raises(pkg.SymtileError) as e:
                query(device)
            assert e.value.name == "EINVAL" and "device" in str(e.value)
            x = normal_rows(2, 100, "bf16", 1)
            op = pkg.TokenLogprobs(2, 100, torch.bfloat16)
            op.run(x.cuda(), torch.zeros(2, dtype=torch.int64, device="cuda"))
            check_logprobs(op, x, [0, 0], 1.0, 0)
