"""GPU tests of the verification of drafted tokens where a decision or a draw hangs on one
number: drafted ids outside the vocabulary, rows whose largest logits are far apart, logits
whose difference is no fp32 number, residuals that leave nothing."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import require_gpu, sym
from tests.test_gpu_verify import TD, call, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 28672, 50001])
def test_drafted_ids_far_outside_the_vocabulary(V, dtype):
    """Such an id has p = 0 and takes nothing from p: the token that its lowest 32 bits name,
    which has nearly all of the probability, is drawn."""
    S, k = 5, 2
    v = torch.tensor([0, V // 3, V - 1, V // 2, 7])
    x = torch.zeros((S, k + 1, V))
    x[torch.arange(S), :, v] = 30.0
    high = torch.tensor([2 ** 32, 2 ** 40, 2 ** 62, 2 ** 32 * 5, 2 ** 33])
    ids = torch.stack([high + v, v], 1)
    u = torch.zeros((S, k))
    e = 0.5 + torch.rand((S, V), generator=torch.Generator().manual_seed(V))
    op = call(S, k, V, dtype, (x.view(-1, V).to(TD[dtype]), ids, u, e, None), "tokens", least=S)
    assert op.accepted.tolist() == [0] * S
    assert op.tokens[:, 0].cpu().tolist() == v.tolist()


@pytest.mark.parametrize("V", [3, 28672])
@pytest.mark.parametrize("at", [(2476475.5, 3000000.0), (3000000.0, 1913162.75)], ids=["target_below", "draft_below"])
def test_rows_on_both_sides_of_the_exponents_forms(at, V):
    """Exponentials are taken of rounded products up to a size of the largest logit and of
    differences beyond it.  With one row on each side p - q has the same scale for both: token
    1, with p = 0.404 and q = 0.419, has no residual, though its noise is the smallest."""
    S, k = 2, 1
    tokens = [0, V // 2, V - 1]
    x = torch.full((S, k + 1, V), -math.inf)
    y = torch.full((S, k, V), -math.inf)
    x[:, :, tokens] = at[0] + torch.tensor([0.0, 0.0, -0.75])
    y[:, :, tokens] = at[1] + torch.tensor([-0.25, 0.0, -0.5])
    ids = torch.full((S, k), tokens[1])
    u = torch.full((S, k), 0.9999)
    e = torch.ones((S, V))
    e[:, tokens[1]] = 0.01
    op = call(S, k, V, "f32", (x.view(-1, V), ids, u, e, y.view(-1, V)), "draft", least=S)
    assert op.accepted.tolist() == [0] * S
    assert op.tokens[:, 0].tolist() == [0] * S


@pytest.mark.parametrize("mode", ["draft", "tokens"])
def test_decisions_are_made_in_64_bits(mode):
    """Two logits whose difference is no fp32 number, and a u between p (or p / q) as it is and
    as the rounded difference would have it.  The largest logit's probability is 1 in fp32, the
    sum that the decision takes."""
    S, V, scale = 256, 2, np.float32(0.05)
    g = np.random.default_rng(5)
    m = g.uniform(500.0, 1000.0, S).astype(np.float32)
    d = (-g.uniform(1e-3, 500.0, S)).astype(np.float32)
    exact = np.exp((d.astype(np.float64) - m.astype(np.float64)) * np.float64(scale))
    rounded = np.exp((d - m).astype(np.float64) * np.float64(scale))
    x = torch.zeros((S, 2, V))
    y = torch.zeros((S, 1, V))
    if mode == "tokens":
        x[:, 0, 0], x[:, 0, 1] = torch.from_numpy(m), torch.from_numpy(d)
        border, other = exact, rounded
    else:
        # p of an exact difference, a little below q
        t = np.floor((d.astype(np.float64) - m) * 16) / 16 - 2
        p = np.exp(t * np.float64(scale))
        x[:, 0, 1] = torch.from_numpy(t.astype(np.float32))
        y[:, 0, 0], y[:, 0, 1] = torch.from_numpy(m), torch.from_numpy(d)
        border, other = p / exact, p / rounded
    u = ((border + other) / 2).astype(np.float32)
    want = u.astype(np.float64) < border
    tells = (u.astype(np.float64) < other) != want
    # (half of a difference's last place, some 0.00003, times the scale is 25 times u's; where u
    # comes next to the border itself the device's exponential and numpy's may differ)
    tells &= np.abs(u.astype(np.float64) / border - 1) > 1e-9
    assert tells.sum() > S // 2 and 0 < want[tells].sum() < tells.sum()
    ids = torch.ones((S, 1), dtype=torch.int64)
    op = sym().DraftVerification(S, 1, V, torch.float32, float(scale), float(scale))
    op.run(x.view(-1, V).cuda(), ids.cuda(), torch.from_numpy(u)[:, None].cuda(),
           torch.ones((S, V), device="cuda"), y.view(-1, V).cuda() if mode == "draft" else None)
    torch.cuda.synchronize()
    got = op.accepted.cpu().numpy() == 1
    assert (got == want)[tells].all(), int((got != want)[tells].sum())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,V", [(1, 28672), (4, 50001), (2, 2097147)])
def test_nothing_of_the_residual_is_left(S, V, dtype):
    """Where the draft is the target the token is drawn from p, over the whole of a row that
    several workgroups take; without the draft's logits where the drafted token is the only one."""
    k = 2
    x, _, _, e, _ = inputs(S, k, V, dtype, V, short=False)
    y = x.view(S, k + 1, V)[:, :k].reshape(-1, V)
    ids = torch.randint(0, V, (S, k), generator=torch.Generator().manual_seed(V))
    u = torch.full((S, k), 2.0)
    op = call(S, k, V, dtype, (x, ids, u, e, y), "draft", least=0)
    assert op.accepted.tolist() == [0] * S
    lp = torch.log_softmax(x.view(S, k + 1, V)[:, 0].double(), 1)
    score, order = (lp - e.double().log()).sort(1, descending=True)
    assert bool((score[:, 0] - score[:, 1] > 1e-4).all())
    assert op.tokens[:, 0].cpu().tolist() == order[:, 0].tolist()
    alone = torch.full((S * (k + 1), V), -math.inf)
    alone.view(S, k + 1, V)[torch.arange(S), :, ids[:, 0]] = 3.0
    op = call(S, k, V, dtype, (alone.to(TD[dtype]), ids, u, e, None), "tokens", least=0)
    assert op.accepted.tolist() == [0] * S
    assert op.tokens[:, 0].cpu().tolist() == ids[:, 0].tolist()


@pytest.mark.parametrize("mode", ["draft", "tokens", "greedy"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_drafts_over_rows_in_many_segments(dtype, mode):
    S, k, V = 3, 2, 140001
    t = inputs(S, k, V, dtype, 8, mode, short=False)
    assert bool((t[1] >= 0).all())
    call(S, k, V, dtype, t, mode)
