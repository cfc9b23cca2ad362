"""GPU tests of the operators at a model's two ends where addresses pass 32 bits and where one
call takes several launches: the first and last rows against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import ends_oracle as o
from tests.gpu_util import require_gpu, sym
from tests.test_gpu_verify import check as check_verify

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def ends(n):
    return torch.cat([torch.arange(5), torch.arange(n - 5, n)]).cuda()


def test_quantise_and_product():
    """4.4 GB of elements a matrix; the weights of few columns.  Whole numbers: exact."""
    pkg = sym()
    M, K, N = 270000, 32768, 24
    g = torch.Generator(device="cuda").manual_seed(1)
    x4 = pkg.MX4Matrix.empty(M, K)
    x4.q.zero_()
    x4.scales.fill_(127)
    at = ends(M)
    # 17.7 GB of 16 bits, zero but for the ends
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    x[at] = torch.randint(-6, 7, (10, K), generator=g, device="cuda").to(torch.bfloat16)
    x[at, ::32] = 4.0                                     # every block's scale is 1
    x4.quantise(x)
    q, scales = o.mx4_quantise(x[at].double().cpu().numpy())
    assert np.array_equal(x4.q[at].cpu().numpy(), q) and np.array_equal(x4.scales[at].cpu().numpy(), scales)
    del x
    w = pkg.MX4Matrix.empty(N, K)
    wf = torch.zeros((N, K), device="cuda")
    wf[:, :64] = torch.randint(-1, 2, (N, 64), generator=g, device="cuda").float()
    wf[:, -64:] = torch.randint(-1, 2, (N, 64), generator=g, device="cuda").float()
    w.quantise(wf)
    heap = pkg.Heap(1, M * N * 2 + (M // 64 + 1) * 2 * 4 + 8192)
    out = pkg.GatheredOutput(heap, M, N, torch.float16, pkg.MX4_TILE_M, pkg.MX4_TILE_N)
    out.run_mx4(x4, w, 0)
    heap.barrier()
    want = o.mx4_values(q, scales) @ wf.double().cpu().numpy().T
    assert np.abs(want).max() < 2048 and np.array_equal(out.C(0)[at].double().cpu().numpy(), want)
    assert bool((out.arrived(0) == 1).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_verification(dtype):
    """4.3 GB of logits of each kind in 32 bits, 2.1 of noise."""
    pkg = sym()
    S, k, V = 4096, 1, 131072 + 8
    g = torch.Generator(device="cuda").manual_seed(2)
    op = pkg.DraftVerification(S, k, V, dtype)
    x = torch.empty((S * (k + 1), V), dtype=dtype, device="cuda").normal_(0, 2.5, generator=g)
    y = x.view(S, 2, V)[:, 0].contiguous()
    y[:, ::3] += 0.5
    ids = torch.randint(0, V, (S, k), generator=g, device="cuda")
    ids[::2] = y[::2].argmax(1, keepdim=True)
    u = torch.rand((S, k), generator=g, device="cuda")
    e = torch.empty((S, V), device="cuda").exponential_(generator=g).clamp_(min=1e-20)
    op.run(x, ids, u, e, y)
    torch.cuda.synchronize()
    few = torch.tensor([0, 1, 2, S - 3, S - 2, S - 1])
    part = type("Outputs", (), {n: getattr(op, n)[few.cuda()] for n in ("tokens", "accepted", "logprob")})
    rows = (2 * few[:, None] + torch.arange(2)).flatten().cuda()
    f = few.cuda()
    check_verify(len(few), k, part, x[rows].cpu(), ids[f].cpu(), u[f].cpu(), e[f].cpu(), y[f].cpu(), 1.0, 1.0, 3)


def test_many_sequences_of_long_drafts():
    """More rows than one launch takes."""
    from tests.test_gpu_verify import call, inputs
    S, k, V = 600, 32, 90
    for mode in ("draft", "tokens", "greedy"):
        call(S, k, V, "f32", inputs(S, k, V, "f32", 3, mode), mode)


def test_embedding():
    """A table and rows of more than 4 GB each, and their gradient into 8."""
    pkg = sym()
    T, D, rows = 140000, 16384, 140000
    g = torch.Generator(device="cuda").manual_seed(4)
    table = torch.empty((rows, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    tokens = torch.randint(0, rows, (T,), generator=g, device="cuda")
    tokens[-1], tokens[0] = rows - 1, 0
    heap = pkg.Heap(1, T * D * 2 + (T // 16 + 1) * (D // 1024) * 4 + 8192)
    out = pkg.GatheredRows(heap, T, D, torch.bfloat16)
    out.run(tokens, table, 0)
    heap.barrier()
    got = out.rows(0)
    for t0 in range(0, T, 20000):
        assert torch.equal(got[t0:t0 + 20000], table[tokens[t0:t0 + 20000]])
    assert bool((out.arrived(0) == 1).all())
    del table
    # the gradient of the rows that were looked up, by themselves
    grad = pkg.EmbeddingGrad(T, D, torch.bfloat16)
    dtable = torch.full((rows, D), math.nan, device="cuda")
    grad.run(tokens, got, dtable, scale=0.5)
    counts = torch.bincount(tokens, minlength=rows)
    of = torch.zeros((rows,), dtype=torch.int64, device="cuda").scatter_(0, tokens, torch.arange(T, device="cuda"))
    for v0 in range(0, rows, 20000):
        n = counts[v0:v0 + 20000, None]
        row = got[of[v0:v0 + 20000]].float() * (0.5 * n)
        # n equal terms: n roundings of 2^-24 of their sum at most, and the product's
        err = (dtable[v0:v0 + 20000] - row).abs() - row.abs() * (n + 2) * 2.0 ** -24
        assert bool((torch.where(n > 0, err, dtable[v0:v0 + 20000].abs()) <= 0).all())
