"""GPU test of a model's two ends run together, as a step of speculative decoding and of
training would: drafted tokens' rows from the sharded table, hidden states in 4-bit
blocks times every rank's shard of the head, the gathered logits verified, and the
gradient of the table by the tokens that came out; eagerly and replayed from a graph."""
import numpy as np
import pytest
import torch

from tests import ends_oracle as o
from tests.gpu_util import require_gpu, sym
from tests.test_gpu_verify import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("world,S,k,D,shard", [(2, 3, 2, 256, 264), (8, 8, 4, 1024, 512)])
def test_a_step(world, S, k, D, shard):
    require_gpu()
    pkg = sym()
    dt, M, V = torch.bfloat16, S * (k + 1), world * shard
    g = torch.Generator().manual_seed(world)
    table = (torch.randn((V, D), generator=g) * 0.5).to(dt)
    tokens = torch.randint(0, V, (M,), generator=g)
    scale = 2.0
    heap = pkg.Heap(world, M * D * 2 + M * V * 2 + world * 8 * V + (1 << 20))
    rows = pkg.GatheredRows(heap, M, D, dt)
    out = pkg.GatheredOutput(heap, M, shard, dt, pkg.MX4_TILE_M, pkg.MX4_TILE_N)
    x4 = pkg.MX4Matrix.empty(M, D)
    dev = [table[r * shard:(r + 1) * shard].cuda() for r in range(world)]
    w4 = [pkg.MX4Matrix.empty(shard, D) for _ in range(world)]
    for r in range(world):
        w4[r].quantise(dev[r])
    op = pkg.DraftVerification(S, k, V, dt, scale=0.3)
    grads = pkg.EmbeddingGrad(M, D, dt)
    dtable = torch.empty((shard, D), device="cuda")
    ids = torch.where(torch.rand((S, k), generator=g) < 0.8, tokens.view(S, k + 1)[:, 1:], -1)
    u = torch.rand((S, k), generator=g) * 0.2
    e = (-torch.log1p(-torch.rand((S, V), generator=g))).clamp(min=1e-20)
    d_tokens, d_ids, d_u, d_e = tokens.cuda(), ids.cuda(), u.cuda(), e.cuda()

    def step():
        for r in range(world):
            rows.run(d_tokens, dev[r], r, scale=scale)
        # (any slot holds all rows, and all logits)
        x4.quantise(rows.rows(world - 1))
        for r in range(world):
            out.run_mx4(x4, w4[r], r)
        op.run(out.C(0), d_ids, d_u, d_e)
        grads.run(op.tokens.view(-1), rows.rows(0), dtable, first=shard)

    def compare(calls):
        heap.barrier()
        assert bool((rows.arrived_all() == calls).all()) and bool((out.arrived_all() == calls).all())
        x = (table[tokens].float() * scale).to(dt)
        for s in range(world):
            assert torch.equal(rows.rows(s).cpu(), x)
        xq, xs = o.mx4_quantise(x.double().numpy())
        assert np.array_equal(x4.q.cpu().numpy(), xq) and np.array_equal(x4.scales.cpu().numpy(), xs)
        xv = o.mx4_values(xq, xs)
        wv = o.mx4_values(*o.mx4_quantise(table.double().numpy()))
        want, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
        got = out.C(0).double().cpu().numpy()
        assert (np.abs(got - want) <= (D / 32 + 64) * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(want) + 1e-30).all()
        check(S, k, op, out.C(0).cpu(), ids, u, e, None, 0.3, 1.0)
        g_want, g_size, n = o.embedding_grad(op.tokens.view(-1).cpu(), x.double(), shard, shard, 1.0)
        assert (np.abs(dtable.double().cpu().numpy() - g_want) <= (n[:, None] + 1) * 2.0 ** -24 * g_size).all()

    step()
    compare(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        d_tokens.copy_(tokens)
        graph.replay()
        torch.cuda.synchronize()
        compare(2 + i)
    heap.close()
