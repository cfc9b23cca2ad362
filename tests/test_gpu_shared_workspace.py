"""GPU test of one workspace that calls of several operators use in turn: each finds its
counters at zero and leaves them so, whatever ran before."""
import pytest
import torch

from tests.gpu_util import require_gpu, sym

pytestmark = pytest.mark.gpu


def test_operators_in_turn():
    require_gpu()
    pkg = sym()
    g = torch.Generator().manual_seed(3)
    bf = torch.bfloat16
    steps = []

    def step(name, need, swap, run, results):
        """`run` with the operator's own workspace, then its results are what all later runs give."""
        run()
        torch.cuda.synchronize()
        steps.append((name, need, swap, run, results, [r.clone() for r in results]))
        assert need > 65536, name

    S, k, V = 2, 3, 50001
    x = (torch.randn((S * (k + 1), V), generator=g) * 2).to(bf).cuda()
    y = (torch.randn((S * k, V), generator=g) * 2).to(bf).cuda()
    ids = torch.randint(0, V, (S, k), generator=g).cuda()
    u = torch.rand((S, k), generator=g).cuda()
    e = (-torch.log1p(-torch.rand((S, V), generator=g))).clamp(min=1e-20).cuda()
    dv = pkg.DraftVerification(S, k, V, bf)
    step("verify", dv.ws.numel(),
         lambda at, n: setattr(dv, "_out", (*dv._out[:3], at, n)), lambda: dv.run(x, ids, u, e, y),
         [dv.tokens, dv.accepted, dv.logprob])

    rows, vocab = 3, 140001
    logits = torch.randn((rows, vocab), generator=g).to(bf).cuda()
    lp = pkg.TokenLogprobs(rows, vocab, bf, top=5)
    step("logprobs", lp.ws.numel(), lambda at, n: setattr(lp, "_ws", (at, n)),
         lambda: lp.run(logits, torch.arange(rows, device="cuda")), [lp.logprob, lp.top_ids, lp.top_logprobs])

    M, K, N = 64, 8192, 64
    heap = pkg.Heap(2, 1 << 20)
    out = pkg.GatheredOutput(heap, M, N, bf, pkg.MX4_TILE_M, pkg.MX4_TILE_N)
    a, w = pkg.MX4Matrix.empty(M, K), pkg.MX4Matrix.empty(N, K)
    a.quantise(torch.randn((M, K), generator=g).cuda())
    w.quantise(torch.randn((N, K), generator=g).cuda())

    def product(at, n):
        out.ws_mx4[K] = shared
    step("product", pkg.symtile_mx4_workspace_bytes(0, M, N, K), product, lambda: out.run_mx4(a, w, 1),
         [out.C(0), out.C(1)])

    few = pkg.GatheredOutput(heap, 24, N, bf, pkg.W4_TILE_M, pkg.W4_TILE_N)
    xw = torch.randn((24, K), generator=g).to(bf).cuda()
    w4 = pkg.W4Weight(torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8).cuda(),
                      torch.rand((N, K // 128), generator=g).to(bf).cuda())

    def integers(at, n):
        few.ws_w4[K, 128] = shared
    step("integer weights", pkg.symtile_w4_workspace_bytes(0, 24, N, K, 128), integers,
         lambda: few.run_w4(xw, w4, 0), [few.C(0), few.C(1)])

    for T in (500, 5000, 70000):
        D, shard = 64, 300
        tokens = torch.randint(0, 2 * shard, (T,), generator=g).cuda()
        d = torch.randn((T, D), generator=g).cuda()
        op, table = pkg.EmbeddingGrad(T, D, torch.float32), torch.empty((shard, D), device="cuda")
        step(f"gradient of {T}", op.ws.numel(), lambda at, n, op=op: setattr(op, "_ws", (at, n)),
             lambda op=op, t=tokens, d=d, table=table: op.run(t, d, table, first=shard), [table])

    shared = torch.zeros(max(s[1] for s in steps), dtype=torch.uint8, device="cuda")
    shared[65536:] = 0xFF            # (what lies behind the counters may be anything)
    for _, need, swap, *_ in steps:
        swap(shared.data_ptr(), shared.numel())
    order = [0, 4, 1, 5, 3, 6, 2, 5, 0, 2, 4, 0, 3, 4, 1, 6, 2, 5, 0, 6, 3]
    for i in order:
        name, _, _, run, results, want = steps[i]
        for r in results:
            r.zero_()
        run()
        torch.cuda.synchronize()
        assert not bool(shared[:65536].any()), name
        for r, v in zip(results, want):
            assert torch.equal(r, v), name
    heap.close()
