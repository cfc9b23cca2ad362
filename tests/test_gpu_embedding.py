"""GPU tests of the embedding's lookup with All-Scatter (GatheredRows), bit by bit, and
of its gradient (EmbeddingGrad) against sums in 64 bits: n terms in fp32 are off by at
most n roundings of 2^-24 of the sum of magnitudes, then come a product and, when added
to what is held, a sum (2^-24 each), and half an ulp of the table's type."""
import math

import numpy as np
import pytest
import torch

from tests import ends_oracle as o
from tests.gpu_util import require_gpu, sym
from tests.head_oracle import half_ulp

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


def some_tokens(T, vocab, seed, hot=0.0):
    """Tokens of -1 .. vocab + 2 (padding, and ids that no shard holds), a share of them one."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(-1, vocab + 3, (T,), generator=g)
    return torch.where(torch.rand((T,), generator=g) < hot, vocab // 2, t)


LOOKUPS = [  # tokens, D, rows of a shard, world, scale
    (1, 8, 3, 1, 1.0), (1, 8192, 50, 8, 1.5), (15, 264, 20, 2, 0.5), (16, 1024, 33, 3, 11.3137), (17, 1032, 7, 4, -1.0),
    (64, 520, 100, 8, 2.0), (100, 72, 1, 2, 0.0), (333, 2056, 64, 2, 1.0), (1000, 128, 5000, 1, 0.1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", LOOKUPS, ids=lambda s: "t%d_d%d_v%d_w%d_%g" % s)
def test_lookup(shape, dtype):
    T, D, rows, world, scale = shape
    pkg = sym()
    g = torch.Generator().manual_seed(T + D)
    wide = torch.randn((world * rows, D + 8), generator=g).to(TD[dtype]).cuda()
    table = wide[:, :D]                                     # rows apart
    tokens = some_tokens(T, world * rows, T + D)
    heap = pkg.Heap(world, 2 * T * D * 4 + world * (T + 16) * (D // 256 + 2) * 4 + 8192)
    out = pkg.GatheredRows(heap, T, D, TD[dtype])
    esize = TD[dtype].itemsize
    assert out.arrived(0).shape == (world, -(-T // 16), -(-D * esize // 2048))
    bits = out.rows_all().view(torch.int16)
    bits.fill_(-1)
    dev = tokens.cuda()
    want = torch.full((T, D), -1, dtype=torch.int16).repeat(1, esize // 2)
    for r in range(world):
        out.run(dev, table[r * rows:(r + 1) * rows], r, scale=scale)
        heap.barrier()
        mine = (tokens >= r * rows) & (tokens < (r + 1) * rows)
        value = (table.cpu()[tokens[mine]].float() * torch.tensor(scale, dtype=torch.float32)).to(TD[dtype])
        want[mine] = value.view(torch.int16)
        if r == 0:
            want[tokens < 0] = 0
        for s in range(world):
            assert torch.equal(bits[s].cpu(), want), (r, s)
        counts = torch.zeros_like(out.arrived_all())
        counts[:, :r + 1] = 1
        assert torch.equal(out.arrived_all(), counts)
    out.run(dev, table[:rows], 0, scale=scale)              # a second call writes the same
    heap.barrier()
    assert torch.equal(bits[world - 1].cpu(), want)
    assert bool((out.arrived(0)[0] == 2).all())


def test_lookup_of_a_shard_anywhere():
    """Shards of different sizes by their first ids; an empty one counts its tiles."""
    pkg = sym()
    T, D = 40, 64
    heap = pkg.Heap(3, 1 << 20)
    out = pkg.GatheredRows(heap, T, D, torch.float32)
    table = torch.arange(10 * D, dtype=torch.float32, device="cuda").view(10, D)
    tokens = torch.arange(T, device="cuda") % 10
    for r, (a, b) in enumerate(((0, 3), (3, 3), (3, 10))):
        out.run(tokens, table[a:b], r, first=a)
    heap.barrier()
    assert torch.equal(out.rows(2), table[tokens])
    assert bool((out.arrived_all() == 1).all())
    far = torch.full((T,), 2 ** 62, device="cuda")
    out.run(far, table, 1, first=2 ** 62 - 4)
    heap.barrier()
    assert torch.equal(out.rows(0), table[4].expand(T, D))


def test_lookup_refusals():
    pkg = sym()
    heap = pkg.Heap(2, 1 << 20)
    out = pkg.GatheredRows(heap, 4, 64, torch.bfloat16)
    tokens = torch.zeros(4, dtype=torch.int64, device="cuda")
    table = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda")
    for bad in ((tokens[:3], table), (tokens, table[:, :32]), (tokens.cpu(), table), (tokens, table.t())):
        with pytest.raises(ValueError):
            out.run(*bad, 0)
    for bad in ((tokens.int(), table), (tokens, table.float())):
        with pytest.raises(TypeError):
            out.run(*bad, 0)
    for kw in ({"scale": math.inf}, {"scale": math.nan}, {"first": -1}):
        with pytest.raises(pkg.SymtileError) as e:
            out.run(tokens, table, 0, **kw)
        assert e.value.name == "EINVAL"
    with pytest.raises(pkg.SymtileError):
        out.run(tokens, table, 2)
    with pytest.raises(pkg.SymtileError):                   # rows not at multiples of 16 bytes
        out.run(tokens, torch.zeros((8, 68), dtype=torch.bfloat16, device="cuda")[:, 1:65], 0)
    with pytest.raises(pkg.SymtileError):
        pkg.GatheredRows(heap, 4, 12, torch.bfloat16).run(tokens, table[:, :12].contiguous(), 0)
    args = [heap.handle, tokens.data_ptr(), 4, table.data_ptr(), 8, 64, 0, pkg.BF16, 0, 1.0,
            heap.ptr(0, out.out_off), heap.ptr(0, out.flag_off), 0, 2]
    for i, bad in ((0, 0), (1, 0), (2, -1), (3, 0), (4, -1), (4, (1 << 21) + 1), (6, 32), (7, 9), (10, args[10] + 8),
                   (10, heap.ptr(1, out.out_off)), (11, args[10]), (11, args[11] + 2), (12, -1), (13, 3)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_embed_all_scatter(*args[:i], bad, *args[i + 1:])
        assert e.value.name == "EINVAL", i
    heap.barrier()
    assert not bool(out.arrived_all().any())
    pkg.GatheredRows(heap, 0, 64, torch.bfloat16).run(tokens[:0], table, 0)


# ---- gradient ------------------------------------------------------------------------------
def check_grad(got, held, tokens, d, first, rows, scale, accumulate, table):
    want, size, count = o.embedding_grad(tokens, d, first, rows, scale)
    n = count[:, None]
    tol = (n + 1) * 2.0 ** -24 * size
    if accumulate:
        h = held.double().numpy()
        want = want + h
        tol = tol + 2.0 ** -24 * (np.abs(want) + size)
    tol = tol + (half_ulp(np.abs(want) + tol, table) if table != "f32" else 2.0 ** -24 * np.abs(want) + 2.0 ** -149)
    g = got.double().cpu().numpy()
    err = np.abs(g - want)
    assert np.isfinite(g).all() and (err <= tol).all(), (float((err - tol).max()), int((err > tol).sum()))
    none = count == 0
    assert np.array_equal(g[none], held.double().numpy()[none] if accumulate else np.zeros_like(g[none]))


GRADS = [  # tokens, D, rows, first, scale, share of one token
    (1, 8, 1, 0, 1.0, 0.0), (2, 64, 5, 3, 2.0, 0.0), (31, 72, 4, 0, 0.5, 0.0), (32, 256, 1, 7, 1.0, 0.9),
    (33, 2048, 3, 0, 1.0, 0.5), (100, 2056, 1000, 50, 1.5, 0.0), (1000, 136, 300, 300, 45.25, 0.3),
    (2048, 520, 64, 0, 1.0, 0.0), (2049, 64, 100, 10, 1.0, 0.6), (5000, 32, 2000, 0, 1.0, 0.1),
    (9000, 16, 3, 1, 0.1, 0.97), (20000, 8, 30000, 0, 1.0, 0.0), (70000, 8, 40, 20, 1.0, 0.2),
    (65536, 8, 500, 0, 1.0, 0.0), (65537, 16, 256, 0, 1.0, 0.3), (66000, 8, 1, 1, 1.0, 0.5), (70000, 8, 100000, 5, 0.5, 0.1),
    (100001, 8, 30000, 0, 1.0, 0.01), (67000, 24, 2000000, 9, 1.0, 0.0),
    (600000, 8, 3000, 0, 1.0, 0.2)]


@pytest.mark.parametrize("types", [("bf16", "f32"), ("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16")],
                         ids="_".join)
@pytest.mark.parametrize("shape", GRADS, ids=lambda s: "t%d_d%d_v%d_f%d_%g_h%g" % s)
def test_gradient(shape, types):
    T, D, rows, first, scale, hot = shape
    dtype, table = types
    g = torch.Generator().manual_seed(T + D)
    tokens = some_tokens(T, first + rows + 2, T + rows, hot)
    d = torch.randn((T, D), generator=g).to(TD[dtype])
    held = torch.randn((rows, D), generator=g).to(TD[table])
    wide = torch.full((T, D + 8), math.nan, dtype=TD[dtype], device="cuda")
    wide[:, :D] = d
    op = sym().EmbeddingGrad(T, D, TD[dtype])
    if op.ws is not None:
        op.ws.fill_(0xFF)
    for accumulate in (False, True):
        to = torch.full((rows, D + 16), 3.0, dtype=TD[table], device="cuda")
        to[:, :D] = held.cuda() if accumulate else math.nan
        op.run(tokens.cuda(), wide[:, :D], to[:, :D], first, scale, accumulate)
        torch.cuda.synchronize()
        check_grad(to[:, :D], held, tokens, d.double(), first, rows, scale, accumulate, table)
        assert bool((to[:, D:] == 3).all())
        again = torch.full((rows, D), math.nan, dtype=TD[table], device="cuda")
        if accumulate:
            again.copy_(held)
        op.run(tokens.cuda(), d.cuda(), again, first, scale, accumulate)
        torch.cuda.synchronize()
        assert torch.equal(again, to[:, :D])                # to the last bit, whatever the strides


def test_gradient_against_differences():
    """The lookup is linear in its table: its change along a direction is the gradient's
    product with it."""
    pkg = sym()
    T, D, rows, scale = 50, 64, 9, 3.0
    g = torch.Generator().manual_seed(2)
    tokens = some_tokens(T, rows, 4).clamp(max=rows - 1).cuda()
    table, step, d = (torch.randint(-8, 9, s, generator=g).float().cuda() for s in ((rows, D), (rows, D), (T, D)))
    heap = pkg.Heap(1, 1 << 20)
    out = pkg.GatheredRows(heap, T, D, torch.float32)
    loss = []
    for t in (table - step, table + step):
        out.run(tokens, t, 0, scale=scale)
        heap.barrier()
        loss.append((out.rows(0).double() * d.double()).sum())
    grad = torch.empty((rows, D), device="cuda")
    pkg.EmbeddingGrad(T, D, torch.float32).run(tokens, d, grad, scale=scale)
    torch.cuda.synchronize()
    assert float((loss[1] - loss[0]) / 2) == float((grad.double() * step.double()).sum())


def test_whole_numbers_are_exact():
    T, D, rows = 6000, 64, 50
    g = torch.Generator().manual_seed(3)
    tokens = some_tokens(T, rows, 1, 0.4)
    d = torch.randint(-4, 5, (T, D), generator=g).float()
    got = torch.empty((rows, D), device="cuda")
    sym().EmbeddingGrad(T, D, torch.bfloat16).run(tokens.cuda(), d.bfloat16().cuda(), got, 0, 0.5)
    torch.cuda.synchronize()
    assert np.array_equal(got.cpu().numpy(), o.embedding_grad(tokens, d, 0, rows, 0.5)[0])


def test_the_longest_table():
    """Ids up to the largest allowed, present and absent ones side by side."""
    rows, D, T = 1 << 21, 8, 4096
    g = torch.Generator().manual_seed(0)
    tokens = torch.cat([torch.full((T // 2,), rows - 1), torch.randint(rows - 5, rows + 2, (T // 2,), generator=g)])
    d = torch.randint(-4, 5, (T, D), generator=g).float()
    for n in (T, 2048, 100):
        got = torch.empty((rows, D), device="cuda", dtype=torch.bfloat16)
        sym().EmbeddingGrad(n, D, torch.float32).run(tokens[-n:].cuda(), d[-n:].cuda(), got)
        torch.cuda.synchronize()
        assert not bool(got[:rows - 5].any())
        want = o.embedding_grad(tokens[-n:], d[-n:], rows - 5, 5, 1.0)[0]
        assert torch.equal(got[rows - 5:].cpu(), torch.from_numpy(want).bfloat16())


def test_gradient_captured_and_on_another_stream():
    """Replays on new tokens, among eager calls of the same object."""
    for T in (500, 5000, 66000):
        D, rows = 128, 40
        g = torch.Generator().manual_seed(T)
        op = sym().EmbeddingGrad(T, D, torch.float32)
        cases = [(some_tokens(T, rows, s, 0.2 * s), torch.randn((T, D), generator=g)) for s in range(3)]
        tokens, d = cases[0][0].cuda(), cases[0][1].cuda()
        got = torch.empty((rows, D), device="cuda")
        op.run(tokens, d, got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            op.run(tokens, d, got)
        for i in range(5):
            t, x = cases[i % 3]
            tokens.copy_(t)
            d.copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            check_grad(got, None, t, x.double(), 0, rows, 1.0, False, "f32")
            if i == 1:
                s = torch.cuda.Stream()
                got.fill_(math.nan)
                s.wait_stream(torch.cuda.current_stream())
                op.run(tokens, d, got, stream=s.cuda_stream)
                s.synchronize()
                check_grad(got, None, t, x.double(), 0, rows, 1.0, False, "f32")


def test_gradient_refusals():
    pkg = sym()
    T, D = 10, 64
    op = pkg.EmbeddingGrad(T, D, torch.float32)
    tokens = torch.zeros(T, dtype=torch.int64, device="cuda")
    d, table = torch.ones((T, D), device="cuda"), torch.full((5, D), 2.0, device="cuda")
    for bad in ((tokens[:5], d, table), (tokens, d[:5], table), (tokens, d, table[:, :32]), (tokens, d, table[0]),
                (tokens, d, table.cpu()), (tokens, d.t().contiguous().t(), table)):
        with pytest.raises(ValueError):
            op.run(*bad)
    for bad in ((tokens.int(), d, table), (tokens, d.half(), table), (tokens, d, table.double())):
        with pytest.raises(TypeError):
            op.run(*bad)
    for kw in ({"first": -1}, {"scale": math.nan}):
        with pytest.raises(pkg.SymtileError) as e:
            op.run(tokens, d, table, **kw)
        assert e.value.name == "EINVAL"
    with pytest.raises(pkg.SymtileError) as e:
        op.run(tokens, d, d[:4])                            # the table inside the rows
    assert e.value.name == "EINVAL"
    with pytest.raises(pkg.SymtileError):
        op.run(tokens, torch.ones((T, D + 2), device="cuda")[:, :D], table)
    for bad in ((0, -1, D), (0, T, 12), (0, 1 << 25, D), (99, T, D)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_embed_workspace_bytes(*bad)
        assert e.value.name == "EINVAL", bad
    need = pkg.symtile_embed_workspace_bytes(0, T, D)
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    args = [0, tokens.data_ptr(), T, d.data_ptr(), D, 0, pkg.F32, 0, 5, 1.0, table.data_ptr(), 0, pkg.F32, 0]
    for at, n in ((0, need - 1), (8, need)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_embed_backward(*args, ws.data_ptr() + at, n)
        assert e.value.name == "EINVAL"
    torch.cuda.synchronize()
    assert bool((table == 2).all())
    # no tokens: the table is zeroed, or left alone
    none = pkg.EmbeddingGrad(0, D, torch.float32)
    none.run(tokens[:0], d[:0], table, accumulate=True)
    torch.cuda.synchronize()
    assert bool((table == 2).all())
    none.run(tokens[:0], d[:0], table)
    torch.cuda.synchronize()
    assert not bool(table.any())
