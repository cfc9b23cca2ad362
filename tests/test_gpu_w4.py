"""GPU tests of the 4-bit product with All-Scatter (GatheredOutput.run_w4) against
the definition in 64 bits.

Whole-number inputs are exact in fp32 whatever the order and must come back as
the exact sum rounded once; placement and counters are compared exactly.  For
other inputs the bound is half an output ulp plus the walk of K fp32 roundings:
each is at most 2^-24 of a partial sum, partial sums of weights up to 144 apart
from their zero point (128 + 15, and the zero point's own term) over a group of at
most 128 stay near 12 * 144 * max|x| * max scale, and K independent roundings add
up to sqrt(K) of them; 8 such deviations."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import require_gpu, sym
from tests.head_oracle import half_ulp

pytestmark = pytest.mark.gpu

TD = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def inputs(M, K, N, dtype, group, zeros, seed, whole=False):
    g = gen(seed)
    G = -(-K // group)
    q = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (N, G), generator=g, dtype=torch.uint8) if zeros else None
    if whole:
        X = torch.randint(-2, 3, (M, K), generator=g).to(TD[dtype])
        s = torch.tensor([0.25, 0.5, 1.0])[torch.randint(0, 3, (N, G), generator=g)].to(TD[dtype])
    else:
        X = torch.randn((M, K), generator=g).to(TD[dtype])
        s = ((torch.rand((N, G), generator=g) + 0.5) * 0.2 / math.sqrt(max(K, 1))).to(TD[dtype])
    return X, q, s, z


def expected(X, q, s, z, group):
    """[M, N] in 64 bits, weight by weight as the layout says."""
    qn = q.numpy()
    N, K = qn.shape[0], 2 * qn.shape[1]
    w = np.empty((N, K))
    w[:, 0::2], w[:, 1::2] = qn & 15, qn >> 4
    zn = np.full(tuple(s.shape), 8.0) if z is None else (z.numpy() & 15).astype(np.float64)
    at = np.arange(K) // group
    w = (w - zn[:, at]) * s.double().numpy()[:, at] if K else w
    return X.double().numpy() @ w.T


class Call:
    def __init__(self, M, N, world, dtype, tensors, group, ldx_pad=0):
        pkg = sym()
        self.tiles = -(-N // 16)
        self.heap = pkg.Heap(world, M * world * N * 2 + world * self.tiles * 4 + 8192)
        self.out = pkg.GatheredOutput(self.heap, M, N, TD[dtype], pkg.W4_TILE_M, pkg.W4_TILE_N)
        X, q, s, z = tensors
        wide = torch.full((M, X.shape[1] + ldx_pad), math.nan, dtype=TD[dtype], device="cuda")
        self.X = wide[:, :X.shape[1]]
        self.X.copy_(X)
        self.w = pkg.W4Weight(q.cuda(), s.cuda(), None if z is None else z.cuda(), group)
        self.out.C_all().view(torch.int16).fill_(-1)

    def run(self, rank, **kw):
        self.out.run_w4(self.X, self.w, rank, **kw)

    def check(self, rank, want, dtype, bound, calls=1):
        w, N, M = self.heap.world, self.out.N_local, self.out.M
        self.heap.barrier()
        C = self.out.C_all()
        for s in range(1, w):
            assert torch.equal(C[s].view(torch.int16), C[0].view(torch.int16)), s
        bits = C[0].view(torch.int16)
        for r in range(w):
            if r != rank:
                assert bool((bits[:, r * N:(r + 1) * N] == -1).all()), f"block of rank {r} written"
        got = C[0][:, rank * N:(rank + 1) * N].double().cpu().numpy()
        if bound is None:
            assert np.array_equal(got, torch.from_numpy(want).to(TD[dtype]).double().numpy())
        else:
            err = np.abs(got - want)
            tol = bound + half_ulp(np.abs(want) + bound, dtype)
            assert np.isfinite(got).all() and (err <= tol).all(), (float((err - tol).max()), int((err > tol).sum()))
        arrived = self.out.arrived_all().cpu().numpy()
        counts = np.zeros_like(arrived)
        counts[:, rank] = calls
        assert np.array_equal(arrived, counts)


def walk(X, s, K):
    return 8 * 2.0 ** -24 * math.sqrt(max(K, 1)) * 12 * 144 * float(X.abs().max()) * float(s.abs().max())


SHAPES = [  # M, K, N, world, rank, group
    (1, 32, 8, 1, 0, 32), (1, 64, 16, 2, 1, 64), (2, 128, 24, 3, 0, 128), (1, 160, 40, 8, 7, 64),
    (3, 96, 72, 2, 0, 128), (4, 1024, 64, 4, 2, 32), (5, 2080, 136, 8, 3, 128), (7, 992, 16, 1, 0, 64),
    (15, 256, 256, 2, 1, 128), (16, 4096, 48, 2, 0, 64), (17, 480, 32, 4, 1, 32), (31, 1056, 88, 1, 0, 64),
    (32, 512, 512, 2, 1, 128), (33, 2048, 40, 2, 0, 128), (47, 800, 104, 8, 4, 32), (48, 1184, 200, 2, 1, 64),
    (49, 64, 8, 8, 0, 32), (63, 3104, 56, 2, 1, 64), (64, 1024, 1480, 4, 1, 128)]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "m%d_k%d_n%d_w%d_r%d_g%d" % s)
def test_products(shape, dtype, zeros):
    M, K, N, world, rank, group = shape
    t = inputs(M, K, N, dtype, group, zeros, M + K + N, whole=True)
    c = Call(M, N, world, dtype, t, group, ldx_pad=8 * (M % 3))
    c.run(rank)
    c.check(rank, expected(*t, group), dtype, None)
    t = inputs(M, K, N, dtype, group, zeros, M + K + N + 1)
    c = Call(M, N, world, dtype, t, group)
    c.run(rank)
    c.run(rank)
    c.check(rank, expected(*t, group), dtype, walk(t[0], t[2], K), calls=2)


BUILDS = [  # long columns and many tiles: every build and its rest at the ends of K and N
    (1, 16416, 24, 2, 0, 32), (2, 24640, 40, 1, 0, 128), (4, 544, 4360, 2, 1, 64), (3, 8224, 4104, 1, 0, 128),
    (16, 16416, 40, 2, 1, 64), (9, 544, 4360, 2, 0, 32), (16, 8224, 4104, 1, 0, 128), (13, 20512, 4104, 1, 0, 64),
    (20, 16416, 72, 2, 0, 32), (32, 8224, 136, 1, 0, 128), (17, 160, 4360, 1, 0, 64), (50, 12320, 104, 2, 1, 128),
    (64, 8224, 4104, 1, 0, 64), (33, 24640, 24, 1, 0, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", BUILDS, ids=lambda s: "m%d_k%d_n%d_w%d_r%d_g%d" % s)
def test_long_columns_and_many_tiles(shape, dtype):
    M, K, N, world, rank, group = shape
    t = inputs(M, K, N, dtype, group, True, M + K + N)
    want, bound = expected(*t, group), walk(t[0], t[2], K)
    c = Call(M, N, world, dtype, t, group)
    for calls in (1, 2):                 # the second runs on what the first left in the workspace
        c.out.C_all().view(torch.int16).fill_(-1)
        c.run(rank)
        c.check(rank, want, dtype, bound, calls=calls)


@pytest.mark.parametrize("M,K,N", [(24, 2048, 136), (64, 8192, 200)])
def test_without_a_workspace(M, K, N):
    """The C call without a workspace does not split K; a workspace too small is refused."""
    pkg = sym()
    t = inputs(M, K, N, "bf16", 64, True, 3, whole=True)
    c = Call(M, N, 2, "bf16", t, 64)
    args = [c.heap.handle, c.X.data_ptr(), c.w.q.data_ptr(), c.w.scales.data_ptr(), c.w.zeros.data_ptr(),
            c.heap.ptr(1, c.out.c_off), c.heap.ptr(1, c.out.flag_off), M, N, K, 0, 64, pkg.BF16, 1, 2]
    need = pkg.symtile_w4_workspace_bytes(0, M, N, K, 64)
    assert need > 0 and need % 16 == 0
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    with pytest.raises(pkg.SymtileError) as e:
        pkg.symtile_w4_all_scatter(*args, ws.data_ptr(), need - 1, pkg.current_stream())
    assert e.value.name == "EINVAL"
    with pytest.raises(pkg.SymtileError):
        pkg.symtile_w4_all_scatter(*args, ws.data_ptr() + 8, need, pkg.current_stream())
    pkg.symtile_w4_all_scatter(*args, stream=pkg.current_stream())
    c.check(1, expected(*t, 64), "bf16", None)
    for bad in ((0, -1, N, K, 64), (0, M, N, 48, 64), (0, M, 12, K, 64), (0, M, N, K, 96)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_w4_workspace_bytes(*bad)
        assert e.value.name == "EINVAL", bad
    with pytest.raises(pkg.SymtileError) as e:
        pkg.symtile_w4_workspace_bytes(0, 65, N, K, 64)
    assert e.value.name == "EUNSUPPORTED"
    assert pkg.symtile_w4_workspace_bytes(0, 0, N, K, 64) == 0


@pytest.mark.parametrize("M,dtype", [(1, "bf16"), (16, "f16"), (64, "bf16")])
def test_the_large_layer(M, dtype):
    K, N, world, rank, group = 8192, 3584, 8, 3, 128
    t = inputs(M, K, N, dtype, group, True, M)
    c = Call(M, N, world, dtype, t, group)
    c.run(rank)
    c.check(rank, expected(*t, group), dtype, walk(t[0], t[2], K))


def test_every_nibble_is_its_own_weight():
    """X one-hot in k: the product is the weight itself, for every k and column."""
    K, N, group = 256, 32, 64
    _, q, s, z = inputs(1, K, N, "bf16", group, True, 5, whole=True)
    for k0 in range(0, K, 64):
        X = torch.zeros((64, K), dtype=torch.bfloat16)
        X[torch.arange(64), k0 + torch.arange(64)] = 1.0
        c = Call(64, N, 1, "bf16", (X, q, s, z), group)
        c.run(0)
        c.check(0, expected(X, q, s, z, group), "bf16", None)


def test_no_inner_dimension_stores_zeros():
    c = Call(3, 24, 2, "bf16", (torch.zeros((3, 0)), torch.zeros((24, 0), dtype=torch.uint8),
                                torch.zeros((24, 0)).bfloat16(), None), 32)
    c.run(1)
    c.check(1, np.zeros((3, 24)), "bf16", None)


def test_rows_do_not_touch_each_other():
    """A row of X with infinities leaves the others as they were."""
    t = inputs(20, 512, 64, "bf16", 64, False, 3, whole=True)
    X = t[0].clone()
    X[4, 100], X[17, 3] = math.inf, math.nan
    c = Call(20, 64, 2, "bf16", (X, *t[1:]), 64)
    c.run(0)
    c.heap.barrier()
    got = c.out.C(1)[:, :64].double().cpu().numpy()
    want = expected(*t, 64)
    keep = [m for m in range(20) if m not in (4, 17)]
    assert np.array_equal(got[keep], torch.from_numpy(want[keep]).bfloat16().double().numpy())
    assert not np.isfinite(got[[4, 17]]).any()


def test_upper_bits_of_zeros_are_ignored():
    X, q, s, z = inputs(2, 128, 32, "f16", 32, True, 1, whole=True)
    c = Call(2, 32, 1, "f16", (X, q, s, z | 0xF0), 32)
    c.run(0)
    c.check(0, expected(X, q, s, z, 32), "f16", None)


def test_streams_and_graph_replays():
    M, K, N = 4, 1024, 128
    t = inputs(M, K, N, "bf16", 64, True, 1)
    c = Call(M, N, 2, "bf16", t, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(1)
    torch.cuda.current_stream().wait_stream(side)
    c.check(1, expected(*t, 64), "bf16", walk(t[0], t[2], K))
    eager = c.out.C_all().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(1)
    for i in range(4):
        c.out.C_all().view(torch.int16).fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out.C_all().view(torch.int16), eager.view(torch.int16)), i
    c.check(1, expected(*t, 64), "bf16", walk(t[0], t[2], K), calls=5)


def test_refusals():
    pkg = sym()
    t = inputs(2, 64, 16, "bf16", 32, True, 1)
    c = Call(2, 16, 2, "bf16", t, 32)
    args = dict(h=c.heap.handle, X=c.X.data_ptr(), q=c.w.q.data_ptr(), scales=c.w.scales.data_ptr(),
                zeros=0, C=c.heap.ptr(0, c.out.c_off), arrived=c.heap.ptr(0, c.out.flag_off), M=2,
                N=16, K=64, ldx=0, group=32, dtype=pkg.BF16, rank=0, world=2)
    for change, name in ((dict(dtype=pkg.F32), "EUNSUPPORTED"), (dict(world=3), "EINVAL"),
                         (dict(rank=2), "EINVAL"), (dict(M=-1), "EINVAL"), (dict(M=65), "EUNSUPPORTED"),
                         (dict(group=48), "EINVAL"), (dict(K=48), "EINVAL"), (dict(N=12), "EINVAL"),
                         (dict(ldx=63), "EINVAL"), (dict(ldx=32), "EINVAL"), (dict(X=0), "EINVAL"),
                         (dict(q=0), "EINVAL"), (dict(scales=0), "EINVAL"), (dict(C=0), "EINVAL"),
                         (dict(X=args["X"] + 2), "EINVAL"), (dict(q=args["q"] + 1), "EINVAL"),
                         (dict(C=args["C"] + 2), "EINVAL"), (dict(C=args["X"]), "EINVAL"),
                         (dict(arrived=args["X"]), "EINVAL"), (dict(arrived=args["C"]), "EINVAL"),
                         (dict(rank=1), "EINVAL")):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_w4_all_scatter(*{**args, **change}.values())
        assert e.value.name == name, change
    pkg.symtile_w4_all_scatter(*{**args, "M": 0}.values())
    pkg.symtile_w4_all_scatter(*{**args, "N": 0}.values())
    c.heap.barrier()
    assert int(c.out.arrived_all().sum()) == 0
    w = c.w
    with pytest.raises(TypeError):
        c.out.run_w4(c.X.half(), w, 0)
    with pytest.raises(ValueError):
        c.out.run_w4(c.X[:1], w, 0)
    with pytest.raises(ValueError):
        c.out.run_w4(c.X.t(), w, 0)
    other = pkg.GatheredOutput(pkg.Heap(1, 1 << 20), 2, 16, torch.bfloat16, 64, 64)
    with pytest.raises(ValueError):
        other.run_w4(c.X, w, 0)
    for bad, err in (((w.q.int(), w.scales), TypeError), ((w.q, w.scales.float()), TypeError),
                     ((w.q, w.scales[:, :1]), ValueError), ((w.q.cpu(), w.scales), ValueError),
                     ((w.q, w.scales, w.zeros[:8]), ValueError)):
        with pytest.raises(err):
            pkg.W4Weight(*bad, group=32)
    with pytest.raises(ValueError):
        pkg.W4Weight(w.q, w.scales, None, 48)


def test_one_workspace_for_calls_of_all_sizes():
    """Few columns, many, few again, with other M, on one workspace of the C call."""
    pkg = sym()
    sizes = [(64, 8192, 3584), (64, 8192, 8192), (20, 4096, 40), (16, 8192, 6000), (33, 8192, 8000), (64, 8192, 3584)]
    need = max(pkg.symtile_w4_workspace_bytes(0, M, N, K, 128) for M, K, N in sizes)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    for M, K, N in sizes:
        t = inputs(M, K, N, "bf16", 128, True, M + N)
        c = Call(M, N, 1, "bf16", t, 128)
        pkg.symtile_w4_all_scatter(c.heap.handle, c.X.data_ptr(), *c.w.pointers, c.heap.ptr(0, c.out.c_off),
                                   c.heap.ptr(0, c.out.flag_off), M, N, K, 0, 128, pkg.BF16, 0, 1,
                                   ws.data_ptr(), ws.numel(), pkg.current_stream())
        c.check(0, expected(*t, 128), "bf16", walk(t[0], t[2], K))


@pytest.mark.parametrize("M,K,N", [(64, 8192, 200), (16, 2048, 4360)])
def test_the_first_call_on_another_stream(M, K, N):
    """stream= for the first call, whose workspace is made in it, while torch's current stream is
    busy and the memory of the workspace held other values before; then replays of a graph."""
    pkg = sym()
    t = inputs(M, K, N, "bf16", 64, True, 1)
    want, bound = expected(*t, 64), walk(t[0], t[2], K)
    c = Call(M, N, 2, "bf16", t, 64)
    need = pkg.symtile_w4_workspace_bytes(0, M, N, K, 64)
    assert need > 0
    side = torch.cuda.Stream()
    for s in (torch.cuda.current_stream(), side):        # what a new workspace of either may get
        with torch.cuda.stream(s):
            dirty = torch.full((need,), 3, dtype=torch.uint8, device="cuda")
            del dirty
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    c.run(1, stream=side.cuda_stream)
    side.synchronize()
    early = c.out.C(1).clone()
    c.check(1, want, "bf16", bound)
    assert torch.equal(early.view(torch.int16), c.out.C(1).view(torch.int16))
    c.run(1)                                             # the same workspace on the current stream
    c.check(1, want, "bf16", bound, calls=2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(1)
    for i in range(4):
        c.out.C_all().view(torch.int16).fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        c.check(1, want, "bf16", bound, calls=3 + i)


def test_the_first_call_on_the_null_stream_beside_another():
    t = inputs(64, 8192, 200, "bf16", 64, True, 1)
    c = Call(64, 200, 2, "bf16", t, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(20_000_000)
        c.run(1, stream=0)
    c.check(1, expected(*t, 64), "bf16", walk(t[0], t[2], 8192))


def test_one_row_expanded_to_several_is_refused():
    """Rows without a distance between them are not rows K apart."""
    t = inputs(3, 64, 16, "bf16", 32, True, 1)
    c = Call(3, 16, 2, "bf16", t, 32)
    with pytest.raises(ValueError):
        c.out.run_w4(c.X[:1].expand(3, 64), c.w, 0)
    with pytest.raises(ValueError):
        c.out.run_w4(c.X.flatten()[:128].as_strided((3, 64), (32, 1)), c.w, 0)
    one = inputs(1, 64, 16, "bf16", 32, True, 1)
    c = Call(1, 16, 2, "bf16", one, 32)
    c.out.run_w4(c.X.expand(1, 64), c.w, 1)          # a single row has no distance
    c.check(1, expected(*one, 32), "bf16", walk(one[0], one[2], 64))
