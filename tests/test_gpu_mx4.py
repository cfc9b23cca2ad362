"""GPU tests of the matrices in blocks of 4-bit floating point: MX4Matrix.quantise bit by
bit, and GatheredOutput.run_mx4 against the definition in 64 bits.

The product's bound: products are exact, a block's 32 are summed without loss beside the
running sum's own rounding, so a result is off by at most 2^-24 of the sum of magnitudes
for every block of K and for every join of partial sums (at most 64), and by half an ulp
of the output.  Whole-number inputs are exact and compared exactly."""
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


def gen(seed):
    return torch.Generator().manual_seed(seed)


def spread(rows, K, dtype, seed):
    """Blocks of sizes far apart, ties and values beside them."""
    g = gen(seed)
    x = torch.randn((rows, K), generator=g)
    tie = torch.randint(-28, 29, (rows, K), generator=g) / 4.0
    x = torch.where(torch.rand((rows, K), generator=g) < 0.4, tie, x)
    far = 30 if dtype != "f16" else 6
    e = torch.randint(-far, far + 1, (rows, -(-K // 32)), generator=g).repeat_interleave(32, 1)[:, :K]
    return torch.ldexp(x, e).to(TD[dtype])


def run_quantise(x, values=None, **kw):
    m = sym().MX4Matrix.empty(x.shape[0], x.shape[1])
    m.q.fill_(0x5A)
    m.scales.fill_(0x5A)
    m.quantise(x, values, **kw)
    torch.cuda.synchronize()
    return m


def check_quantise(x, m, values=None):
    q, s = o.mx4_quantise(x.double().cpu().numpy())
    assert np.array_equal(m.scales.cpu().numpy(), s)
    assert np.array_equal(m.q.cpu().numpy(), q)
    if values is not None:
        want = torch.from_numpy(o.mx4_values(q, s)).to(values.dtype)
        got = values.cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(nan=1.0), want.nan_to_num(nan=1.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (3, 64), (1, 96), (5, 1056), (64, 8192), (333, 160), (2, 32 * 3001)])
def test_quantise(rows, K, dtype):
    x = spread(rows, K, dtype, rows + K).cuda()
    values = torch.full_like(x, math.nan)
    check_quantise(x, run_quantise(x, values), values)
    check_quantise(x, run_quantise(x))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_quantise_rows_anywhere(dtype):
    """Rows any distance apart, starting at any element; values beside them, or in place."""
    x0 = spread(37, 128, dtype, 5)
    wide = torch.full((37, 131), math.nan, dtype=TD[dtype], device="cuda")
    x = wide[:, 1:129]
    x.copy_(x0)
    other = torch.full((37, 137), 7.0, dtype=TD[dtype], device="cuda")
    values = other[:, 3:131]
    check_quantise(x0, run_quantise(x, values), values)
    assert bool((other[:, :3] == 7).all()) and bool((other[:, 131:] == 7).all())
    assert torch.equal(x.cpu(), x0)
    check_quantise(x0, run_quantise(x, x), x)
    assert bool(wide[:, 0].isnan().all()) and bool(wide[:, 129:].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_quantise_ends_of_the_range(dtype):
    """Zeros, the smallest and largest numbers, infinities and NaN."""
    f = torch.finfo(TD[dtype])
    x = torch.zeros((1, 32 * 10), dtype=TD[dtype])
    x[0, 40] = -0.0
    x[0, 64:96] = f.smallest_normal
    x[0, 100] = f.smallest_normal * f.eps          # the smallest number
    x[0, 128:160] = torch.linspace(-1, 1, 32).to(TD[dtype]) * f.max
    x[0, 170] = math.inf
    x[0, 200], x[0, 201] = math.nan, 1.0
    x[0, 225] = -math.inf
    x[0, 256:288] = torch.arange(32).to(TD[dtype]) * f.smallest_normal * f.eps
    x[0, 288:320] = torch.arange(-16, 16).to(TD[dtype]) * f.smallest_normal
    x = x.cuda()
    values = torch.zeros_like(x)
    check_quantise(x, run_quantise(x, values), values)


def test_quantise_refusals():
    pkg = sym()
    x = torch.zeros((4, 64), device="cuda")
    m = pkg.MX4Matrix.empty(4, 64)
    for bad in (torch.zeros((4, 32), device="cuda"), torch.zeros((4, 128), device="cuda")[:, ::2], torch.zeros((4, 64))):
        with pytest.raises(ValueError):
            m.quantise(bad)
    with pytest.raises(TypeError):
        m.quantise(x.double())
    with pytest.raises(TypeError):
        m.quantise(x, x.half())
    flat = torch.zeros(4 * 64 + 64, device="cuda")
    with pytest.raises(pkg.SymtileError) as e:      # the rows, moved by one
        m.quantise(flat[:256].view(4, 64), flat[64:320].view(4, 64))
    assert e.value.name == "EINVAL"
    pkg.MX4Matrix.empty(0, 64).quantise(x[:0])
    pkg.MX4Matrix.empty(4, 0).quantise(x[:, :0])
    for bad in (lambda: pkg.MX4Matrix(m.q, m.scales[:, :1]), lambda: pkg.MX4Matrix(m.q.t(), m.scales),
                lambda: pkg.MX4Matrix.empty(4, 48), lambda: pkg.MX4Matrix(m.q.cpu(), m.scales.cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        pkg.MX4Matrix(m.q.int(), m.scales)


# ---- product ----------------------------------------------------------------------------
def operands(M, K, N, seed, whole=False):
    g = gen(seed)
    xq = torch.randint(0, 256, (M, K // 2), generator=g, dtype=torch.uint8)
    wq = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    lo, hi = (127, 128) if whole else (120, 130)
    xs = torch.randint(lo, hi, (M, K // 32), generator=g, dtype=torch.uint8)
    ws = torch.randint(lo, hi, (N, K // 32), generator=g, dtype=torch.uint8)
    if whole:         # sums that the output types hold exactly
        keep = 0x22 if K > 64 else 0xFF
        xq, wq = xq & (keep | 0x88), wq & (keep | 0x88)
    return xq, xs, wq, ws


class Call:
    def __init__(self, M, K, N, world, dtype, t):
        pkg = sym()
        self.shape, self.dtype, self.t = (M, K, N), dtype, t
        tiles = -(-M // 64) * -(-N // 16)
        self.heap = pkg.Heap(world, M * world * N * 2 + world * tiles * 4 + 8192)
        self.out = pkg.GatheredOutput(self.heap, M, N, TD[dtype], pkg.MX4_TILE_M, pkg.MX4_TILE_N)
        self.x = pkg.MX4Matrix(t[0].cuda(), t[1].cuda())
        self.w = pkg.MX4Matrix(t[2].cuda(), t[3].cuda())
        self.out.C_all().view(torch.int16).fill_(-1)

    def want(self):
        x = o.mx4_values(self.t[0].numpy(), self.t[1].numpy())
        w = o.mx4_values(self.t[2].numpy(), self.t[3].numpy())
        x, w = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
        return (x @ w.t()).cpu().numpy(), (x.abs() @ w.abs().t()).cpu().numpy()

    def check(self, rank, whole=False, calls=1):
        M, K, N = self.shape
        w = self.heap.world
        self.heap.barrier()
        C = self.out.C_all()
        for s in range(1, w):
            assert torch.equal(C[s].view(torch.int16), C[0].view(torch.int16)), s
        bits = C[0].view(torch.int16)
        for r in range(w):
            if r != rank:
                assert bool((bits[:, r * N:(r + 1) * N] == -1).all()), f"block of rank {r} written"
        got = C[0][:, rank * N:(rank + 1) * N].double().cpu().numpy()
        want, size = self.want()
        if whole:
            assert np.array_equal(got, torch.from_numpy(want).to(TD[self.dtype]).double().numpy())
        else:
            tol = (K / 32 + 64) * 2.0 ** -24 * size
            tol = tol + half_ulp(np.abs(want) + tol, self.dtype)
            err = np.abs(got - want)
            assert np.isfinite(got).all() and (err <= tol).all(), (float((err - tol).max()), int((err > tol).sum()))
        counts = np.zeros((w, w, self.out.tiles_m, self.out.tiles_n), dtype=np.int32)
        counts[:, rank] = calls
        assert np.array_equal(self.out.arrived_all().cpu().numpy(), counts)


SHAPES = [  # M, K, N, world, rank
    (1, 32, 8, 1, 0), (1, 64, 16, 2, 1), (2, 96, 24, 3, 0), (1, 128, 40, 8, 7), (3, 160, 72, 2, 0),
    (7, 512, 64, 4, 2), (16, 544, 136, 8, 3), (17, 992, 16, 1, 0), (33, 1024, 256, 2, 1), (49, 2080, 48, 2, 0),
    (64, 4096, 1480, 4, 1), (65, 32, 8, 1, 0), (100, 480, 88, 2, 1), (128, 1056, 264, 8, 5), (129, 256, 128, 1, 0),
    (255, 800, 104, 2, 0), (256, 512, 256, 4, 3), (257, 544, 520, 2, 1), (300, 2048, 1000, 1, 0),
    (511, 1120, 248, 2, 1), (700, 8224, 40, 1, 0), (1000, 96, 1016, 2, 0), (40, 16416, 4104, 1, 0),
    (1000, 544, 2400, 1, 0), (3000, 608, 3000, 1, 0), (2900, 1024, 3200, 2, 1), (64, 512, 16400, 1, 0),
    (50, 544, 16424, 2, 1), (120, 1056, 8200, 1, 0), (700, 1024, 4104, 2, 0), (16, 1056, 4104, 1, 0),
    (1, 8192, 8200, 1, 0), (20, 8192, 264, 8, 7)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "m%d_k%d_n%d_w%d_r%d" % s)
def test_products(shape, dtype):
    M, K, N, world, rank = shape
    c = Call(M, K, N, world, dtype, operands(M, K, N, sum(shape), whole=True))
    c.out.run_mx4(c.x, c.w, rank)
    c.check(rank, whole=True)
    t = operands(M, K, N, sum(shape) + 1)
    if dtype == "f16":
        t = (t[0], t[1] - 4, t[2], t[3] - 4)
    c = Call(M, K, N, world, dtype, t)
    for calls in (1, 2):           # the second runs on what the first left in the workspace
        c.out.run_mx4(c.x, c.w, rank)
        c.check(rank, calls=calls)


@pytest.mark.parametrize("M,K,N,world", [(1, 8192, 3584, 8), (64, 8192, 3584, 8), (4096, 8192, 3584, 2),
                                         (2048, 4096, 1024, 8), (1100, 8192, 28672, 1)])
def test_the_layers(M, K, N, world):
    c = Call(M, K, N, world, "bf16", operands(M, K, N, M))
    c.out.run_mx4(c.x, c.w, world - 1)
    c.check(world - 1)


def test_every_place_is_its_own():
    """A token with one element: the product is the weight itself, for every k and column."""
    M, K, N = 64, 1088, 32
    for first in range(0, K, M):
        xq = torch.zeros((M, K // 2), dtype=torch.uint8)
        k = first + torch.arange(M)
        xq[torch.arange(M), k // 2] = torch.where(k % 2 == 0, 2, 32).to(torch.uint8)     # 1.0
        _, _, wq, ws = operands(M, K, N, 3)
        c = Call(M, K, N, 1, "bf16", (xq, torch.full((M, K // 32), 127, dtype=torch.uint8), wq, ws))
        c.out.run_mx4(c.x, c.w, 0)
        c.check(0, whole=True)


@pytest.mark.parametrize("M", [5, 300])
def test_scales_at_their_ends(M):
    """The smallest and largest scales meet in exact products; a NaN scale stays in its row
    and its column; no inner dimension stores zeros."""
    K, N = 96, 40
    t = operands(M, K, N, 3, whole=True)
    t[1][0] = 0
    t[3][:] = 254 - 30
    t[1][1:] = 30 + 127 - 127
    t[1][0] = 30
    c = Call(M, K, N, 2, "bf16", t)
    c.out.run_mx4(c.x, c.w, 1)
    c.check(1, whole=True)
    t = operands(M, K, N, 4, whole=True)
    t[1][3, 1] = 255
    t[3][17, 2] = 255
    c = Call(M, K, N, 2, "bf16", t)
    c.out.run_mx4(c.x, c.w, 0)
    c.heap.barrier()
    got = c.out.C(1)[:, :N].float().cpu()
    bad = torch.zeros((M, N), dtype=torch.bool)
    bad[3], bad[:, 17] = True, True
    assert torch.equal(got.isnan(), bad)
    want = torch.from_numpy(c.want()[0]).to(torch.bfloat16).float()
    assert torch.equal(got[~bad], want[~bad])
    c = Call(M, 0, N, 2, "bf16", operands(M, 0, N, 4))
    c.out.run_mx4(c.x, c.w, 1)
    c.check(1, whole=True)


@pytest.mark.parametrize("M,K,N", [(24, 4096, 136), (64, 8192, 264), (200, 4096, 520)])
def test_without_a_workspace_and_refusals(M, K, N):
    pkg = sym()
    c = Call(M, K, N, 2, "bf16", operands(M, K, N, 5, whole=True))
    args = [c.heap.handle, *c.x.pointers, *c.w.pointers, c.heap.ptr(1, c.out.c_off), c.heap.ptr(1, c.out.flag_off),
            M, N, K, pkg.BF16, 1, 2]
    need = pkg.symtile_mx4_workspace_bytes(0, M, N, K)
    if need:
        ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        for at, n in ((0, need - 1), (8, need)):
            with pytest.raises(pkg.SymtileError) as e:
                pkg.symtile_mx4_all_scatter(*args, ws.data_ptr() + at, n, pkg.current_stream())
            assert e.value.name == "EINVAL"
    pkg.symtile_mx4_all_scatter(*args, stream=pkg.current_stream())
    c.check(1, whole=True)
    for i, bad in ((0, 0), (1, 0), (1, args[1] + 8), (3, args[3] + 1), (5, args[5] + 8), (5, c.heap.ptr(0, c.out.c_off)),
                   (6, args[5]), (6, args[6] + 2), (7, -1), (8, N + 4), (9, K - 16), (10, pkg.F32), (11, 2), (11, -1),
                   (12, 1)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_mx4_all_scatter(*args[:i], bad, *args[i + 1:], stream=pkg.current_stream())
        assert e.value.name == ("EUNSUPPORTED" if i == 10 else "EINVAL"), i
    with pytest.raises(ValueError):
        c.out.run_mx4(c.w, c.x, 0)
    other = pkg.GatheredOutput(c.heap, 1, 8, torch.bfloat16, 64, 64)
    with pytest.raises(ValueError):
        other.run_mx4(pkg.MX4Matrix.empty(1, 64), pkg.MX4Matrix.empty(8, 64), 0)
    c.check(1, whole=True)
    for bad in ((0, -1, N, K), (0, M, 12, K), (0, M, N, 48), (99, M, N, K)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_mx4_workspace_bytes(*bad)
        assert e.value.name == "EINVAL", bad


@pytest.mark.parametrize("M,K,N", [(1, 4096, 1024), (48, 8192, 264), (300, 2048, 520)])
def test_captured_and_on_another_stream(M, K, N):
    """Quantisation and product captured together; replays on new inputs, among eager calls."""
    pkg = sym()
    world, rank = 2, 1
    g = gen(M)
    xs = [torch.randn((M, K), generator=g).bfloat16() for _ in range(3)]
    _, _, wq, ws = operands(M, K, N, 7)
    x = xs[0].cuda()
    t = [*(torch.from_numpy(a) for a in o.mx4_quantise(xs[0].double().numpy())), wq, ws]
    c = Call(M, K, N, world, "bf16", t)
    c.x = pkg.MX4Matrix.empty(M, K)
    c.x.quantise(x)
    c.out.run_mx4(c.x, c.w, rank)
    c.check(rank)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.x.quantise(x)
        c.out.run_mx4(c.x, c.w, rank)
    calls = 1
    for i in range(4):
        x.copy_(xs[i % 3])
        c.t = [*(torch.from_numpy(a) for a in o.mx4_quantise(xs[i % 3].double().numpy())), wq, ws]
        graph.replay()
        calls += 1
        c.check(rank, calls=calls)
        if i == 1:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            c.x.quantise(x, stream=s.cuda_stream)
            c.out.run_mx4(c.x, c.w, rank, stream=s.cuda_stream)
            s.synchronize()
            calls += 1
            c.check(rank, calls=calls)


def test_captured_before_any_eager_call():
    """A workspace that a capture allocates would be zero in its replays alone: the captured
    call has none, and an eager one before the first replay makes its own."""
    pkg = sym()
    M, K, N = 64, 8192, 264
    assert pkg.symtile_mx4_workspace_bytes(0, M, N, K) > 0
    c = Call(M, K, N, 2, "bf16", operands(M, K, N, 5, whole=True))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.out.run_mx4(c.x, c.w, 1)
    assert not c.out.ws_mx4
    for calls in range(1, 5):
        if calls % 2:
            c.out.run_mx4(c.x, c.w, 1)
        else:
            graph.replay()
        c.check(1, whole=True, calls=calls)
    assert int(c.out.ws_mx4[K][:65536].sum()) == 0
