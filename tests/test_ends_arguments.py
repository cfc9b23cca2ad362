"""Arguments of the operators at a model's two ends that are refused before any device
work: by the C entries (addresses that are never read), and by the Python classes for
tensors on another GPU than the object's (stand-ins for tensors)."""
import types

import pytest
import torch

import paper_2511_12500_amd as pkg
from paper_2511_12500_amd import head, heap
from tests.test_head_arguments import Tensor, bare

A = 1 << 20                        # an address; apart from each other by 16 MB
P = [A + (i << 24) for i in range(12)]


def refused(f, args, changes, status="EINVAL"):
    for change in changes:
        bad = list(args)
        for i, v in change.items():
            bad[i] = v
        with pytest.raises(pkg.SymtileError) as e:
            f(*bad)
        assert e.value.name == status, change


def test_quantise():
    args = [0, P[0], 4, 64, 0, pkg.BF16, P[1], P[2], P[3], 0]
    refused(pkg.symtile_mx4_quantise, args, [
        {1: 0}, {2: -1}, {3: -32}, {3: 48}, {4: 63}, {5: 0}, {5: 4}, {6: 0}, {6: P[1] + 8}, {7: 0}, {9: 32},
        {1: P[0] + 1}, {8: P[3] + 1}, {8: P[0] + 2}, {8: P[0], 9: 128}, {6: P[0] + 64}, {7: P[0] + 64},
        {7: P[1] + 16}, {6: P[3] + 16}, {7: P[3]}, {4: 1 << 62}])
    pkg.symtile_mx4_quantise(0, 0, 0, 64, 0, pkg.F32, 0, 0)          # nothing to do
    pkg.symtile_mx4_quantise(0, 0, 4, 0, 0, pkg.F32, 0, 0)


def test_sizes_of_workspaces():
    refused(pkg.symtile_mx4_workspace_bytes, [0, 4, 16, 64],
            [{1: -1}, {2: -8}, {2: 12}, {3: -32}, {3: 40}, {3: (1 << 22) + 32}, {1: (1 << 21) + 1}])
    refused(pkg.symtile_verify_workspace_bytes, [0, 4, 2, 100, pkg.F32],
            [{1: -1}, {2: -1}, {2: 33}, {3: 0}, {3: (1 << 21) + 1}, {4: 0}, {1: (1 << 24) + 1}])
    refused(pkg.symtile_embed_workspace_bytes, [0, 4, 64],
            [{1: -1}, {2: -8}, {2: 12}, {1: (1 << 24) + 1}, {2: (1 << 20) + 8}, {1: 1 << 24, 2: 1 << 20}])


def test_verify():
    args = [0, P[0], 2, 3, 100, 0, pkg.F32, 1.0, P[1], P[2], 0, 1.0, P[3], P[4], 0, P[5], P[6], P[7], P[8], 1 << 23]
    refused(pkg.symtile_verify_draft, args, [
        {1: 0}, {1: P[0] + 2}, {2: -1}, {3: 33}, {3: -1}, {4: 0}, {5: 99}, {6: 7}, {7: 0.0}, {7: float("inf")},
        {7: float("nan")}, {8: 0}, {10: 50}, {11: -1.0}, {12: 0}, {13: 0}, {13: 0, 12: 0}, {14: 99}, {15: 0}, {16: 0},
        {17: 0}, {18: 0}, {18: P[8] + 4}, {19: 100}, {8: P[1] + 4}, {12: P[3] + 2}, {13: P[4] + 2}, {15: P[5] + 4},
        {16: P[6] + 4}, {17: P[7] + 2}])
    pkg.symtile_verify_draft(0, 0, 0, 3, 100, 0, pkg.F32, 1.0, 0, 0, 0, 1.0, 0, 0, 0, 0, 0, 0, 0, 0)


def test_embedding():
    refused(pkg.symtile_embed_all_scatter, [0] + [P[0], 4, P[1], 8, 64, 0, pkg.F32, 0, 1.0, P[2], P[3], 0, 1], [{}])
    args = [0, P[0], 10, P[1], 64, 0, pkg.F32, 0, 5, 1.0, P[2], 0, pkg.F32, 0, P[3], 1 << 23]
    refused(pkg.symtile_embed_backward, args, [
        {1: 0}, {1: P[0] + 4}, {2: -1}, {2: (1 << 24) + 1}, {3: 0}, {3: P[1] + 8}, {4: 12}, {4: -8}, {5: 56}, {5: 66},
        {6: 0}, {7: -1}, {8: -1}, {8: (1 << 21) + 1}, {9: float("nan")}, {9: float("inf")}, {10: 0}, {10: P[2] + 4},
        {10: P[1] + 64}, {11: 32}, {12: 9}, {13: 2}, {14: 0}, {14: P[3] + 8}, {15: 100}])
    pkg.symtile_embed_backward(0, 0, 0, 0, 64, 0, pkg.F32, 0, 5, 1.0, P[2], 0, pkg.F32, 1)   # nothing to add
    pkg.symtile_embed_backward(0, P[0], 10, P[1], 64, 0, pkg.F32, 0, 0, 1.0, 0, 0, pkg.F32, 0)


def test_product_without_a_heap():
    refused(pkg.symtile_mx4_all_scatter, [0, P[0], P[1], P[2], P[3], P[4], P[5], 1, 16, 64, pkg.BF16, 0, 1], [{}])


def test_tensors_of_another_gpu_are_refused():
    bf, u8, f32, i64 = torch.bfloat16, torch.uint8, torch.float32, torch.int64
    with pytest.raises(ValueError, match="one GPU"):
        head.MX4Matrix(Tensor((16, 32), u8, 1), Tensor((16, 2), u8, 0))
    m = head.MX4Matrix(Tensor((16, 32), u8, 1), Tensor((16, 2), u8, 1))
    assert (m.rows, m.K, m.device) == (16, 64, 1)
    for x, values in ((Tensor((16, 64), bf, 0), None), (Tensor((16, 64), bf, 1), Tensor((16, 64), bf, 0))):
        with pytest.raises(ValueError, match="cuda:1"):
            m.quantise(x, values)
    x = head.MX4Matrix(Tensor((4, 32), u8, 0), Tensor((4, 2), u8, 0))
    for device in (0, 1):
        out = bare(heap.GatheredOutput, heap=types.SimpleNamespace(device=device), dtype=bf, M=4, N_local=16,
                   tile_m=64, tile_n=16)
        with pytest.raises(ValueError, match=f"cuda:{device}"):
            out.run_mx4(x, m, 0)
    op = bare(head.DraftVerification, sequences=2, drafted=1, vocab=9, dtype=f32, device=1, scale=1.0, draft_scale=1.0,
              _dt=3, _out=(0,) * 5)
    good = [Tensor((4, 9), f32, 1), Tensor((2, 1), i64, 1), Tensor((2, 1), f32, 1), Tensor((2, 9), f32, 1),
            Tensor((2, 9), f32, 1)]
    for i in range(5):
        bad = list(good)
        bad[i] = Tensor(good[i].shape, good[i].dtype, 0)
        with pytest.raises(ValueError, match="cuda:1"):
            op.run(*bad)
    rows = bare(heap.GatheredRows, heap=types.SimpleNamespace(device=1), T=3, D=64, dtype=bf)
    for a, b in ((0, 1), (1, 0)):
        with pytest.raises(ValueError, match="cuda:1"):
            rows.run(Tensor((3,), i64, a), Tensor((5, 64), bf, b), 0)
    grad = bare(head.EmbeddingGrad, T=3, D=64, dtype=bf, device=1, _ws=(0, 0))
    good = [Tensor((3,), i64, 1), Tensor((3, 64), bf, 1), Tensor((5, 64), f32, 1)]
    for i in range(3):
        bad = list(good)
        bad[i] = Tensor(good[i].shape, good[i].dtype, 0)
        with pytest.raises(ValueError, match="cuda:1"):
            grad.run(*bad)
