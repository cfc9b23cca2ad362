"""GPU test of examples/vocab_head.py: the 4-bit head, its log probabilities and
the distillation run together over the gathered logits of the heap."""
import importlib.util
import os

import pytest
import torch

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("args", [
    ["--world", "2", "--hidden", "256", "--shard", "264", "--tokens", "5", "--top", "16"],
    ["--world", "8", "--hidden", "1024", "--shard", "512", "--tokens", "40"],
])
def test_vocab_head(args):
    require_gpu()
    spec = importlib.util.spec_from_file_location(
        "vocab_head", os.path.join(ROOT, "examples", "vocab_head.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main([*args, "--steps", "10"])
    torch.cuda.synchronize()
    # 15 steps a group of normal weights leave some 10% noise: logits of spread 2.5 move by
    # about 0.3, the log probability of the first choice by less than one on average
    assert got["shift"] < 1.0
    assert got["losses"][-1] < 0.8 * got["losses"][0]
