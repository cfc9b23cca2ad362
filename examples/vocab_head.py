"""A vocabulary-parallel head in 4 bits, checked against and tuned to the 16-bit one.

    python examples/vocab_head.py [--world 8 --hidden 4096 --shard 1024 --tokens 48 --steps 20]

Every rank holds a column shard of the head.  The 16-bit head is the fused GEMM +
All-Scatter; its most likely tokens are the teacher's lists.  The 4-bit head is
the product that reads 4-bit weights, its logits gathered into every slot the
same way.  The 4-bit head's log probabilities are compared with the 16-bit
head's, and a bias over the vocabulary, added to its logits, is trained against
the teacher's lists.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2511_12500_amd as sym  # noqa: E402

GROUP = 64


def quantise(shard: torch.Tensor) -> sym.W4Weight:
    """A shard [K, N] as 4-bit weights: per column and group of k the range of
    its weights in 15 steps, the zero point a whole number."""
    K, N = shard.shape
    w = shard.t().float().reshape(N, K // GROUP, GROUP)
    low, high = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    scales = ((high - low) / 15).clamp(min=1e-6).to(shard.dtype)
    step = scales.float()
    zeros = (-low / step).round().clamp(0, 15)
    q = (w / step[:, :, None] + zeros[:, :, None]).round().clamp(0, 15)
    q = q.reshape(N, K).to(torch.uint8)
    return sym.W4Weight((q[:, 0::2] | q[:, 1::2] << 4).contiguous(), scales.contiguous(),
                        zeros.to(torch.uint8).contiguous(), GROUP)


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser()
    ap.add_argument("--world", type=int, default=8)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--shard", type=int, default=1024, help="columns of the vocabulary a rank")
    ap.add_argument("--tokens", type=int, default=48, help="at most 64")
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--lr", type=float, default=2.0)
    a = ap.parse_args(argv)
    w, K, N, M = a.world, a.hidden, a.shard, a.tokens
    vocab, dt = w * N, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(0)

    X = torch.randn((M, K), generator=gen, device="cuda").to(dt)
    shards = [(torch.randn((K, N), generator=gen, device="cuda") * (2.5 / K ** 0.5)).to(dt)
              for _ in range(w)]
    weights = [quantise(s) for s in shards]

    heap = sym.Heap(w, 2 * (M * vocab * 2 + w * vocab * 4) + (1 << 20))
    full = sym.GatheredOutput(heap, M, N, dt, 64, 64)
    small = sym.GatheredOutput(heap, M, N, dt, sym.W4_TILE_M, sym.W4_TILE_N)
    for r in range(w):
        full.run(X, shards[r], r, sym.FUSED_SEQ)
        small.run_w4(X, weights[r], r)
    heap.barrier()
    # any slot holds the gathered logits; take the last rank's
    teacher, student = full.C(w - 1), small.C(w - 1)

    at_teacher = sym.TokenLogprobs(M, vocab, dt, top=a.top)
    at_teacher.run(teacher)
    chosen = at_teacher.top_ids[:, 0].contiguous()
    at_student = sym.TokenLogprobs(M, vocab, dt, top=1)
    at_student.run(student, chosen)
    kept = (at_student.top_ids[:, 0] == chosen).float().mean().item()
    shift = (at_student.logprob - at_teacher.top_logprobs[:, 0]).abs().mean().item()
    print(f"4-bit head of {vocab} tokens: the 16-bit head's first choice kept for "
          f"{100 * kept:.0f}% of {M} rows, its log probability moved by {shift:.3f} on average")

    # a bias over the vocabulary, trained on the teacher's lists and their remaining mass
    bias = torch.zeros(vocab, device="cuda")
    kd = sym.TopDistillation(M, vocab, torch.float32, a.top, rest=True)
    weight = torch.full((M,), 1.0 / M, device="cuda")
    losses = []
    for step in range(a.steps):
        logits = student.float() + bias
        kd.run(logits, at_teacher.top_ids, at_teacher.top_logprobs, weight, logits)   # in place
        losses.append((kd.loss * weight).sum().item())
        bias -= a.lr * M * logits.sum(0)
    print(f"distillation loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    heap.close()
    return {"kept": kept, "shift": shift, "losses": losses}


if __name__ == "__main__":
    main()
