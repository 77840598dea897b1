"""A quantized output projection learns from labels and from a teacher's stored top logits.

    python examples/train_head.py [--steps 40] [--rows 512] [--fmt fp8|int4] [--top-k 32]

One training step is three calls on the same arrays: the two losses of every token (HeadLoss.forward), their gradients
(HeadLoss.backward), and the optimizer step that applies grad_weights to the codes (Plan.step).  The projection has the shape of
the 30 M transformer's embedding of `workloads` and stays FP8 or INT4 throughout: the losses read its codes and scales, and no
master weights exist.  Synthetic data: hidden states around a hidden "concept" of each token, a teacher that knows it.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads                                              # noqa: E402
from paper_2601_22101_amd import binding as eco, harness      # noqa: E402


def train(steps: int = 40, rows: int = 512, fmt: str = "fp8", top_k: int = 32, temperature: float = 2.0, lr: float = 1e-3, seed: int = 1, report=None):
    """(mean cross entropy, mean distillation loss) before each step."""
    spec = next(t for t in workloads.config2().tensors if t.name == "embed")
    vocab, dim = spec.shape
    code, group = {"fp8": eco.ECO_FMT_FP8_E4M3, "int4": eco.ECO_FMT_INT4}[fmt], 128
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")        # noqa: E731

    # the teacher's projection, and the student's, which starts from noise
    teacher = normal(vocab, dim) * 0.05
    student = normal(vocab, dim) * 0.02
    weights = torch.empty(vocab * dim // (1 if fmt == "fp8" else 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty(vocab * dim // group, dtype=torch.float32, device="cuda")
    eco.eco_quantize_init(student, eco.ECO_DT_FP32, vocab * dim, code, group, eco.ECO_DT_FP32, weights, scales)

    target = (vocab * torch.rand(rows, generator=gen, device="cuda") ** 3).long()
    hidden = (normal(rows, dim) + 4.0 * teacher[target] / 0.05).to(torch.bfloat16)
    top = (hidden.float() @ teacher.t()).topk(top_k, dim=1)
    labels = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.2, -100, target)      # a fifth of the tokens is prompt: the teacher alone
    grad_ce = torch.full((rows,), 0.5 / rows, device="cuda")
    grad_kd = torch.full((rows,), 0.5 / rows, device="cuda")

    head = harness.HeadLoss(rows, vocab, dim, weights=weights, fmt=code, scales=scales, group_size=group, top_k=top_k, temperature=temperature)
    m, v = torch.zeros(vocab * dim, device="cuda"), torch.zeros(vocab * dim, device="cuda")
    tensor = eco.make_tensor(weights, scales, head.grad_weights, m, v, vocab * dim, 0, code)
    losses = []
    with eco.Plan([tensor], eco.make_hparams(block_size=group)) as plan:
        for k in range(1, steps + 1):
            ce, kd = head.forward(hidden, labels, top.indices.int(), top.values)
            head.backward(grad_ce, grad_kd)
            plan.step(eco.make_hparams(lr=lr, step=k, block_size=group, seed=seed))
            losses.append((float(ce.sum() / (labels >= 0).sum()), float(kd.mean())))
            if report and (k == 1 or k % 10 == 0):
                report(f"step {k:3d}  cross entropy {losses[-1][0]:.4f}  distillation {losses[-1][1]:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--fmt", choices=("fp8", "int4"), default="fp8")
    ap.add_argument("--top-k", type=int, default=32)
    a = ap.parse_args()
    train(a.steps, a.rows, a.fmt, a.top_k, report=print)
