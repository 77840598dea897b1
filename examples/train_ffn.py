"""The feed-forward half of a layer learns on quantized weights: norm, gated unit and down projection, forward, backward and the optimizer step.

    python examples/train_ffn.py [--steps 40] [--rows 2048] [--fmt fp8|int4] [--act silu|gelu]

A training step is seven calls on the same arrays.  The residual stream x goes through RowNorm (8-bit rows), GatedUnit (8-bit rows) and Linear, which adds what RowNorm passed on;
backward goes the same way back, and Plan.step applies the bf16 gradients to the codes of gate, up and down and to the bf16 gain.  The matrices have the shapes of the
DeepSeek-MoE-16B experts of `workloads` and stay FP8 or INT4 throughout; no master weights exist.  Synthetic data: the layer is to do what another, random layer does.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads                                              # noqa: E402
from paper_2601_22101_amd import binding as eco, harness      # noqa: E402


class Layer:
    """Codes, scales and optimizer state of the four tensors, and the units that read them."""

    def __init__(self, rows: int, dim: int, width: int, fmt: str, act: str, gen: torch.Generator):
        code, self.group = {"fp8": eco.ECO_FMT_FP8_E4M3, "int4": eco.ECO_FMT_INT4}[fmt], 128
        self.codes, self.scales = {}, {}
        for name, shape in (("gate", (width, dim)), ("up", (width, dim)), ("down", (dim, width))):
            n = shape[0] * shape[1]
            w = torch.randn(shape, generator=gen, device="cuda") * 0.02
            self.codes[name] = torch.empty(n // (1 if fmt == "fp8" else 2), dtype=torch.uint8, device="cuda")
            self.scales[name] = torch.empty(n // self.group, device="cuda")
            eco.eco_quantize_init(w, eco.ECO_DT_FP32, n, code, self.group, eco.ECO_DT_FP32, self.codes[name], self.scales[name])
        self.gain = torch.ones(dim, dtype=torch.bfloat16, device="cuda")
        c, s = self.codes, self.scales
        self.norm = harness.RowNorm(rows, dim, gain=self.gain, residual=True, training=True)
        self.unit = harness.GatedUnit(rows, dim, width, gate=c["gate"], gate_scales=s["gate"], up=c["up"], up_scales=s["up"], fmt=code, group_size=self.group, act=act,
                                      training=True)
        self.down = harness.Linear(rows, width, dim, weights=c["down"], scales=s["down"], fmt=code, group_size=self.group, training=True)
        self.state, tensors = [], []
        for k, (name, grad) in enumerate((("gate", self.unit.grad_gate), ("up", self.unit.grad_up), ("down", self.down.grad_weights))):
            m, v = torch.zeros(grad.numel(), device="cuda"), torch.zeros(grad.numel(), device="cuda")
            self.state.append((m, v))
            tensors.append(eco.make_tensor(c[name], s[name], grad, m, v, grad.numel(), k, code))
        m, v = torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
        self.state.append((m, v))
        tensors.append(eco.make_tensor(self.gain, None, self.norm.grad_gain, m, v, dim, 3, eco.ECO_FMT_BF16_PLAIN))
        self.plan = eco.Plan(tensors, eco.make_hparams(block_size=self.group))

    def forward(self, x: torch.Tensor, residual: torch.Tensor) -> torch.Tensor:
        y, scales, stream = self.norm.forward(x, residual)
        return self.down.forward(*self.unit.forward(y, scales), add=stream)

    def backward(self, grad: torch.Tensor) -> torch.Tensor:
        grad_h, _ = self.down.backward(grad)
        grad_y, _, _ = self.unit.backward(grad_h)
        return self.norm.backward(grad_y, grad)[0]


def train(steps: int = 40, rows: int = 2048, fmt: str = "fp8", act: str = "silu", lr: float = 1e-3, seed: int = 1, report=None):
    """The mean squared error before each step, and the layer."""
    spec = next(t for t in workloads.config5(layers=1).tensors if t.name.endswith("gate"))
    width, dim = spec.shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    layer, teacher = Layer(rows, dim, width, fmt, act, gen), Layer(rows, dim, width, "fp8", act, gen)
    losses = []
    for k in range(1, steps + 1):
        x, residual = (torch.randn(rows, dim, generator=gen, device="cuda").bfloat16() for _ in range(2))
        error = layer.forward(x, residual).float() - teacher.forward(x, residual).float()
        layer.backward((error * (2.0 / error.numel())).bfloat16())
        layer.plan.step(eco.make_hparams(lr=lr, step=k, block_size=layer.group, seed=seed))
        losses.append(float(error.square().mean()))
        if report and (k == 1 or k % 10 == 0):
            report(f"step {k:3d}  mean squared error {losses[-1]:.6f}")
    layer.plan.close()
    teacher.plan.close()
    return losses, layer


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--rows", type=int, default=2048)
    ap.add_argument("--fmt", choices=("fp8", "int4"), default="fp8")
    ap.add_argument("--act", choices=("silu", "gelu"), default="silu")
    a = ap.parse_args()
    train(a.steps, a.rows, a.fmt, a.act, report=print)
