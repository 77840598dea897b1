"""Inputs and bounds that tell apart in how many bfloat16 terms the logits' gradient g enters the gradients of the losses at the output projection."""
import torch

from head_util import inputs


def label_rows(rows, device="cuda"):
    """A cross entropy whose labels are rows of weights hundreds of times the others' size: grad_hidden is made of g at the label, and so is its error."""
    s = inputs(rows, 64, 600, seed=12, std=0.001, device=device)
    gen = torch.Generator().manual_seed(12)
    labels = torch.randperm(600, generator=gen)[:rows]
    w = s["weights"].float().cpu()
    w[labels] = torch.randn(rows, 64, generator=gen) * 0.3
    s["weights"] = w.to(s["weights"].dtype).to(device)
    s["w"], s["labels"] = s["weights"].double(), labels.to(device)
    s["hidden"] = torch.randn(rows, 64, generator=gen).to(s["hidden"].dtype).to(device)
    return s


def apart_from_the_label(s, want):
    """`want` (head_util's exact, g in one term) with grad_hidden's bound for a g whose rounding to one term is made good at the label: there
    the 2^-8 is 2^-22, that of an fp32 product and sum."""
    g = s["grad_ce"].double().abs() * -torch.expm1(-want["ce"])           # of the label's logit: a (1 - p)
    at = g[:, None] * s["w"][s["labels"]].abs()
    return dict(want, grad_hidden_tol=want["grad_hidden_tol"] - at * (2.0 ** -8 - 2.0 ** -22))
