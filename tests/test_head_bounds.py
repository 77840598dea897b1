"""The bounds that the GPU tests of the losses at the output projection hold gradients to tell g's terms apart: float64 results whose g is rounded to fewer bfloat16
terms than the library promises fall outside them, and those with the promised ones inside.  No GPU is needed."""
import pytest
import torch

from head_terms import apart_from_the_label, label_rows
from head_util import exact, hold, inputs


def rounded(s, terms, mend_label=False):
    """grad_hidden and grad_weights of a cross entropy in float64 but for g, which is `terms` bfloat16 of itself over the first row's upstream gradient;
    `mend_label`: grad_hidden takes g at the label as it is."""
    h, w = s["hidden"].double(), s["w"]
    a = s["grad_ce"].double()[:, None]
    g = a * torch.softmax(h @ w.t(), 1)
    g.scatter_add_(1, s["labels"][:, None], -a)
    unit = a[0].abs()
    kept, rest = torch.zeros_like(g), g / unit
    for _ in range(terms):
        term = rest.bfloat16().double()
        kept, rest = kept + term, rest - term
    kept = kept * unit
    gh, gw = kept @ w, kept.t() @ h
    if mend_label:
        gh = gh + (g - kept).gather(1, s["labels"][:, None]) * w[s["labels"]]
    return gh.bfloat16(), gw.bfloat16()


@pytest.mark.parametrize("rows", [1, 20, 64])
@pytest.mark.parametrize("weights", ["bf16", "fp8"])
def test_a_lost_second_term_shows(rows, weights):
    s = inputs(rows, 96, 1030, weights=weights, group=32, seed=5, device="cpu")
    want = exact(s, quantized=weights == "fp8", g_bits=16)
    for t, name in zip(rounded(s, 2), ("grad_hidden", "grad_weights")):
        hold(t, want, name)
    for t, name in zip(rounded(s, 1), ("grad_hidden", "grad_weights")):
        if rows == 1 and name == "grad_hidden":                 # (96 numbers, none of which need be far off)
            continue
        with pytest.raises(AssertionError, match="its bound"):
            hold(t, want, name)


def test_a_lost_correction_at_the_label_shows():
    s = label_rows(130, device="cpu")
    want = apart_from_the_label(s, exact(s))
    hold(rounded(s, 1, mend_label=True)[0], want, "grad_hidden")
    with pytest.raises(AssertionError, match="its bound"):
        hold(rounded(s, 1)[0], want, "grad_hidden")
