"""The terms in which the logits' gradient enters the gradients of the losses at the output projection: two bfloat16 of up to 64 rows, one of more, with what
that leaves at the label added to grad_hidden.  Bounds as in head_util, for those terms; test_head_bounds.py shows that a lost term falls outside them."""
import pytest
import torch

from head_terms import apart_from_the_label, label_rows
from head_util import exact, hold, inputs
from test_gpu_head import head_for

pytestmark = pytest.mark.gpu


def gradients(s):
    print(f"head rows={s['rows']} dim={s['dim']} vocab={s['vocab']} fmt={s['fmt']} top_k={s['top_k']}", flush=True)
    head = head_for(s)
    head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
    return head.backward(s["grad_ce"], s["grad_kd"])


@pytest.mark.parametrize("rows", [1, 2, 20, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("weights,group", [("bf16", 0), ("fp32", 0), ("fp8", 32), ("int4", 32), ("fp8", 40)])
@pytest.mark.parametrize("top_k", [0, 3])
def test_two_terms_of_g(rows, weights, group, top_k):
    for dim, vocab in ((96, 1030), (77, 300)):
        s = inputs(rows, dim, vocab, weights=weights, group=group, top_k=top_k, tau=2.0, seed=5, ignored=0.2 if rows > 4 else 0.0)
        gh, gw = gradients(s)
        want = exact(s, quantized=weights in ("fp8", "int4"), g_bits=16)
        hold(gh, want, "grad_hidden")
        hold(gw, want, "grad_weights")


@pytest.mark.parametrize("rows", [65, 130, 300])
def test_what_rounding_leaves_of_g_at_the_label(rows):
    s = label_rows(rows)
    gh, gw = gradients(s)
    want = exact(s)
    hold(gw, want, "grad_weights")
    hold(gh, apart_from_the_label(s, want), "grad_hidden")
