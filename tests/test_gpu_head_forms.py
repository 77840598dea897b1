"""The losses at the output projection with weights that are not bf16: few rows' grad_hidden read from the weights as they lie, and logits of fp16
planes of rows that were scaled.  Bounds as in head_util."""
import pytest
import torch

from head_util import DTYPE, inputs
from test_gpu_head import check, head_for

pytestmark = pytest.mark.gpu

FORMS = [("fp32", 0, "fp32"), ("fp8", 64, "fp32"), ("int4", 64, "bf16"), ("fp8", 24, "bf16"), ("int4", 136, "fp32"), ("fp8", 1 << 30, "fp32"), ("int4", 528, "bf16")]


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64])
@pytest.mark.parametrize("weights,group,scales", FORMS)
@pytest.mark.parametrize("hidden,grad", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_grad_hidden_of_few_rows(rows, weights, group, scales, hidden, grad):
    """Scale groups within rows, over several and of a whole row; columns that leave a wave's tile empty in part; vocabularies of less than a step and of
    many parts."""
    for dim, vocab in ((132, 15), (528, 1001), (64, 20011)):
        check(inputs(rows, dim, vocab, hidden=hidden, weights=weights, group=group, scales=scales, top_k=2, tau=2.0, seed=rows + dim + vocab, ignored=0.2 if rows > 4 else 0.0),
              grad_weights=DTYPE[grad])


@pytest.mark.parametrize("weights", ["fp32", "fp8", "int4"])
def test_rows_where_nothing_takes_part(weights):
    s = inputs(20, 64, 500, weights=weights, group=64, top_k=2, tau=2.0, seed=5)
    s["labels"].fill_(-100)
    s["top_ids"].fill_(-1)
    head = check(s)
    assert not head.ce.any() and not head.kd.any()


@pytest.mark.parametrize("rows", [20, 130, 300])
@pytest.mark.parametrize("hidden", ["bf16", "fp32"])
def test_rows_of_very_different_sizes(rows, hidden):
    """Hidden states and weights whose rows are powers of two apart, some of them past the range of an fp16 by far, and rows of zeros."""
    s = inputs(rows, 132, 900, hidden=hidden, weights="fp32", top_k=3, tau=1.0, seed=rows)
    h_scale = torch.tensor([1.0, 2.0 ** -40, 2.0 ** 3, 0.0], device="cuda").repeat(rows)[:rows, None]
    w_scale = torch.tensor([1.0, 2.0 ** -30, 2.0 ** -120, 0.0, 2.0 ** -2], device="cuda").repeat(900)[:900, None]
    s["hidden"] = (s["hidden"].float() * h_scale).to(s["hidden"].dtype)
    s["weights"] = s["weights"] * w_scale
    s["w"] = s["weights"].double()
    check(s, grad_weights=torch.float32)


def test_large_weights_against_small_hidden_states():
    s = inputs(90, 64, 700, hidden="fp32", weights="fp32", seed=8)
    s["weights"], s["hidden"] = s["weights"] * 2.0 ** 90, s["hidden"] * 2.0 ** -90
    s["w"] = s["weights"].double()
    s["grad_ce"] = s["grad_ce"] * 2.0 ** -90
    head = head_for(s, grad_weights=torch.float32)
    ce, _ = head.forward(s["hidden"], s["labels"])
    from head_util import exact, hold
    hold(ce, exact(s), "ce")


@pytest.mark.parametrize("rows", [20, 200])
def test_a_nan_stays_in_its_row(rows):
    for weights in ("fp32", "fp8"):
        s = inputs(rows, 64, 400, hidden="fp32", weights=weights, group=64, seed=9)
        head = head_for(s, training=False)
        clean = head.forward(s["hidden"], s["labels"])[0].clone()
        s["hidden"][7, 3] = float("nan")
        s["hidden"][11, 5] = float("inf")
        s["labels"][7], s["labels"][11], s["labels"][12] = 1, 2, -100
        s["hidden"][12] = float("nan")
        ce = head.forward(s["hidden"], s["labels"])[0]
        others = torch.ones(rows, dtype=torch.bool, device="cuda")
        others[[7, 11, 12]] = False
        assert torch.isnan(ce[7]) and not torch.isfinite(ce[11]) and ce[12] == 0
        assert torch.equal(ce[others], clean[others])
