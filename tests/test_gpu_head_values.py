"""The losses at the output projection where a value is easily lost: losses below zero, teachers whose logits lie at the ends of their type.
Bounds as in head_util."""
import pytest
import torch

from head_util import DTYPE, exact, inputs
from test_gpu_head import check, head_for

pytestmark = pytest.mark.gpu


def confident(rows, dim, vocab, height, std=0.05, **kw):
    """Inputs whose hidden states give the label a logit of about `height`, the others' about 0."""
    s = inputs(rows, dim, vocab, std=std, **kw)
    s["hidden"] = (s["w"][s["labels"]] * (height / (dim * std * std))).to(s["hidden"].dtype)
    return s


@pytest.mark.parametrize("rows", [5, 64, 200])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("weights", ["bf16", "fp8"])
def test_a_distillation_loss_below_zero(rows, tau, weights):
    """An id that comes up k times with equal logits has 1/k of q in each entry: where the student gives it all its weight, kd is -tau^2 ln k."""
    for k in (2, 7):
        s = confident(rows, 64, 500, 40.0 * tau, weights=weights, top_k=k, tau=tau, seed=rows + k)
        s["top_ids"] = s["labels"][:, None].repeat(1, k).int()
        s["top_logits"] = torch.full((rows, k), 1.5, device="cuda")
        assert (exact(s)["kd"] < -0.5).all()
        check(s)
        # beside an ordinary entry, and in a loss of its own
        s["top_ids"][:, k - 1] = (s["labels"] + 1).int() % 500
        check(s)
        check(dict(s, labels=None, grad_ce=None))


def rows_of_nan(rows, **kw):
    """A row whose only entries with a logit are NaN, one with -inf beside it, and one with an ordinary entry."""
    s = inputs(rows, 64, 500, top_k=3, seed=7, **kw)
    nan, none = float("nan"), float("-inf")
    s["top_logits"][1] = nan
    s["top_logits"][2] = torch.tensor([none, nan, none])
    s["top_logits"][3] = torch.tensor([1.0, nan, 2.0])
    s["top_ids"][4], s["top_logits"][4] = -1, nan               # absent: no entry at all
    return s


@pytest.mark.parametrize("rows", [6, 200])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_a_teacher_of_nan(rows, tau):
    """A present entry that is no number makes its row's distillation loss none, and its gradient; other rows are as they were."""
    s = rows_of_nan(rows, tau=tau)
    head = head_for(s)
    ce, kd = head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
    gh, _ = head.backward(s["grad_ce"], s["grad_kd"])
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[1:4] = True
    assert torch.isnan(kd[bad]).all() and torch.isnan(gh[bad]).any(1).all()
    assert torch.isfinite(kd[~bad]).all() and torch.isfinite(gh[~bad]).all() and torch.isfinite(ce).all() and kd[4] == 0


@pytest.mark.parametrize("top", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [0.25, 0.75, 1.0, 3.0])
@pytest.mark.parametrize("rows", [8, 130])
def test_logits_at_the_ends_of_their_type(rows, tau, top):
    """The lowest value is a mask as -inf is, but in a row of nothing else all entries are alike; large logits count by their differences."""
    s = inputs(rows, 64, 500, top_k=4, tau=tau, top=top, seed=9)
    lowest = torch.finfo(DTYPE[top]).min
    s["top_logits"][1] = lowest
    s["top_logits"][2, 1:3] = lowest
    s["top_logits"][3] = -lowest
    s["top_logits"][4, 0], s["top_logits"][4, 1:] = 2.0 ** 127, lowest
    s["top_logits"][5] = torch.tensor([lowest, lowest, float("-inf"), float("-inf")])
    check(s)
    check(dict(s, labels=None, grad_ce=None))


@pytest.mark.parametrize("rows", [1, 40, 200])
@pytest.mark.parametrize("weights", ["bf16", "fp32", "fp8", "int4"])
@pytest.mark.parametrize("loss", ["ce", "kd"])
def test_no_probability_is_above_one(rows, weights, loss):
    """The entries' logits and the sum over the vocabulary round apart: where the student is sure, the gradient at the label may come out as
    nothing, but not with the wrong sign."""
    s = confident(rows, 512, 3000, 60.0, weights=weights, labels=True, top_k=1, tau=1.0, seed=rows)
    s["labels"] = torch.randperm(3000, generator=torch.Generator().manual_seed(rows))[:rows].cuda()
    s["hidden"] = (s["w"][s["labels"]] * (60.0 / (512 * 0.05 ** 2))).bfloat16()
    s["grad_ce"], s["grad_kd"] = torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
    s["top_ids"] = s["labels"][:, None].int()
    if loss == "ce":
        s.update(top_k=0, top_ids=None, top_logits=None, grad_kd=None)
    label = s["labels"]
    if loss == "kd":
        s.update(labels=None, grad_ce=None)
    head = head_for(s, grad_weights=torch.float32)
    head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
    _, gw = head.backward(s["grad_ce"], s["grad_kd"])
    along = (gw[label].double() * s["hidden"].double()).sum(1)
    # (g h.h, where h.h is above 1000; the other rows' share is below e^-30)
    assert (along <= 1e-9).all()
