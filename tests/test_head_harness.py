"""What HeadLoss gives to the library, call by call, without a GPU: the library's two calls are replaced by ones that keep the descriptor they get."""
import pytest
import torch

from head_util import inputs


@pytest.fixture
def calls(monkeypatch):
    """The library's calls as (name, {field: value}) in their order; nothing is launched."""
    from paper_2601_22101_amd import harness
    made = []

    def keep(name):
        def call(head, workspace, workspace_bytes, stream=None):
            made.append((name, {f: getattr(head, f) for f, *_ in head._fields_}))
        return call

    for name in ("eco_head_loss", "eco_head_loss_backward"):
        monkeypatch.setattr(harness.eco, name, keep(name))
    return made


def head_for(s, **kw):
    from paper_2601_22101_amd import harness
    return harness.HeadLoss(s["rows"], s["vocab"], s["dim"], weights=s["weights"], fmt=s["fmt"], scales=s["scales"], group_size=s["group"],
                            hidden_dtype=s["hidden"].dtype, labels=s["labels"] is not None, top_k=s["top_k"], temperature=s["tau"], **kw)


def arguments(s):
    return dict(hidden=s["hidden"], labels=s["labels"], top_ids=s["top_ids"], top_logits=s["top_logits"])


@pytest.mark.parametrize("labels,top_k", [(True, 0), (False, 3), (True, 3)])
def test_backward_needs_a_forward(calls, labels, top_k):
    """Before it the object has no inputs, and no gradient is computed from anything else."""
    from paper_2601_22101_amd import binding
    s = inputs(6, 64, 300, labels=labels, top_k=top_k, device="cpu")
    head = head_for(s)
    with pytest.raises(RuntimeError):
        head.backward(s["grad_ce"], s["grad_kd"])
    assert not calls
    # the descriptor names none either: the library refuses it
    h = head.head
    assert not (h.hidden or h.labels or h.top_ids or h.top_logits)
    h.grad_ce = h.grad_kd = head.picked.data_ptr()
    assert binding.lib.eco_head_loss_backward(h, head.workspace.data_ptr() + 255 & ~255, head.workspace_bytes, None) == binding.ECO_EINVAL
    assert "null hidden" in binding.eco_last_error()
    head.forward(**arguments(s))
    head.backward(s["grad_ce"], s["grad_kd"])
    assert [name for name, _ in calls] == ["eco_head_loss", "eco_head_loss_backward"] and calls[1][1]["hidden"] == s["hidden"].data_ptr()
