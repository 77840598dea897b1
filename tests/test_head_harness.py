"""What HeadLoss gives to the library, call by call, without a GPU: the library's two calls are replaced by ones that keep the descriptor they get."""
import pytest
import torch

from head_util import inputs


@pytest.fixture
def calls(monkeypatch):
    """The library's calls as (name, {field: value}) in their order; nothing is launched."""
    from paper_2601_22101_amd import harness
    made = []
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)          # the tensors here stand for ones on a GPU

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


def test_a_refused_forward_changes_nothing(calls):
    """Inputs are looked at before any of them gets into the descriptor: after a refusal backward() has the last forward()'s, all of them."""
    s, other = inputs(6, 64, 300, top_k=3, device="cpu"), inputs(6, 64, 300, top_k=3, seed=1, device="cpu")
    head = head_for(s)
    head.forward(**arguments(s))
    kept = head._inputs
    good = arguments(other)
    for name, bad in (("labels", other["labels"].int()), ("labels", None), ("top_ids", other["top_ids"].long()), ("top_logits", other["top_logits"].half()),
                      ("top_logits", torch.zeros(6, 5)[:, :3])):
        with pytest.raises(ValueError):
            head.forward(**{**good, name: bad})
        assert all(a is b for a, b in zip(head._inputs, kept))
    head.backward(s["grad_ce"], s["grad_kd"])
    for name, t in arguments(s).items():
        assert calls[-1][1][name] == t.data_ptr(), name


def test_a_forward_that_fails_leaves_nothing_to_differentiate(calls, monkeypatch):
    """A call that the library refuses, or fails, may have written some of what the backward pass reads."""
    from paper_2601_22101_amd import binding, harness
    s = inputs(6, 64, 300, device="cpu")
    head = head_for(s)
    head.forward(s["hidden"], s["labels"])

    def fails(*args):
        raise binding.EcoError(binding.ECO_EHIP, "head kernel launch")

    with monkeypatch.context() as m:
        m.setattr(harness.eco, "eco_head_loss", fails)
        with pytest.raises(binding.EcoError):
            head.forward(s["hidden"], s["labels"])
    with pytest.raises(RuntimeError):
        head.backward(s["grad_ce"])
    head.forward(s["hidden"], s["labels"])
    head.backward(s["grad_ce"])


def test_a_refused_gradient_changes_nothing(calls):
    s = inputs(6, 64, 300, top_k=3, device="cpu")
    head = head_for(s)
    head.forward(**arguments(s))
    with pytest.raises(ValueError):
        head.backward(s["grad_ce"], s["grad_kd"].double())
    assert head.head.grad_ce is None and head.head.grad_kd is None


@pytest.mark.parametrize("weights", ["bf16", "fp8"])
def test_weights_off_the_gpu_are_refused(weights):
    """Their addresses are no memory of a kernel's."""
    with pytest.raises(ValueError, match="GPU"):
        head_for(inputs(6, 64, 300, weights=weights, device="cpu"))


def test_scales_off_the_weights_device_are_refused(calls):
    s = inputs(6, 64, 300, weights="fp8", device="cpu")
    with pytest.raises(ValueError, match="scales"):
        head_for(dict(s, scales=s["scales"].to("meta")))
    with pytest.raises(ValueError, match="scales"):
        head_for(dict(s, scales=s["scales"].half()))
    head_for(s)


def test_memory_of_a_call_on_another_stream_is_not_handed_out_again(calls, monkeypatch):
    """Work on `stream` may be under way when a tensor that it reads or writes is let go: the allocator has to know of it."""
    from types import SimpleNamespace
    s, stream = inputs(6, 64, 300, weights="fp8", top_k=3, device="cpu"), SimpleNamespace(cuda_stream=0x5000)
    head = head_for(s)
    noted = set()
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, on: noted.add((t.data_ptr(), on.cuda_stream)))
    head.forward(**arguments(s))
    head.backward(s["grad_ce"], s["grad_kd"])
    assert not noted                                            # on the current stream, whose allocations follow each other
    both = [head.weights, head.scales, head.lse, head.lse_tau, head.picked, head.workspace, *arguments(s).values()]
    head.forward(**arguments(s), stream=stream)
    assert noted == {(t.data_ptr(), 0x5000) for t in (*both, head.ce, head.kd)}
    noted.clear()
    head.backward(s["grad_ce"], s["grad_kd"], stream=stream)
    assert noted == {(t.data_ptr(), 0x5000) for t in (*both, s["grad_ce"], s["grad_kd"], head.grad_hidden, head.grad_weights)}
