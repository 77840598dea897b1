"""HeadLoss on a stream that is not the current one."""
import pytest
import torch

from head_util import exact, hold, inputs
from test_gpu_head import head_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("as_address", [False, True])
def test_inputs_that_are_let_go_while_their_call_waits(as_address):
    """Inputs of this stream, a call on another that is still busy, and new tensors of the same sizes: they are given other memory."""
    s, other = (inputs(40, 64, 2000, top_k=3, tau=2.0, seed=seed) for seed in (1, 2))
    head = head_for(s)
    stream = torch.cuda.Stream()
    on = stream.cuda_stream if as_address else stream
    hidden, grad = s["hidden"].clone(), s["grad_ce"].clone()
    at = {hidden.data_ptr(), grad.data_ptr()}
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)
    head.forward(hidden, s["labels"], s["top_ids"], s["top_logits"], stream=on)
    gh, gw = head.backward(grad, s["grad_kd"], stream=on)
    with torch.cuda.stream(stream):
        got = [t.clone() for t in (head.ce, head.kd, gh, gw)]
    head.forward(other["hidden"], other["labels"], other["top_ids"], other["top_logits"], stream=on)      # (lets go of the first ones)
    del hidden, grad
    new = [torch.full_like(t, float("nan")) for t in (s["hidden"], s["grad_ce"]) for _ in range(4)]
    assert not stream.query() and not at & {t.data_ptr() for t in new}
    stream.synchronize()
    want = exact(s)
    for t, name in zip(got, ("ce", "kd", "grad_hidden", "grad_weights")):
        hold(t, want, name)
    hold(head.ce, exact(dict(other, w=s["w"])), "ce")               # (the weights are the first ones)


def test_the_default_stream_by_its_address():
    s = inputs(7, 64, 300, seed=3)
    head = head_for(s)
    head.forward(s["hidden"], s["labels"], stream=0)
    torch.cuda.synchronize()
    hold(head.ce, exact(s), "ce")
