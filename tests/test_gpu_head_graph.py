"""The losses at the output projection in a captured graph, on each of the ways that few rows and weights which are not bf16 take: replays with other inputs, and
with eager work between them, give the eager results."""
import pytest
import torch

from head_util import inputs
from test_gpu_head import head_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 40, 200])
@pytest.mark.parametrize("weights,group", [("bf16", 0), ("fp32", 0), ("fp8", 64), ("int4", 64)])
def test_replays(rows, weights, group):
    s, other = (inputs(rows, 128, 1500, weights=weights, group=group, top_k=4, tau=2.0, seed=seed, ignored=0.2 if rows > 1 else 0.0) for seed in (44, 45))
    head = head_for(s)
    names = ("hidden", "labels", "top_ids", "top_logits", "grad_ce", "grad_kd")
    held = {n: s[n].clone() for n in names}

    def both():
        head.forward(held["hidden"], held["labels"], held["top_ids"], held["top_logits"])
        head.backward(held["grad_ce"], held["grad_kd"])

    graph = torch.cuda.CUDAGraph()                              # (nothing has run before the capture)
    with torch.cuda.graph(graph):
        both()
    for x in (s, other, s, other):
        for n in names:
            held[n].copy_(x[n])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (head.ce, head.kd, head.grad_hidden, head.grad_weights)]
        head.workspace.fill_(255)
        both()
        torch.cuda.synchronize()
        for a, b in zip(got, (head.ce, head.kd, head.grad_hidden, head.grad_weights)):
            assert torch.equal(a, b)
