"""The losses at the output projection on each of the ways that the library takes them: few rows read past LDS or through tiles, rows in
two terms, the tile shapes, hidden dimensions that their tiles leave partly empty, vocabularies of many groups and pieces.  Bounds as in
head_util."""
import pytest
import torch

from head_util import DTYPE, exact, inputs
from test_gpu_head import check, head_for

pytestmark = pytest.mark.gpu

FORMATS = [("bf16", 0, "fp32"), ("fp32", 0, "fp32"), ("fp8", 64, "fp32"), ("int4", 64, "bf16"), ("fp8", 40, "bf16"), ("int4", 1 << 30, "fp32")]


@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 63, 64])
@pytest.mark.parametrize("weights,group,scales", FORMATS)
def test_few_rows(rows, weights, group, scales):
    for dim, vocab in ((160, 1030), (96, 40000)):
        check(inputs(rows, dim, vocab, weights=weights, group=group, scales=scales, top_k=3, tau=2.0, seed=rows + dim, ignored=0.2 if rows > 4 else 0.0))


@pytest.mark.parametrize("rows,dim", [(40, 2560), (64, 1280), (20, 5120), (3, 5200)])
def test_few_rows_that_fill_lds(rows, dim):
    """Hidden states that fit LDS, only just, or not."""
    check(inputs(rows, dim, 700, seed=dim, std=0.02))


@pytest.mark.parametrize("rows", [65, 128, 129, 300])
@pytest.mark.parametrize("dim", [64, 192, 328, 576])
def test_large_tiles(rows, dim):
    """Enough of the vocabulary for the large tiles, with a last one that is partly empty."""
    check(inputs(rows, dim, 33100, top_k=2, tau=1.5, seed=rows + dim, ignored=0.1))


@pytest.mark.parametrize("hidden,weights,grad_weights", [("fp32", "fp32", "fp32"), ("bf16", "fp32", "fp32"), ("fp32", "bf16", "bf16"), ("bf16", "fp8", "fp32")])
@pytest.mark.parametrize("dim", [77, 192, 520])
def test_planes_in_large_tiles(hidden, weights, grad_weights, dim):
    check(inputs(260, dim, 33001, hidden=hidden, weights=weights, group=64, top_k=2, tau=1.0, seed=dim), grad_weights=DTYPE[grad_weights])


def test_rows_share_nothing():
    """Upstream gradients of very different sizes and signs, zero in the first row: what g is kept divided by is the first row's."""
    for rows in (2, 40, 200):
        for first in (0.0, 1e-30, 1e25, -3.0):
            s = inputs(rows, 64, 600, top_k=3, tau=2.0, seed=rows)
            s["grad_ce"] = s["grad_ce"] * 10.0 ** torch.linspace(-4, 4, rows, device="cuda")
            s["grad_ce"][0], s["grad_kd"][0] = first, 0.0
            check(s)


def test_offsets_past_32_bits():
    """Weights of more than 2^32 bytes: the losses and gradients of the last rows of the vocabulary."""
    vocab, dim, rows = (1 << 24) - 3, 136, 3
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda").normal_(0, 0.05, generator=gen)
    hidden = torch.randn(rows, dim, device="cuda", generator=gen).bfloat16()
    labels = torch.tensor([vocab - 1, vocab - 2, 0], device="cuda")
    s = dict(rows=rows, dim=dim, vocab=vocab, fmt=2, group=0, scales=None, tau=1.0, top_k=0, labels=labels, top_ids=None, top_logits=None, weights=w, hidden=hidden)
    head = head_for(s)
    ce, _ = head.forward(hidden, labels)
    gh, gw = head.backward(torch.full((rows,), 1.0 / rows, device="cuda"))
    total, zy, top, grad = torch.zeros(rows, dtype=torch.float64, device="cuda"), [], vocab - 4096, torch.zeros(rows, dim, dtype=torch.float64, device="cuda")
    for lo in range(0, vocab, 1 << 20):
        part = w[lo:lo + (1 << 20)].double()
        e = torch.exp(hidden.double() @ part.t())
        total += e.sum(1)
        grad += e @ part
    z = (hidden.double() * w[labels].double()).sum(1)
    # (fp32 statistics of 2^24 terms: within 2^-16 of a loss of 17)
    assert ((ce.double() - (torch.log(total) - z)).abs() <= 2.0 ** -12).all()
    grad = (grad / total[:, None] - w[labels].double()) / rows
    assert ((gh.double() - grad).norm() <= 2.0 ** -7 * grad.norm())
    p = torch.exp(hidden.double() @ w[top:].double().t()) / total[:, None]
    for t in range(2):
        p[t, labels[t] - top] -= 1
    want = p.t() @ hidden.double() / rows
    assert (gw[top:].double() - want).norm() <= 2.0 ** -7 * want.norm()


def test_refusals_of_the_harness():
    s = inputs(8, 64, 300, top_k=2, seed=1)
    head = head_for(s)
    ok = dict(hidden=s["hidden"], labels=s["labels"], top_ids=s["top_ids"], top_logits=s["top_logits"])
    head.forward(**ok)
    for name, bad in (("hidden", s["hidden"].float()), ("hidden", s["hidden"][:7]), ("hidden", s["hidden"].t().contiguous().t()), ("hidden", s["hidden"][:1].expand(8, 64)),
                      ("labels", s["labels"].int()), ("labels", None), ("top_ids", s["top_ids"].long()), ("top_logits", s["top_logits"].half()), ("hidden", s["hidden"].cpu()),
                      ("top_logits", torch.zeros(8, 4, device="cuda")[:, :2])):
        with pytest.raises(ValueError):
            head.forward(**{**ok, name: bad})
    with pytest.raises(ValueError):
        head.backward(s["grad_ce"].double(), s["grad_kd"])
    with pytest.raises(RuntimeError):
        head_for(s, training=False).backward(s["grad_ce"], s["grad_kd"])
    with pytest.raises(ValueError):
        head_for(s, weights=s["weights"].float())


def test_training_matches_exact_after_a_step():
    """The handle is used again with other inputs: nothing of the first call is left."""
    a, b = inputs(50, 64, 900, top_k=4, tau=2.0, seed=61), inputs(50, 64, 900, top_k=4, tau=2.0, seed=62, ignored=0.5)
    b["weights"], b["w"] = a["weights"], a["w"]
    head = head_for(a)
    head.forward(a["hidden"], a["labels"], a["top_ids"], a["top_logits"])
    head.backward(a["grad_ce"], a["grad_kd"])
    head.forward(b["hidden"], b["labels"], b["top_ids"], b["top_logits"])
    gh, gw = head.backward(b["grad_ce"], b["grad_kd"])
    from head_util import hold
    want = exact(b)
    hold(head.ce, want, "ce"); hold(head.kd, want, "kd"); hold(gh, want, "grad_hidden"); hold(gw, want, "grad_weights")


@pytest.mark.parametrize("fmt", ["fp8", "int4"])
def test_the_example_learns(fmt):
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from train_head import train
    losses = train(steps=30, rows=256, fmt=fmt)
    assert losses[-1][0] < 0.8 * losses[0][0] and losses[-1][1] < 0.8 * losses[0][1]
