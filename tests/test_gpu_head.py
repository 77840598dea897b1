"""The losses at the output projection against float64, on the GPU: sizes around the tiles, formats and types, masks, strides,
streams and graphs.  The bounds are head_util's."""
import pytest
import torch

from head_util import DTYPE, FMT, exact, hold, inputs

pytestmark = pytest.mark.gpu


def head_for(s, training=True, grad_weights=torch.bfloat16, **kw):
    from paper_2601_22101_amd import harness
    return harness.HeadLoss(s["rows"], s["vocab"], s["dim"], weights=kw.get("weights", s["weights"]), fmt=s["fmt"], scales=s["scales"], group_size=s["group"],
                            hidden_dtype=s["hidden"].dtype, labels=s["labels"] is not None, top_k=s["top_k"], temperature=s["tau"],
                            training=training, grad_weights_dtype=grad_weights)


def check(s, grad_weights=torch.bfloat16, hidden=None, **kw):
    print(f"head rows={s['rows']} dim={s['dim']} vocab={s['vocab']} fmt={s['fmt']} hidden={s['hidden'].dtype} top_k={s['top_k']} tau={s['tau']}", flush=True)
    head = head_for(s, grad_weights=grad_weights, **kw)
    ce, kd = head.forward(s["hidden"] if hidden is None else hidden, s["labels"], s["top_ids"], s["top_logits"])
    gh, gw = head.backward(s["grad_ce"], s["grad_kd"])
    torch.cuda.synchronize()
    g_bits = 8 if s["hidden"].dtype == torch.bfloat16 and grad_weights == torch.bfloat16 else 22
    want = exact(s, quantized=s["scales"] is not None, g_bits=g_bits)
    if ce is not None:
        hold(ce, want, "ce")
        hold(head.lse, want, "lse")
    if kd is not None:
        hold(kd, want, "kd")
    hold(head.picked, want, "picked")
    hold(gh, want, "grad_hidden")
    hold(gw, want, "grad_weights")
    return head


@pytest.mark.parametrize("rows,dim,vocab", [(1, 8, 1), (1, 64, 300), (2, 32, 257), (3, 40, 128), (31, 576, 1000), (32, 64, 255), (33, 96, 513), (64, 128, 256),
                                            (127, 72, 129), (128, 512, 1024), (129, 1152, 640), (255, 64, 4097), (256, 200, 333), (257, 1024, 777), (700, 320, 2050)])
@pytest.mark.parametrize("loss", ["ce", "kd", "both", "both1"])
def test_sizes(rows, dim, vocab, loss):
    k = 0 if loss == "ce" else min(vocab, 5)
    check(inputs(rows, dim, vocab, labels=loss != "kd", top_k=k, tau=1.0 if loss in ("ce", "both1") else 2.0, seed=rows + dim + vocab))


@pytest.mark.parametrize("hidden", ["bf16", "fp32"])
@pytest.mark.parametrize("weights,group,scales", [("bf16", 0, "fp32"), ("fp32", 0, "fp32"), ("fp8", 128, "fp32"), ("fp8", 96, "bf16"), ("fp8", 32, "fp32"),
                                                  ("int4", 128, "bf16"), ("int4", 96, "fp32"), ("int4", 1 << 30, "fp32"), ("fp8", 1 << 30, "fp32")])
@pytest.mark.parametrize("grad_weights", ["bf16", "fp32"])
def test_formats(hidden, weights, group, scales, grad_weights):
    for rows, dim, vocab, seed in ((5, 96, 700, 1), (150, 96, 1100, 2)):
        check(inputs(rows, dim, vocab, hidden=hidden, weights=weights, group=group, scales=scales, top_k=4, tau=1.5, seed=seed, ignored=0.2),
              grad_weights=DTYPE[grad_weights])


@pytest.mark.parametrize("dim", [1, 3, 7, 9, 33, 77, 100, 515])
@pytest.mark.parametrize("weights,group", [("bf16", 0), ("fp32", 0), ("fp8", 64), ("int4", 64)])
def test_odd_dimensions(dim, weights, group):
    for rows in (2, 130):
        check(inputs(rows, dim, 413, weights=weights, group=group, top_k=3, tau=1.0, seed=dim))


@pytest.mark.parametrize("top_k,top", [(1, "fp32"), (2, "bf16"), (63, "bf16"), (64, "fp32"), (65, "fp32"), (300, "bf16"), (1024, "fp32")])
def test_numbers_of_entries(top_k, top):
    for rows in (1, 40):
        check(inputs(rows, 64, 1500, top_k=top_k, top=top, tau=2.5, seed=top_k))


@pytest.mark.parametrize("tau", [0.25, 1.0, 8.0])
def test_temperatures(tau):
    check(inputs(70, 64, 900, labels=False, top_k=9, tau=tau, seed=3))
    check(inputs(70, 64, 900, top_k=9, tau=tau, seed=4))


def test_masks():
    """Labels and entries that are none, rows that take no part and hold what is not a number, entries with a logit of -inf and garbage under
    absent ids, ids that come up twice."""
    for rows, hidden in ((12, "bf16"), (200, "bf16"), (200, "fp32")):
        s = inputs(rows, 72, 777, hidden=hidden, top_k=6, tau=2.0, seed=11, ignored=0.3)
        v = s["vocab"]
        s["labels"][0], s["labels"][1], s["labels"][2] = v, -1, 2 ** 62
        s["top_ids"][3] = -1
        s["top_ids"][4], s["top_logits"][4] = torch.arange(6, device="cuda").int(), float("-inf")
        s["top_ids"][5, 2:] = v
        s["top_logits"][5, 2:] = float("nan")
        s["top_ids"][6], s["top_logits"][6, 1] = 5, float("-inf")
        s["top_ids"][7, 3] = s["top_ids"][7, 0]
        if s["labels"][8] >= 0:
            s["top_ids"][8, 1] = s["labels"][8].int()
        s["labels"][9], s["top_ids"][9] = -100, 2 ** 31 - 1
        s["labels"][10], s["top_ids"][10], s["top_logits"][10] = -100, 3, float("-inf")
        s["hidden"][9], s["hidden"][10] = float("nan"), float("inf")
        clean = dict(s, hidden=torch.where(torch.isfinite(s["hidden"]), s["hidden"], 0.0))
        want_rows = [9, 10]
        head = check(clean, hidden=s["hidden"])
        assert (head.ce[want_rows] == 0).all() and (head.kd[want_rows] == 0).all() and (head.grad_hidden[want_rows] == 0).all()


def test_no_row_takes_part():
    for rows in (1, 3, 300):
        s = inputs(rows, 64, 500, top_k=3, seed=5)
        s["labels"][:] = -100
        s["top_ids"][:] = -1
        s["hidden"][:] = float("nan")
        head = head_for(s)
        head.grad_hidden.fill_(7)
        head.grad_weights.fill_(7)
        ce, kd = head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
        gh, gw = head.backward(s["grad_ce"], s["grad_kd"])
        for t in (ce, kd, gh, gw, head.lse, head.lse_tau, head.picked):
            assert (t == 0).all()


def test_one_loss_without_a_gradient():
    for drop in ("grad_ce", "grad_kd"):
        for tau in (1.0, 2.0):
            check(dict(inputs(60, 64, 500, top_k=3, tau=tau, seed=6), **{drop: None}))


def test_large_logits():
    """Logits of several hundreds: the sums need their maximum."""
    check(inputs(40, 512, 3000, std=1.0, top_k=3, tau=1.0, seed=8, hidden="fp32", weights="fp32"), grad_weights=torch.float32)
    s = inputs(40, 512, 3000, std=1.0, top_k=3, tau=4.0, seed=9)
    check(s)


def test_strides_and_offsets():
    """Rows with gaps, hidden states that start off 16 bytes, outputs with gaps whose padding stays as it was."""
    from paper_2601_22101_amd import binding as eco
    for dim, odd in ((64, 3), (64, 8), (77, 1)):
        s = inputs(50, dim, 600, top_k=4, tau=2.0, seed=dim + odd)
        wide = torch.full((51, dim + odd), float("nan"), dtype=torch.bfloat16, device="cuda")
        hidden = wide[1:, odd:]
        hidden.copy_(s["hidden"])
        weights = torch.full((600, dim + odd), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :dim]
        weights.copy_(s["weights"])
        ids, logits = torch.full((50, 9), -1, dtype=torch.int32, device="cuda"), torch.full((50, 9), float("nan"), device="cuda")
        ids[:, 2:6], logits[:, 2:6] = s["top_ids"], s["top_logits"]
        head = check(dict(s, top_ids=ids[:, 2:6], top_logits=logits[:, 2:6]), hidden=hidden, weights=weights)
        gh = torch.full((50, dim + odd), 7.0, dtype=torch.bfloat16, device="cuda")
        gw = torch.full((600, dim + odd), 7.0, dtype=torch.bfloat16, device="cuda")
        h = head.head
        h.grad_hidden, h.grad_hidden_stride, h.grad_weights, h.grad_weights_stride = gh.data_ptr(), dim + odd, gw.data_ptr(), dim + odd
        eco.eco_head_loss_backward(h, head.workspace, head.workspace_bytes)
        assert torch.equal(gh[:, :dim], head.grad_hidden) and torch.equal(gw[:, :dim], head.grad_weights)
        assert (gh[:, dim:] == 7).all() and (gw[:, dim:] == 7).all()


@pytest.mark.parametrize("weights,group", [("bf16", 0), ("fp8", 128)])
def test_pieces_of_the_vocabulary(weights, group):
    """More rows and vocabulary than one piece holds."""
    check(inputs(3000, 64, 100500 if weights == "bf16" else 50300, weights=weights, group=group, top_k=2, tau=2.0, seed=21, ignored=0.1))


def test_differences():
    """The gradients against central differences of the losses themselves, in fp32."""
    s = inputs(6, 32, 200, hidden="fp32", weights="fp32", top_k=5, tau=2.0, seed=31)
    head = head_for(s, grad_weights=torch.float32)
    # the losses are good to 2^-20 (1 + lse) each and (sum of upstream gradients < 4): over a step of 2^-5 that is 2^-11; the third
    # derivative of a softmax's logarithm is below 1 in the direction's logit, which the weights' 0.3 and 32 dimensions keep below 2
    step, tol = 2.0 ** -5, 2.0 ** -10

    def total(hidden):
        ce, kd = head.forward(hidden, s["labels"], s["top_ids"], s["top_logits"])
        return float((ce.double() * s["grad_ce"].double()).sum() + (kd.double() * s["grad_kd"].double()).sum())

    total(s["hidden"])
    gh, gw = (t.clone() for t in head.backward(s["grad_ce"], s["grad_kd"]))
    gen = torch.Generator().manual_seed(5)
    for _ in range(8):
        d = torch.randn(6, 32, generator=gen).cuda()
        d /= d.norm()
        diff = (total(s["hidden"] + step * d) - total(s["hidden"] - step * d)) / (2 * step)
        assert abs(diff - float((gh.double() * d.double()).sum())) <= tol
        e = torch.randn(200, 32, generator=gen).cuda()
        e /= e.norm()
        head.weights += step * e
        up = total(s["hidden"])
        head.weights -= 2 * step * e
        down = total(s["hidden"])
        head.weights += step * e
        assert abs((up - down) / (2 * step) - float((gw.double() * e.double()).sum())) <= tol


def test_same_bits_again_and_on_another_stream():
    s = inputs(300, 128, 5000, top_k=8, tau=2.0, seed=41, ignored=0.2)
    head = head_for(s)

    def both():
        ce, kd = head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
        gh, gw = head.backward(s["grad_ce"], s["grad_kd"])
        return [t.clone() for t in (ce, kd, gh, gw)]

    first = both()
    head.workspace.fill_(255)                       # nothing of the workspace is kept from one call to the next
    second = both()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        third = both()
    stream.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_graph():
    s = inputs(90, 64, 2000, top_k=8, tau=2.0, seed=42)
    other = inputs(90, 64, 2000, top_k=8, tau=2.0, seed=43)
    head = head_for(s)
    hidden, labels = s["hidden"].clone(), s["labels"].clone()

    def both():
        head.forward(hidden, labels, s["top_ids"], s["top_logits"])
        head.backward(s["grad_ce"], s["grad_kd"])

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for x in (s, other, s, other):
        hidden.copy_(x["hidden"])
        labels.copy_(x["labels"])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (head.ce, head.kd, head.grad_hidden, head.grad_weights)]
        both()
        torch.cuda.synchronize()
        for a, b in zip(got, (head.ce, head.kd, head.grad_hidden, head.grad_weights)):
            assert torch.equal(a, b)


def test_the_step_reads_the_gradient():
    """The projection of a quantized model learns its batch: losses, gradients and eco_step on the same arrays."""
    from paper_2601_22101_amd import binding as eco
    rows, dim, vocab = 64, 128, 512
    s = inputs(rows, dim, vocab, weights="fp8", group=128, top_k=4, tau=2.0, seed=51, std=0.02)
    s["grad_ce"], s["grad_kd"] = torch.full((rows,), 1.0 / rows, device="cuda"), torch.full((rows,), 0.5 / rows, device="cuda")
    head = head_for(s)
    m, v = torch.zeros(vocab * dim, device="cuda"), torch.zeros(vocab * dim, device="cuda")
    layout = eco.make_hparams(block_size=128)
    tensor = eco.make_tensor(s["weights"], s["scales"], head.grad_weights, m, v, vocab * dim, 0, eco.ECO_FMT_FP8_E4M3)
    losses = []
    with eco.Plan([tensor], layout) as plan:
        for k in range(1, 31):
            ce, kd = head.forward(s["hidden"], s["labels"], s["top_ids"], s["top_logits"])
            losses.append(float(ce.mean() + 0.5 * kd.mean()))
            head.backward(s["grad_ce"], s["grad_kd"])
            plan.step(eco.make_hparams(lr=3e-3, step=k, block_size=128))
    assert losses[-1] < 0.8 * losses[0] and all(b < a + 0.05 for a, b in zip(losses, losses[1:]))


def test_fmt_names():
    from paper_2601_22101_amd import binding as eco
    assert FMT == {"fp8": eco.ECO_FMT_FP8_E4M3, "int4": eco.ECO_FMT_INT4, "bf16": eco.ECO_FMT_BF16_PLAIN, "fp32": eco.ECO_FMT_FP32_IDENTITY}
