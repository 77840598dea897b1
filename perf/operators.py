"""The losses at the output projection of a language model, as cases that can be timed and compared: cross entropy with the
next token, distillation from a teacher's top logits, and their gradients, over the shapes that the embeddings of
`workloads/` have (and odd ones), from one token to thousands, with the projection in each of the library's weight formats.

With h_t a row of `hidden` and w_v a row of the weights (dec(code) * scale where they are quantized):
    z_tv = h_t . w_v
    ce_t = ln sum_v exp z_tv - z_t,label                         0 where the label is outside [0, vocab)
    q_tj = softmax over the present entries j of row t of teacher_logit / tau    (an entry is present where its id is in [0, vocab))
    kd_t = tau^2 sum_j q_tj (ln q_tj - ln p_t,id(j)),  p_t = softmax over the vocabulary of z_t / tau    0 where no entry is present
and for training, with the upstream gradients a_t = dL/dce_t and b_t = dL/dkd_t,
    g_tv = a_t (exp(z_tv - lse_t) - [v = label]) + b_t tau (p_tv - sum of q_tj over the entries with id v)
    grad_hidden = g W,  grad_weights = g^T hidden.

A case is a dict of plain values.  `op` is "score" (the losses) or "train" (the losses and both gradients); `labels` and `top_k`
say which of the two losses are there; `active` is the share of the rows that take part (the others have neither a label
nor a teacher's entries: prompts and padding); `weights` is a storage format, with scale groups of `group` elements.
"""
import math

import torch

own = False

IGNORED = -100
WEIGHT_STD = 0.02                     # as the workloads' weights
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _case(name, op, rows, dim, vocab, *, hidden="bf16", weights="bf16", group=0, scales="fp32", labels=True, top_k=0, tau=1.0, active=1.0):
    c = {"op": op, "rows": rows, "dim": dim, "vocab": vocab, "hidden": hidden, "weights": weights, "group": group, "scales": scales,
         "labels": labels, "top_k": top_k, "tau": tau, "active": active}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token's loss under a 30 M transformer's embedding: latency and one reading of the weights
        _case("score_one_token", "score", 1, 512, 32000),
        # a few tokens of a quantized student held against its teacher, DeepSeek-MoE-16B-shaped INT4 embedding
        _case("score_few_int4_kd", "score", 24, 2048, 102400, weights="int4", group=128, scales="bf16", labels=False, top_k=32, tau=2.0),
        # evaluation of a sparse-MoE model on a sequence of 2048 tokens
        _case("score_sequence", "score", 2048, 1024, 50304),
        # evaluation of a distilled student: ordinary number of rows, one short of a whole tile, 64 teacher entries
        _case("score_kd", "score", 4095, 512, 32000, labels=False, top_k=64),
        # one token of training with both losses, the paper's own sparse-MoE embedding: the smallest training call
        _case("train_one_token", "train", 1, 576, 32128, top_k=16, tau=2.0),
        # a short answer to fine-tune on: few rows, the widest vocabulary (Gemma-3-1B shapes)
        _case("train_short", "train", 67, 1152, 262144),
        # a batch of the paper's own sparse-MoE model, 40 % of it prompt
        _case("train_ce", "train", 2048, 576, 32128, active=0.6),
        # the same loss with everything in fp32
        _case("train_ce_fp32", "train", 1000, 512, 32000, hidden="fp32", weights="fp32"),
        # odd sizes everywhere, a projection kept in fp32 under bf16 activations, high temperature
        _case("train_odd_kd", "train", 333, 77, 5003, weights="fp32", top_k=7, tau=3.0, active=0.9),
        # distillation into the FP8 embedding of the benchmark's sparse-MoE configuration, groups of 128
        _case("train_kd_fp8", "train", 2047, 1024, 50304, weights="fp8", group=128, labels=False, top_k=64, tau=2.0),
        # both losses on a batch for DeepSeek-MoE-16B shapes, a quarter of it prompt
        _case("train_both", "train", 4096, 2048, 102400, top_k=32, tau=1.5, active=0.75),
        # a batch of 8192 tokens over the Gemma vocabulary: the largest
        _case("train_large", "train", 8192, 1152, 262144),
    ]


SHAPES = [(512, 32000), (1152, 262144), (1024, 50304), (2048, 102400), (576, 32128)]      # (hidden size, vocabulary) of the workloads
MOST = 8192 * 1152 * 262144


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        if rng.random() < 0.6:
            dim, vocab = rng.choice(SHAPES)
        else:
            dim, vocab = _log_int(rng, 40, 2048), _log_int(rng, 1000, 262144)
            if rng.random() < 0.5:
                dim = max(64, dim // 64 * 64)
        rows = _log_int(rng, 1, 8192)
        if rows * dim * vocab > MOST * 0.9 or dim == 3072 or vocab == 3072 or rows == 3072:
            continue
        weights = rng.choice(["bf16", "bf16", "bf16", "fp32", "fp8", "int4"])
        hidden = "fp32" if rng.random() < (0.5 if weights == "fp32" else 0.1) else "bf16"
        quantized = weights in ("fp8", "int4")
        group = 0 if not quantized else dim if dim % 8 == 0 and rng.random() < 0.3 else rng.choice([32, 64, 128, 128, 256])
        which = rng.random()
        return _case(None, rng.choice(["score", "train", "train"]), rows, dim, vocab, hidden=hidden, weights=weights, group=group,
                     scales=rng.choice(["fp32", "bf16"]) if quantized else "fp32", labels=which < 0.65,
                     top_k=0 if which < 0.3 else _log_int(rng, 1, 128), tau=rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]),
                     active=rng.choice([1.0, 1.0, 0.8, 0.5]))


def _taking_part(case):
    return max(1, int(round(case["rows"] * case["active"])))


def _quantize(w, fmt, group, scale_dtype):
    """Codes and scales of `w` in the library's formats (abs-max scaling, nearest): made here, as inputs."""
    flat = w.flatten()
    pad = -flat.numel() % group
    g = torch.nn.functional.pad(flat, (0, pad)).view(-1, group)
    rho = 448.0 if fmt == "fp8" else 7.0
    scales = (g.abs().amax(1).clamp_min(1e-12) / rho).to(scale_dtype)
    y = (g / scales.float()[:, None]).clamp(-rho, rho).flatten()[:flat.numel()]
    if fmt == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scales
    c = torch.nn.functional.pad(y.round().to(torch.int32), (0, flat.numel() % 2)) & 15
    return (c[0::2] | c[1::2] << 4).to(torch.uint8), scales


def prepare(case, seed):
    rows, dim, vocab, k = case["rows"], case["dim"], case["vocab"], case["top_k"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")       # noqa: E731
    w = torch.empty(vocab, dim, device="cuda").normal_(0.0, WEIGHT_STD, generator=gen)
    # the next token: common ones by far the most often, as in text
    target = (vocab * rand(rows) ** 3).long().clamp_(max=vocab - 1)
    # a model under training gives it a logit some way above the others'
    hidden = torch.empty(rows, dim, device="cuda").normal_(0.0, 1.0, generator=gen)
    hidden += w[target] * ((2.0 + 8.0 * rand(rows, 1)) / (dim * WEIGHT_STD ** 2))
    order = torch.randperm(rows, generator=gen, device="cuda")
    part = torch.zeros(rows, dtype=torch.bool, device="cuda")
    part[order[:_taking_part(case)]] = True
    state = {"case": case, "hidden": hidden.to(DTYPE[case["hidden"]]), "scales": None, "labels": None, "top_ids": None, "top_logits": None,
             "grad_ce": None, "grad_kd": None}
    if case["weights"] in DTYPE:
        state["weights"] = w.to(DTYPE[case["weights"]])
    else:
        state["weights"], state["scales"] = _quantize(w, case["weights"], case["group"], DTYPE[case["scales"]])
    if case["labels"]:
        state["labels"] = torch.where(part, target, IGNORED)
        state["grad_ce"] = torch.full((rows,), 1.0 / _taking_part(case), device="cuda")      # the mean over the tokens that count
    if k:
        # distinct ids, common ones the most often; the target among them in most rows; logits that fall from about 12
        ids = ((vocab - k) * rand(rows, k) ** 3).long().sort(1).values + torch.arange(k, device="cuda")
        ids = ids.gather(1, rand(rows, k).argsort(1))
        ids[:, 0] = torch.where((ids[:, 1:] == target[:, None]).any(1), ids[:, 0], target)
        logits = 12.0 - 3.0 * torch.cumsum(rand(rows, k) / torch.arange(1, k + 1, device="cuda"), 1)
        last = 1 + (k * rand(rows, 1)).long()                    # some rows come with fewer entries than there is room for
        short = (torch.arange(k, device="cuda") >= last) & (rand(rows, 1) < 0.1)
        ids = torch.where(part[:, None] & ~short, ids, -1)
        if k > 2:                                                # and a masked token's logit is -inf
            logits[:, k // 2] = torch.where(rand(rows) < 0.1, float("-inf"), logits[:, k // 2])
        state["top_ids"], state["top_logits"] = ids.int(), logits.to(DTYPE[case["hidden"]])
        state["grad_kd"] = torch.full((rows,), 0.5 / _taking_part(case), device="cuda")
    if own:
        # what a training program keeps between steps: the descriptor with its output arrays and its workspace
        from paper_2601_22101_amd import binding, harness
        fmt = {"bf16": binding.ECO_FMT_BF16_PLAIN, "fp32": binding.ECO_FMT_FP32_IDENTITY, "fp8": binding.ECO_FMT_FP8_E4M3,
               "int4": binding.ECO_FMT_INT4}[case["weights"]]
        state["head"] = harness.HeadLoss(rows, vocab, dim, weights=state["weights"], fmt=fmt, scales=state["scales"], group_size=case["group"],
                                         hidden_dtype=state["hidden"].dtype, labels=case["labels"], top_k=k, temperature=case["tau"],
                                         training=case["op"] == "train",
                                         grad_weights_dtype=DTYPE["fp32" if case["weights"] == "fp32" else "bf16"])
    return state


def _plain_weights(s, dtype):
    """The weights as vocab x dim values of `dtype`."""
    case = s["case"]
    if case["weights"] in DTYPE:
        return s["weights"].to(dtype)
    n = case["vocab"] * case["dim"]
    if case["weights"] == "fp8":
        y = s["weights"].view(torch.float8_e4m3fn).to(dtype)
    else:
        c = s["weights"].to(torch.int8)
        y = torch.stack([(c << 4) >> 4, c >> 4], 1).flatten()[:n].to(dtype)
    return (y * s["scales"].to(dtype).repeat_interleave(case["group"])[:n]).view(case["vocab"], case["dim"])


def _plain(s):
    case, tau = s["case"], s["case"]["tau"]
    h, w = s["hidden"].float(), _plain_weights(s, torch.float32)
    train = case["op"] == "train"
    out = {}
    part = torch.zeros(case["rows"], dtype=torch.bool, device=h.device)
    if s["labels"] is not None:
        part = part | (s["labels"] >= 0)
    if s["top_ids"] is not None:
        part = part | (s["top_ids"] >= 0).any(1)
    h = torch.where(part[:, None], h, 0.0)
    z = h @ w.t()
    g = torch.zeros_like(z) if train else None
    if s["labels"] is not None:
        there = s["labels"] >= 0
        y = torch.where(there, s["labels"], 0)[:, None]
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1, keepdim=True)
        out["ce"] = torch.where(there, (m + torch.log(total) - z.gather(1, y))[:, 0], 0.0)
        if train:
            a = torch.where(there, s["grad_ce"], 0.0)[:, None]
            g += e * (a / total)
            g.scatter_add_(1, y, -a)
        del e
    if s["top_ids"] is not None:
        there = s["top_ids"] >= 0
        ids = torch.where(there, s["top_ids"], 0).long()
        l = torch.where(there, s["top_logits"].float() / tau, float("-inf"))
        best = l.amax(1, keepdim=True)
        some = best > float("-inf")
        q = torch.exp(l - torch.where(some, best, 0.0))
        q = q / q.sum(1, keepdim=True).clamp_min(1e-30)
        m = z.amax(1, keepdim=True) / tau
        e = torch.exp(z / tau - m)
        total = e.sum(1, keepdim=True)
        log_p = z.gather(1, ids) / tau - m - torch.log(total)
        terms = torch.where(q > 0, q * (torch.log(q.clamp_min(1e-38)) - log_p), 0.0)
        out["kd"] = torch.where(some[:, 0], tau * tau * terms.sum(1), 0.0)
        if train:
            b = torch.where(some, s["grad_kd"][:, None] * tau, 0.0)
            g += e * (b / total)
            g.scatter_add_(1, ids, -b * q)
        del e
    if train:
        out["grad_hidden"] = (g @ w).to(s["hidden"].dtype)
        out["grad_weights"] = (g.t() @ h).to(DTYPE["fp32" if case["weights"] == "fp32" else "bf16"])
    return out


def run(state):
    if not own:
        return _plain(state)
    head = state["head"]
    ce, kd = head.forward(state["hidden"], labels=state["labels"], top_ids=state["top_ids"], top_logits=state["top_logits"])
    out = {}
    if ce is not None:
        out["ce"] = ce
    if kd is not None:
        out["kd"] = kd
    if state["case"]["op"] == "train":
        out["grad_hidden"], out["grad_weights"] = head.backward(grad_ce=state["grad_ce"], grad_kd=state["grad_kd"])
    return out


def work(case):
    n, rows, dim, vocab, k = _taking_part(case), case["rows"], case["dim"], case["vocab"], case["top_k"]
    size = {"bf16": 2, "fp32": 4}
    per_weight = {"bf16": 2.0, "fp32": 4.0, "fp8": 1.0, "int4": 0.5}[case["weights"]]
    if case["weights"] in ("fp8", "int4"):
        per_weight += size[case["scales"]] / case["group"]
    moved = n * dim * size[case["hidden"]] + vocab * dim * per_weight
    moved += rows * ((12 if case["labels"] else 0) + (4 + k * (4 + size[case["hidden"]]) if k else 0))
    flops = 2.0 * n * dim * vocab
    if case["op"] == "train":
        moved += rows * dim * size[case["hidden"]] + vocab * dim * (4 if case["weights"] == "fp32" else 2)
        flops *= 3                    # the logits, and one product for either gradient
    return {"bytes": moved, "flops": flops}


def exact(case, seed):
    """By torch's own loss functions and their derivatives in float64, some rows at a time."""
    s = prepare(case, seed)
    rows, dim, vocab, tau = case["rows"], case["dim"], case["vocab"], case["tau"]
    train = case["op"] == "train"
    w = _plain_weights(s, torch.float64).requires_grad_(train)
    out = {name: torch.zeros(rows, dtype=torch.float64, device="cuda") for name, there in (("ce", case["labels"]), ("kd", case["top_k"])) if there}
    if train:
        out["grad_hidden"] = torch.zeros(rows, dim, dtype=torch.float64, device="cuda")
        out["grad_weights"] = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 28) // vocab)
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        alive = torch.zeros(hi - lo, dtype=torch.bool, device="cuda")
        if case["labels"]:
            alive |= s["labels"][lo:hi] != IGNORED
        if case["top_k"]:
            alive |= (s["top_ids"][lo:hi] >= 0).any(1)
        h = (s["hidden"][lo:hi].double() * alive[:, None]).requires_grad_(train)
        z = h @ w.t()
        objective = torch.zeros((), dtype=torch.float64, device="cuda")
        if case["labels"]:
            ce = torch.nn.functional.cross_entropy(z, s["labels"][lo:hi], ignore_index=IGNORED, reduction="none")
            out["ce"][lo:hi] = ce.detach()
            objective = objective + (ce * s["grad_ce"][lo:hi]).sum()
        if case["top_k"]:
            ids = s["top_ids"][lo:hi].long()
            some = (ids >= 0) & (s["top_logits"][lo:hi] > float("-inf"))
            row = some.any(1)
            teacher = torch.where(some, s["top_logits"][lo:hi].double() / tau, -1e300)
            log_q = torch.log_softmax(teacher, 1)
            log_p = torch.log_softmax(z / tau, 1).gather(1, ids.clamp_min(0))
            kd = (torch.nn.functional.kl_div(log_p, log_q.clamp_min(-700), reduction="none", log_target=True) * some).sum(1) * tau * tau * row
            out["kd"][lo:hi] = kd.detach()
            objective = objective + (kd * s["grad_kd"][lo:hi]).sum()
        if train:
            objective.backward()
            out["grad_hidden"][lo:hi] = h.grad
    if train:
        out["grad_weights"] = w.grad
    return out
