"""Inputs and float64 results for the tests of the losses at the output projection, with the error bounds the results are held to.

The bounds follow from the arithmetic, element by element, before any comparison:
  * a logit is a sum of dim exact products in fp32: off by at most EPS_SUM(dim) * sum |h||w|, where EPS_SUM(n) = (8 + sqrt(n)) 2^-23
    allows for the order of the sum; two-term (quantized) weights add 2^-17 of the same sum, dropped products of three-term
    operands less than 2^-22 of it
  * ce and kd are sums of such errors and of an fp32 logarithm: both softmax statistics and the picked logits count
  * g is off by its softmax's relative error and by its own rounding, 2^-8 (eight bits of significand) as bf16 and 2^-22 as three terms; the
    gradients sum that against |w| or |h|, add their own sum's error, and round once to their type
"""
import torch

FMT = {"fp8": 0, "int4": 1, "bf16": 2, "fp32": 3}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def quantize(w, fmt, group, scale_dtype):
    flat = w.float().flatten()
    group = min(group, flat.numel())
    g = torch.nn.functional.pad(flat, (0, -flat.numel() % group)).view(-1, group)
    rho = 448.0 if fmt == "fp8" else 7.0
    scales = (g.abs().amax(1).clamp_min(1e-12) / rho).to(scale_dtype)
    y = (g / scales.float()[:, None]).clamp(-rho, rho).flatten()[:flat.numel()]
    if fmt == "fp8":
        codes = y.to(torch.float8_e4m3fn)
        values, codes = codes.double(), codes.view(torch.uint8)
    else:
        c = y.round().to(torch.int32)
        values = c.double()
        c = torch.nn.functional.pad(c, (0, flat.numel() % 2)) & 15
        codes = (c[0::2] | c[1::2] << 4).to(torch.uint8)
    return codes, scales, (values * scales.double().repeat_interleave(group)[:flat.numel()]).view(w.shape)


def inputs(rows, dim, vocab, *, hidden="bf16", weights="bf16", group=128, scales="fp32", labels=True, top_k=0, tau=1.0, top="fp32", seed=0,
           std=0.05, ignored=0.0, device="cuda"):
    """A dict of the call's arrays, and `w`, the weights as float64 values."""
    gen = torch.Generator().manual_seed(1000 + seed)
    w = torch.randn(vocab, dim, generator=gen) * std
    s = dict(rows=rows, dim=dim, vocab=vocab, fmt=FMT[weights], group=0, scales=None, tau=tau, top_k=top_k, labels=None, top_ids=None, top_logits=None,
             grad_ce=None, grad_kd=None)
    if weights in DTYPE:
        s["weights"] = w.to(DTYPE[weights])
        s["w"] = s["weights"].double()
    else:
        s["weights"], s["scales"], s["w"] = quantize(w, weights, group, DTYPE[scales])
        s["group"] = group
    s["hidden"] = torch.randn(rows, dim, generator=gen).to(DTYPE[hidden])
    drop = torch.rand(rows, generator=gen) < ignored
    if labels:
        y = torch.randint(0, vocab, (rows,), generator=gen)
        s["hidden"] += (s["w"][y] * (4.0 / max(1e-6, dim * std * std))).to(s["hidden"].dtype)
        s["labels"] = torch.where(drop, -100, y)
        s["grad_ce"] = torch.randn(rows, generator=gen) / rows
    if top_k:
        ids = torch.stack([torch.randperm(vocab, generator=gen)[:top_k] for _ in range(rows)]) if vocab <= 20000 else torch.randint(0, vocab, (rows, top_k), generator=gen)
        s["top_ids"] = torch.where(drop[:, None], -1, ids).int()
        s["top_logits"] = (torch.randn(rows, top_k, generator=gen) * 3).to(DTYPE[top])
        s["grad_kd"] = torch.randn(rows, generator=gen) / rows
    return {k: v.to(device) if isinstance(v, torch.Tensor) else v for k, v in s.items()}


def exact(s, quantized=False, g_bits=8):
    """The results in float64 and, under the same names with "_tol", how far an output may be off before its own last rounding."""
    tau = s["tau"]
    h, w = s["hidden"].double(), s["w"]
    rows, dim = h.shape
    vocab = w.shape[0]
    label_there = torch.zeros(rows, dtype=torch.bool, device=h.device) if s["labels"] is None else (s["labels"] >= 0) & (s["labels"] < vocab)
    taught = torch.zeros_like(label_there)
    q = ids = None
    if s["top_ids"] is not None:
        there = (s["top_ids"] >= 0) & (s["top_ids"] < vocab)
        ids = torch.where(there, s["top_ids"], 0).long()
        l = torch.where(there, s["top_logits"].double() / tau, float("-inf"))
        taught = (l > float("-inf")).any(1)
        q = torch.where(taught[:, None], torch.softmax(torch.where(taught[:, None], l, 0.0), 1), 0.0)
    part = label_there | taught
    h = torch.where(part[:, None], h, 0.0)
    z = h @ w.t()
    eps = lambda n: (8 + n ** 0.5) * 2.0 ** -23                               # noqa: E731
    dz = (h.abs() @ w.abs().t()) * (eps(dim) + 2.0 ** -22 + (2.0 ** -17 if quantized else 0.0))
    dz_max = dz.amax(1)
    out = {}
    g, dg = torch.zeros_like(z), torch.zeros_like(z)
    if s["labels"] is not None:
        y = torch.where(label_there, s["labels"], 0)
        lse = torch.logsumexp(z, 1)
        zy = z.gather(1, y[:, None])[:, 0]
        out["lse"], out["lse_tol"] = torch.where(part, lse, 0.0), dz_max + 2.0 ** -20 * (1 + lse.abs())
        out["ce"], out["ce_tol"] = torch.where(label_there, lse - zy, 0.0), 2 * dz_max + 2.0 ** -20 * (1 + lse.abs() + zy.abs())
        if s["grad_ce"] is not None:
            a = torch.where(label_there, s["grad_ce"].double(), 0.0)[:, None]
            p = torch.exp(z - lse[:, None])
            g += a * p
            g.scatter_add_(1, y[:, None], -a)
            dg += a.abs() * p * (2 * dz_max[:, None] + 2.0 ** -19 * (1 + lse.abs()[:, None]))
    if q is not None:
        lt = torch.logsumexp(z / tau, 1)
        zj = z.gather(1, ids)
        terms = torch.where(q > 0, q * (torch.log(q.clamp_min(1e-300)) - (zj / tau - lt[:, None])), 0.0)
        size = torch.where(q > 0, q * (torch.log(q.clamp_min(1e-300)).abs() + (zj / tau).abs() + lt.abs()[:, None]), 0.0).sum(1)
        out["kd"] = torch.where(taught, tau * tau * terms.sum(1), 0.0)
        out["kd_tol"] = tau * tau * (2 * dz_max / tau + 2.0 ** -19 * (1 + lt.abs() + size))
        if s["grad_kd"] is not None:
            b = torch.where(taught, s["grad_kd"].double() * tau, 0.0)[:, None]
            p = torch.exp(z / tau - lt[:, None])
            g += b * p
            g.scatter_add_(1, ids, -b * q)
            dg += b.abs() * (p * (2 * dz_max[:, None] / tau + 2.0 ** -19 * (1 + lt.abs()[:, None])))
            dg.scatter_add_(1, ids, b.abs() * q * 2.0 ** -19 * (1 + q.clamp_min(1e-30).log().abs()))
    dg = dg + g.abs() * 2.0 ** -g_bits
    out["grad_hidden"], out["grad_weights"] = g @ w, g.t() @ h
    more = (2.0 ** -17 if quantized else 0.0) + 2.0 ** -22
    out["grad_hidden_tol"] = dg @ w.abs() + (g.abs() @ w.abs()) * (eps(vocab) + more)
    out["grad_weights_tol"] = dg.t() @ h.abs() + (g.abs().t() @ h.abs()) * (eps(rows) + more)
    out["picked"] = torch.zeros(rows, 1 + s["top_k"], dtype=torch.float64, device=h.device)
    if s["labels"] is not None:
        out["picked"][:, 0] = torch.where(label_there, zy, 0.0)
    if q is not None:
        out["picked"][:, 1:] = torch.where(there & part[:, None], zj, 0.0)
    out["picked_tol"] = dz_max[:, None] + 2.0 ** -30
    return out


def hold(got, want, name):
    """got is within its bound of want, its last rounding included."""
    x, y, tol = got.double(), want[name], want[name + "_tol"]
    last = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -23}[got.dtype]
    tol = tol + (y.abs() + tol) * last + 1e-37
    assert torch.isfinite(x).all(), f"{name}: not finite"
    worst = ((x - y).abs() / tol).max().item() if x.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound"
    return worst
