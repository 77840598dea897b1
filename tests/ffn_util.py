"""Inputs, float64 results and their bounds for the tests of the feed-forward half of a layer.

The bounds follow from the arithmetic, element by element, before any comparison:
  * fp32 sums of n terms are off by at most EPS_SUM(n) = (8 + sqrt(n)) 2^-23 of the sum of absolute values, which allows for their order;
  * a product in 8 bits leaves out, of eight neighbouring products, what lies below 2^-13 of the largest: at most 8 2^-13 of the sum of absolute values.  Outputs in
    fp32 come from exact products;
  * a rounding to bf16 is off by at most 2^-8, to fp32 by 2^-24 of the value;
  * 8-bit rows: a value that is off by d before it is rounded comes out between the roundings of value - d and value + d, with the block's scale or, where the block's largest lies
    within its own bound of a power of two times 448, the neighbouring one.
"""
import torch

FMT = {"fp8": 0, "int4": 1}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
LAST = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -23}
EIGHT = 8 * 2.0 ** -13


def eps(n):
    return (8 + n ** 0.5) * 2.0 ** -23


def round_e4m3(z):
    """To nearest on the grid of E4M3, in float64; z within [-448, 448] and a little beyond."""
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(z / step) * step


def exponent(largest):
    """The smallest e in [-100, 127] with largest <= 448 2^e."""
    f, p = torch.frexp(largest.double())
    return torch.where(f == 0, -100, p - 9 + (f > 0.875).int()).clamp(-100, 127)


def blocks(y):
    return torch.nn.functional.pad(y, (0, -y.shape[1] % 128)).view(y.shape[0], -1, 128)


def rows8(y):
    """Codes and scale bytes of rows, made from their float64 values."""
    b = blocks(y.double())
    e = exponent(b.abs().amax(2))
    codes = round_e4m3(b * torch.exp2(-e.double())[..., None]).to(torch.float8_e4m3fn)
    return codes.view(y.shape[0], -1)[:, :y.shape[1]].contiguous().view(torch.uint8), (e + 127).to(torch.uint8)


def rows8_values(codes, scales):
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(scales.double() - 127).repeat_interleave(128, 1)[:, :codes.shape[1]]


def hold_rows8(codes, scales, y, d, name):
    """8-bit rows of the values y, each of which is off by at most d."""
    largest, off = blocks(y.abs()).amax(2), blocks(d).amax(2)
    e = scales.double() - 127
    lo, hi = exponent((largest - off).clamp_min(0)), exponent(largest + off)
    assert ((e >= lo) & (e <= hi)).all(), f"{name}: a scale"
    s = torch.exp2(-e).repeat_interleave(128, 1)[:, :y.shape[1]]
    got = codes.view(torch.float8_e4m3fn).double()
    most = torch.full_like(got, 448.0)
    below, above = round_e4m3(((y - d) * s).clamp(-449, 449)), round_e4m3(((y + d) * s).clamp(-449, 449))
    bad = (got < torch.maximum(below, -most)) | (got > torch.minimum(above, most))
    assert not bad.any(), f"{name}: {int(bad.sum())} codes of {bad.numel()}"


def hold(got, want, tol, name):
    x, y = got.double(), want
    tol = tol + (y.abs() + tol) * LAST[got.dtype] + 1e-37
    assert torch.isfinite(x).all(), f"{name}: not finite"
    worst = ((x - y).abs() / tol).max().item() if x.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound"
    return worst


def quantize_weights(w, fmt, group, scale_dtype):
    """Codes, scales and the float64 values that they stand for."""
    flat = w.float().flatten()
    n = flat.numel()
    group = min(group, n)
    g = torch.nn.functional.pad(flat, (0, -n % group)).view(-1, group)
    rho = 448.0 if fmt == "fp8" else 7.0
    scales = (g.abs().amax(1).clamp_min(1e-12) / rho).to(scale_dtype)
    y = (g / scales.float()[:, None]).clamp(-rho, rho).flatten()[:n]
    if fmt == "fp8":
        codes = y.to(torch.float8_e4m3fn)
        values, codes = codes.double(), codes.view(torch.uint8)
    else:
        c = y.round().to(torch.int32)
        values = c.double()
        c = torch.nn.functional.pad(c, (0, n % 2)) & 15
        codes = (c[0::2] | c[1::2] << 4).to(torch.uint8)
    return codes, scales, (values * scales.double().repeat_interleave(group)[:n]).view(w.shape)


def activations(rows, dim, gen, device="cuda"):
    """8-bit rows as a layer has them: a few channels are far larger than the others, rows of different sizes."""
    channels = 1.0 + 20.0 * (torch.rand(dim, generator=gen) < 0.02)
    x = torch.randn(rows, dim, generator=gen) * channels * torch.exp2(4 * torch.randn(rows, 1, generator=gen))
    return tuple(t.to(device) for t in rows8(x))


def weights(width, dim, fmt, group, scales, gen, device="cuda"):
    return tuple(t.to(device) for t in quantize_weights(torch.randn(width, dim, generator=gen) * 0.05, fmt, group, DTYPE[scales]))


def act(a, kind):
    """The activation and its derivative in float64."""
    if kind == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1 + a * (1 - p))
    k = (2 / torch.pi) ** 0.5
    t = torch.tanh(k * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)


def norm_exact(s, gain, eps_norm, grad_out=None, grad_sum=None):
    """Of rows s (float64): y, rstd, grad_input, grad_gain and, under the same names with _tol, their bounds before the last rounding."""
    n = s.shape[1]
    rstd = (s.square().mean(1, keepdim=True) + eps_norm).rsqrt()
    e = eps(n) + 8 * 2.0 ** -24                              # of the mean of squares, and of rstd, which is a root of it
    y = s * rstd * gain
    out = {"y": y, "y_tol": y.abs() * e, "rstd": rstd[:, 0], "rstd_tol": rstd[:, 0] * e}
    if grad_out is not None:
        g, h = grad_out.double(), s * rstd
        u = g * gain
        mean = (u * h).mean(1, keepdim=True)
        d_mean = (u * h).abs().mean(1, keepdim=True) * 2 * e
        more = 0.0 if grad_sum is None else grad_sum.double()
        out["grad_input"] = rstd * (u - h * mean) + more
        size = rstd * (u.abs() + (h * mean).abs())
        out["grad_input_tol"] = rstd * h.abs() * d_mean + size * (2 * e + 2.0 ** -21) + (0.0 if grad_sum is None else more.abs() * 2.0 ** -23)
        out["grad_gain"] = (g * h).sum(0)
        out["grad_gain_tol"] = (g * h).abs().sum(0) * (eps(s.shape[0]) + e)
    return out


def product_bound(x, w, exact=False):
    """The bound of x w^T before it is rounded."""
    return (x.abs() @ w.abs().t()) * (eps(x.shape[1]) + (0.0 if exact else EIGHT) + 2.0 ** -22)


def gradients_exact(grads, ws, x, d_grads):
    """grad_input and each grad_weights of outputs' gradients that are off by d_grads; W is rounded to bf16 on its way."""
    out = {"grad_input": sum(g @ w for g, w in zip(grads, ws)),
           "grad_input_tol": sum((g.abs() @ w.abs()) * (2.0 ** -8 + eps(2 * w.shape[0])) + d @ (w.abs() * (1 + 2.0 ** -8)) for g, w, d in zip(grads, ws, d_grads))}
    for k, (g, d) in enumerate(zip(grads, d_grads)):
        out[f"grad_{k}"] = g.t() @ x
        out[f"grad_{k}_tol"] = (g.abs().t() @ x.abs()) * eps(x.shape[0]) + d.t() @ x.abs()
    return out


def gated_exact(x, gate, up, kind, grad_out=None):
    """h with its bound and, with grad_out, the gradients with theirs."""
    a, b = x @ gate.t(), x @ up.t()
    da, db = product_bound(x, gate), product_bound(x, up)
    f, df = act(a, kind)
    # the activations' derivatives are at most 1.13, their second ones at most 1.2; f and df are off by what fp32 makes of a logistic, 2^-24 (8 + |a|) of |a|
    slack = 2.0 ** -23 * (8 + a.abs().clamp_max(200))
    d_f = 1.13 * da + a.abs() * slack + 2.0 ** -100
    d_df = 1.2 * da + (1 + a.abs()) * slack
    h = f * b
    out = {"h": h, "h_tol": d_f * (b.abs() + db) + f.abs() * db + h.abs() * 2.0 ** -22}
    if grad_out is not None:
        g = grad_out.double()
        ga, gb = g * b * df, g * f
        d_ga = g.abs() * (db * (df.abs() + d_df) + b.abs() * d_df) + ga.abs() * (2.0 ** -8 + 2.0 ** -21)
        d_gb = g.abs() * d_f + gb.abs() * (2.0 ** -8 + 2.0 ** -21)
        out.update(gradients_exact([ga, gb], [gate, up], x, [d_ga, d_gb]))
    return out
