"""The feed-forward half of a layer on the weights that the step keeps, as cases that can be timed and compared: the root-mean-square norm
with the residual's addition and an 8-bit output, the linear product in 8-bit floating point and the gated unit (two such products and their
activation), each with its gradients, over the shapes that the feed-forward matrices of `workloads/` have (and odd ones), from one token to thousands.

8-bit rows: blocks of 128 along a row, the last one possibly shorter, are E4M3 codes times a power of two 2^e, held as the byte e + 127 (E8M0); e is the
smallest whole number of [-100, 127] with max |block| <= 448 2^e.  Codes are rounded to nearest, ties to even.  Weights are E4M3 or INT4 codes with a scale
for each `group` elements of a row (0: one for the whole row), as the step writes them.

    norm     s = x + residual (rounded to its type, as the residual stream is);  r = 1 / sqrt(mean s^2 + eps);  y = s r gain, as 8-bit rows or in the input's type
             grad_x = r (gy - s r mean(gy s r)) + grad_s,  gy = grad_y gain;   grad_gain = sum over rows of grad_y s r
    linear   y = x W^T (+ add), x in 8-bit rows;   grad_x = grad_y W,  grad_W = grad_y^T x
    gated    h = act(x G^T) * (x U^T) as 8-bit rows;   with a = x G^T, b = x U^T:  ga = grad_h b act'(a),  gb = grad_h act(a),
             grad_x = ga G + gb U,  grad_G = ga^T x,  grad_U = gb^T x
The gradients pass the roundings to 8 bits straight through.

A case is a dict of plain values: `op`, whether it is a training pass (`train`: the gradients too), `rows` x `dim` and, of the products, the other dimension `width`.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 128
EPS = 1e-6
WEIGHT_STD = 0.02                     # as the workloads' weights


def _norm(name, rows, dim, *, train=False, dtype="bf16", residual=True, quantize=True, gain="bf16"):
    c = {"op": "norm", "rows": rows, "dim": dim, "train": train, "dtype": dtype, "residual": residual, "quantize": quantize, "gain": gain}
    return dict(c, name=name) if name else c


def _linear(name, rows, dim, width, *, train=False, weights="fp8", group=BLOCK, scales="fp32", out="bf16", add=False):
    c = {"op": "linear", "rows": rows, "dim": dim, "width": width, "train": train, "weights": weights, "group": group, "scales": scales, "out": out, "add": add}
    return dict(c, name=name) if name else c


def _gated(name, rows, dim, width, *, train=False, weights="fp8", group=BLOCK, scales="fp32", act="silu"):
    c = {"op": "gated", "rows": rows, "dim": dim, "width": width, "train": train, "weights": weights, "group": group, "scales": scales, "act": act}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of generation through a 30 M transformer's norm: latency alone
        _norm("norm_one_token", 1, 512),
        # a prompt of 4096 tokens through a Gemma-3-1B-shaped layer
        _norm("norm_prompt", 4096, 1152),
        # training with activations in fp32, odd sizes everywhere: the last block is short, rows begin anywhere
        _norm("norm_train_odd", 333, 777, train=True, dtype="fp32", gain="fp32"),
        # a training batch of DeepSeek-MoE-16B shapes: the largest
        _norm("norm_train", 16384, 2048, train=True),
        # one token through the down projection of a Gemma-3-1B-shaped layer, back to the residual stream
        _linear("linear_one_token", 1, 6912, 1152, add=True),
        # a few sequences' tokens through an INT4 expert of DeepSeek-MoE-16B shapes
        _linear("linear_few_int4", 24, 2048, 1408, weights="int4", scales="bf16"),
        # a prompt of 8192 tokens through the down projection of Gemma-3-1B shapes
        _linear("linear_prompt", 8192, 6912, 1152, add=True),
        # a batch of the paper's own sparse-MoE model, with its one scale a row; one token short of whole tiles
        _linear("linear_train", 4095, 576, 2304, train=True, group=0),
        # one token through the gate and up projections of a Gemma-3-1B-shaped layer
        _gated("gated_one_token", 1, 1152, 6912, act="gelu"),
        # evaluation of 2048 tokens through an expert of the benchmark's sparse-MoE configuration
        _gated("gated_sequence", 2048, 1024, 1024),
        # fine-tuning an INT4 expert of DeepSeek-MoE-16B shapes on the tokens that were sent to it
        _gated("gated_train_int4", 1000, 2048, 1408, train=True, weights="int4", scales="bf16"),
        # a training batch of 8192 tokens of Gemma-3-1B shapes: the largest
        _gated("gated_train", 8192, 1152, 6912, train=True, act="gelu"),
    ]


SHAPES = [(512, 2048), (1152, 6912), (1024, 1024), (2048, 1408), (576, 2304)]      # (hidden size, width) of the workloads' feed-forward matrices
MOST = 12 * 8192 * 1152 * 6912


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "linear", "gated"])
        train = rng.random() < 0.5
        rows = _log_int(rng, 1, 16384)
        if op == "norm":
            dim = rng.choice(SHAPES)[0] if rng.random() < 0.4 else _log_int(rng, 64, 8192)
            if rows * dim > 0.9 * 16384 * 2048:
                continue
            dtype = rng.choice(["bf16", "bf16", "fp32"])
            return _norm(None, rows, dim, train=train, dtype=dtype, residual=rng.random() < 0.7, quantize=rng.random() < 0.7, gain=rng.choice(["bf16", dtype]))
        weights = rng.choice(["fp8", "fp8", "int4"])
        by_row = rng.random() < 0.35
        if rng.random() < 0.5:
            dim, width = rng.choice(SHAPES)
            if op == "linear" and rng.random() < 0.5:
                dim, width = width, dim
        else:
            dim, width = _log_int(rng, 128, 8192), _log_int(rng, 100, 8192)          # any width; rows of weights are whole pieces or blocks
        dim = max(16, dim // 16 * 16) if by_row else max(BLOCK, dim // BLOCK * BLOCK)
        group = 0 if by_row else BLOCK if dim % (2 * BLOCK) or rng.random() < 0.7 else 2 * BLOCK
        times = (4 if op == "gated" else 2) * (3 if train else 1)
        if times * rows * dim * width > 0.9 * MOST:
            continue
        more = {"train": train, "weights": weights, "group": group, "scales": rng.choice(["fp32", "bf16"])}
        if op == "linear":
            return _linear(None, rows, dim, width, out=rng.choice(["bf16", "bf16", "fp32"]), add=rng.random() < 0.4, **more)
        return _gated(None, rows, dim, width, act=rng.choice(["silu", "gelu"]), **more)


# ---- inputs

def _group(case):
    return case["group"] or case["dim"]


def _quantize_weights(w, fmt, group, scale_dtype):
    """Codes and scales of `w` in the library's formats (abs-max scaling, nearest): made here, as inputs."""
    rho = 448.0 if fmt == "fp8" else 7.0
    g = w.view(-1, group)
    scales = (g.abs().amax(1).clamp_min(1e-12) / rho).to(scale_dtype)
    y = (g / scales.float()[:, None]).clamp(-rho, rho).flatten()
    if fmt == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scales
    c = y.round().to(torch.int32) & 15
    return (c[0::2] | c[1::2] << 4).to(torch.uint8), scales


def _rows8(y):
    """Codes and scale bytes of the rows of `y` (fp32): the 8-bit rows described above."""
    rows, dim = y.shape
    b = torch.nn.functional.pad(y, (0, -dim % BLOCK)).view(rows, -1, BLOCK)
    f, p = torch.frexp(b.abs().amax(2))                       # max = f 2^p, f in [0.5, 1): against 448 = 0.875 2^9
    e = torch.where(f == 0, -100, p - 9 + (f > 0.875).int()).clamp(-100, 127)
    codes = torch.ldexp(b, -e[..., None].float()).to(torch.float8_e4m3fn).view(rows, -1)[:, :dim]
    return codes.contiguous(), (e + 127).to(torch.uint8)


def _rows8_values(codes, scales, dtype):
    e = scales.to(torch.int32) - 127
    return codes.to(dtype) * torch.ldexp(torch.ones((), dtype=dtype, device=codes.device), e).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def prepare(case, seed):
    rows, dim = case["rows"], case["dim"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.empty(*shape, device="cuda").normal_(0.0, 1.0, generator=gen)       # noqa: E731
    # activations have a few channels that are far larger than the others, and tokens of different sizes
    channels = 1.0 + 20.0 * (torch.rand(dim, generator=gen, device="cuda") < 0.005)
    x = normal(rows, dim) * channels * (0.5 + torch.rand(rows, 1, generator=gen, device="cuda"))
    token = torch.exp(normal(rows, 1)) / rows                   # tokens' shares of a loss that is a mean
    state = {"case": case}
    if case["op"] == "norm":
        dtype = DTYPE[case["dtype"]]
        state["x"] = x.to(dtype)
        state["residual"] = (3.0 * normal(rows, dim)).to(dtype) if case["residual"] else None
        state["gain"] = (1.0 + 0.1 * normal(dim)).to(DTYPE[case["gain"]])
        if case["train"]:
            state["grad_y"] = (normal(rows, dim) * token).to(dtype)
            state["grad_s"] = (normal(rows, dim) * token).to(dtype) if case["residual"] else None
        if own:
            from paper_2601_22101_amd import harness
            state["unit"] = harness.RowNorm(rows, dim, gain=state["gain"], dtype=dtype, eps=EPS, residual=case["residual"], quantize=case["quantize"],
                                            training=case["train"])
        return state
    width, group = case["width"], _group(case)
    codes, scales = _rows8(x)
    state["codes"], state["scales"] = codes.view(torch.uint8), scales
    names = ["weights"] if case["op"] == "linear" else ["gate", "up"]
    for name in names:
        state[name] = _quantize_weights(normal(width, dim) * WEIGHT_STD, case["weights"], group, DTYPE[case["scales"]])
    if case["op"] == "linear":
        state["add"] = normal(rows, width).to(DTYPE[case["out"]]) if case["add"] else None
    if case["train"]:
        state["grad"] = (normal(rows, width) * token).to(torch.bfloat16)
    if own:
        # what a program keeps between calls: the descriptor with its output arrays and its workspace
        from paper_2601_22101_amd import binding, harness
        fmt = {"fp8": binding.ECO_FMT_FP8_E4M3, "int4": binding.ECO_FMT_INT4}[case["weights"]]
        if case["op"] == "linear":
            state["unit"] = harness.Linear(rows, dim, width, weights=state["weights"][0], scales=state["weights"][1], fmt=fmt, group_size=group,
                                           out_dtype=DTYPE[case["out"]], training=case["train"])
        else:
            state["unit"] = harness.GatedUnit(rows, dim, width, gate=state["gate"][0], gate_scales=state["gate"][1], up=state["up"][0],
                                              up_scales=state["up"][1], fmt=fmt, group_size=group, act=case["act"], training=case["train"])
    return state


# ---- the operators in elementary operations, in 32 bits

def _weight_values(case, codes, scales, dtype):
    if case["weights"] == "fp8":
        y = codes.view(torch.float8_e4m3fn).to(dtype)
    else:
        c = codes.to(torch.int8)
        y = torch.stack([(c << 4) >> 4, c >> 4], 1).to(dtype)
    return (y.view(-1, _group(case)) * scales.to(dtype)[:, None]).view(case["width"], case["dim"])


def _rows8_out(y, out):
    codes, scales = _rows8(y)
    out["codes"], out["scales"] = codes, scales.view(torch.float8_e8m0fnu)


def _plain_norm(s):
    case, out = s["case"], {}
    dtype = DTYPE[case["dtype"]]
    t = s["x"]
    if case["residual"]:
        t = out["sum"] = (t.float() + s["residual"].float()).to(dtype)
    t = t.float()
    r = 1.0 / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)
    n = t * r
    y = n * s["gain"].float()
    if case["quantize"]:
        _rows8_out(y, out)
    else:
        out["y"] = y.to(dtype)
    if case["train"]:
        g = s["grad_y"].float()
        gy = g * s["gain"].float()
        gx = r * (gy - n * (gy * n).mean(1, keepdim=True))
        if s["grad_s"] is not None:
            gx = gx + s["grad_s"].float()
        out["grad_x"] = gx.to(dtype)
        out["grad_gain"] = (g * n).sum(0).to(torch.bfloat16)
    return out


def _plain_linear(s):
    case = s["case"]
    x = _rows8_values(s["codes"].view(torch.float8_e4m3fn), s["scales"], torch.float32)
    w = _weight_values(case, *s["weights"], torch.float32)
    y = x @ w.t()
    if case["add"]:
        y = y + s["add"].float()
    out = {"y": y.to(DTYPE[case["out"]])}
    if case["train"]:
        g = s["grad"].float()
        out["grad_x"] = (g @ w).to(torch.bfloat16)
        out["grad_weights"] = (g.t() @ x).to(torch.bfloat16)
    return out


C_GELU = math.sqrt(2.0 / math.pi)


def _act(a, kind):
    """The activation and its derivative."""
    if kind == "silu":
        p = 1.0 / (1.0 + torch.exp(-a))
        return a * p, p * (1.0 + a * (1.0 - p))
    t = torch.tanh(C_GELU * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * C_GELU * (1.0 + 3 * 0.044715 * a * a)


def _plain_gated(s):
    case, out = s["case"], {}
    x = _rows8_values(s["codes"].view(torch.float8_e4m3fn), s["scales"], torch.float32)
    gate, up = (_weight_values(case, *s[name], torch.float32) for name in ("gate", "up"))
    a, b = x @ gate.t(), x @ up.t()
    f, df = _act(a, case["act"])
    _rows8_out(f * b, out)
    if case["train"]:
        g = s["grad"].float()
        ga, gb = g * b * df, g * f
        out["grad_x"] = (ga @ gate + gb @ up).to(torch.bfloat16)
        out["grad_gate"] = (ga.t() @ x).to(torch.bfloat16)
        out["grad_up"] = (gb.t() @ x).to(torch.bfloat16)
    return out


def _own(s):
    case, unit, out = s["case"], s["unit"], {}
    if case["op"] == "norm":
        y, scales, total = unit.forward(s["x"], s["residual"])
        if case["residual"]:
            out["sum"] = total
        if case["quantize"]:
            out["codes"], out["scales"] = y.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)
        else:
            out["y"] = y
        if case["train"]:
            out["grad_x"], out["grad_gain"] = unit.backward(s["grad_y"], s["grad_s"])
    elif case["op"] == "linear":
        out["y"] = unit.forward(s["codes"], s["scales"], add=s["add"])
        if case["train"]:
            out["grad_x"], out["grad_weights"] = unit.backward(s["grad"])
    else:
        codes, scales = unit.forward(s["codes"], s["scales"])
        out["codes"], out["scales"] = codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)
        if case["train"]:
            out["grad_x"], out["grad_gate"], out["grad_up"] = unit.backward(s["grad"])
    return out


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "linear": _plain_linear, "gated": _plain_gated}[state["case"]["op"]](state)


def work(case):
    size = {"bf16": 2.0, "fp32": 4.0}
    rows, dim, eight = case["rows"], case["dim"], 1.0 + 1.0 / BLOCK
    if case["op"] == "norm":
        e = size[case["dtype"]]
        each = e * (3 if case["residual"] else 1) + (eight if case["quantize"] else e)
        if case["train"]:
            each += e * (3 if case["residual"] else 2)         # the gradients; what was normalised stays with the chip or comes again with the forward's own
        return {"bytes": rows * dim * each + 2 * dim * size[case["gain"]], "flops": rows * dim * (14.0 if case["train"] else 5.0)}
    width = case["width"]
    per_weight = {"fp8": 1.0, "int4": 0.5}[case["weights"]] + size[case["scales"]] / _group(case)
    matrices = 2 if case["op"] == "gated" else 1
    moved = rows * dim * eight + matrices * width * dim * per_weight
    moved += rows * width * (eight if case["op"] == "gated" else size[case["out"]] * (2 if case["add"] else 1))
    flops = 2.0 * matrices * rows * dim * width
    if case["train"]:
        moved += rows * width * 2.0 + rows * dim * 2.0 + matrices * width * dim * 2.0
        flops *= 3                    # the forward's products, and one for either gradient
    return {"bytes": moved, "flops": flops}


# ---- from the definitions, in 64 bits

def _rows8_exact(y, out):
    rows, dim = y.shape
    for name in ("codes", "scales"):
        out[name] = torch.zeros(rows, dim if name == "codes" else -(-dim // BLOCK), dtype=torch.float64, device=y.device)
    for k in range(0, dim, BLOCK):
        part = y[:, k:k + BLOCK]
        largest = part.abs().amax(1)
        e = torch.ceil(torch.log2(largest.clamp_min(1e-60) / 448.0))
        e = torch.where(largest > 448.0 * torch.exp2(e), e + 1, torch.where(largest <= 448.0 * torch.exp2(e - 1), e - 1, e)).clamp(-100, 127)
        scale = torch.exp2(e)
        z = part / scale[:, None]
        # the grid of E4M3: three bits after the leading one, down to 2^-9
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
        out["codes"][:, k:k + BLOCK] = torch.round(z / step) * step
        out["scales"][:, k // BLOCK] = scale


def exact(case, seed):
    """By the definitions and torch's own derivatives in float64."""
    s = prepare(case, seed)
    train, out = case["train"], {}
    if case["op"] == "norm":
        x = s["x"].double()
        if case["residual"]:
            x = (x + s["residual"].double()).to(DTYPE[case["dtype"]])
            out["sum"], x = x.double(), x.double()
        x.requires_grad_(train)
        gain = s["gain"].double().requires_grad_(train)
        y = x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * gain
        if case["quantize"]:
            _rows8_exact(y.detach(), out)
        else:
            out["y"] = y.detach()
        if train:
            y.backward(s["grad_y"].double())
            out["grad_x"] = x.grad if s["grad_s"] is None else x.grad + s["grad_s"].double()
            out["grad_gain"] = gain.grad
        return out
    x = s["codes"].view(torch.float8_e4m3fn).double() * torch.exp2(s["scales"].double() - 127.0).repeat_interleave(BLOCK, 1)[:, :case["dim"]]
    x.requires_grad_(train)
    w = [_weight_values(case, *s[name], torch.float64).requires_grad_(train) for name in (("weights",) if case["op"] == "linear" else ("gate", "up"))]
    if case["op"] == "linear":
        y = x @ w[0].t()
        out["y"] = (y + s["add"].double() if case["add"] else y).detach()
    else:
        a = x @ w[0].t()
        f = torch.nn.functional.silu(a) if case["act"] == "silu" else torch.nn.functional.gelu(a, approximate="tanh")
        y = f * (x @ w[1].t())
        _rows8_exact(y.detach(), out)
    if train:
        y.backward(s["grad"].double())
        out["grad_x"] = x.grad
        for name, v in zip(("grad_weights",) if case["op"] == "linear" else ("grad_gate", "grad_up"), w):
            out[name] = v.grad
    return out
