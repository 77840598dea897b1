"""The size of the whole error of the feed-forward half's products against float64, which a lost term among thousands shows in (the bounds of ffn_checks, over the cases of test_gpu_ffn
and larger inner axes), and their gradients against differences."""
import pytest
import torch

from ffn_checks import LEFT_OUT, ROUND, hold_moved, hold_rows8, hold_whole, root
from ffn_util import FMT, act, gated_exact, gradients_exact, hold, product_bound, rows8, rows8_values, weights
from test_gpu_ffn import GATED, LINEARS, harness, make_gated, make_linear      # noqa: F401

pytestmark = pytest.mark.gpu

LINEAR = [c for c in LINEARS if c[0] * max(c[1], c[2]) >= 4096] + [(96, 8192, 520, 128, "fp8", "fp32"), (600, 8192, 520, 8192, "int4", "bf16")]
UNITS = [c for c in GATED if c[0] * max(c[1], c[2]) >= 4096] + [(96, 4096, 390, 128, "fp8", "fp32", "silu"), (600, 4096, 390, 4096, "int4", "bf16", "gelu")]


def check_linear(harness, rows, in_dim, out_dim, group, fmt, scales, out=torch.bfloat16):
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, group, fmt, scales)
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, fmt=FMT[fmt], group_size=group, out_dtype=out, training=True)
    y, exact = x @ values.t(), out == torch.float32
    got = unit.forward(codes, code_scales)
    hold(got, y, product_bound(x, values, exact=exact), "out")
    if not exact:
        hold_whole(got, [root(x, values.t()) * LEFT_OUT], y, "out")
    g = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    grad_input, grad_weights = unit.backward(g)
    g = g.double()
    want = gradients_exact([g], [values], x, [torch.zeros_like(g)])
    hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
    hold(grad_weights, want["grad_0"], want["grad_0_tol"], "grad_weights")
    hold_whole(grad_input, [root(g, values) * ROUND], want["grad_input"], "grad_input")
    hold_whole(grad_weights, [], want["grad_0"], "grad_weights")


def check_gated(harness, rows, in_dim, width, group, fmt, scales, act_name):
    gen, codes, code_scales, x, gate, up = make_gated(rows, in_dim, width, group, fmt, scales)
    unit = harness.GatedUnit(rows, in_dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], fmt=FMT[fmt], group_size=group, act=act_name, training=True)
    g = torch.randn(rows, width, generator=gen).bfloat16().cuda()
    want = gated_exact(x, gate[2], up[2], act_name, g)
    h, h_scales = unit.forward(codes, code_scales)
    hold_rows8(h, h_scales, want["h"], want["h_tol"], "h")
    hold_moved(h, h_scales, want["h"], "h")
    got = unit.backward(g)
    a, b = x @ gate[2].t(), x @ up[2].t()
    f, df = act(a, act_name)
    ga, gb = g.double() * b * df, g.double() * f
    # the output's gradients of both matrices are rounded, and so are W, whose products add up to grad_input; a and b are off by what the instruction leaves out, which
    # f, f', and through it b f', pass on with factors of at most 1.2 of the activations' slopes
    da, db = root(x, gate[2].t()) * LEFT_OUT, root(x, up[2].t()) * LEFT_OUT
    d_ga = (ga.square() * ROUND ** 2 + (g.double() * df * db).square() + (1.2 * g.double() * b * da).square()).sqrt()
    d_gb = (gb.square() * ROUND ** 2 + (1.2 * g.double() * da).square()).sqrt()
    hold(got[0], want["grad_input"], want["grad_input_tol"], "grad_input")
    hold_whole(got[0], [root(ga, gate[2]) * ROUND, root(gb, up[2]) * ROUND, root(d_ga, gate[2]), root(d_gb, up[2])], want["grad_input"], "grad_input")
    for k, d in ((0, d_ga), (1, d_gb)):
        hold(got[1 + k], want[f"grad_{k}"], want[f"grad_{k}_tol"], f"grad_{k}")
        hold_whole(got[1 + k], [root(d.t(), x)], want[f"grad_{k}"], f"grad_{k}")


@pytest.mark.parametrize("rows,in_dim,out_dim,group,fmt,scales", LINEAR)
def test_linear(harness, rows, in_dim, out_dim, group, fmt, scales):      # noqa: F811
    check_linear(harness, rows, in_dim, out_dim, group, fmt, scales)


@pytest.mark.parametrize("rows,in_dim,width,group,fmt,scales,act_name", UNITS)
def test_gated(harness, rows, in_dim, width, group, fmt, scales, act_name):      # noqa: F811
    check_gated(harness, rows, in_dim, width, group, fmt, scales, act_name)


@pytest.mark.parametrize("rows,fmt", [(3, "fp8"), (70, "int4")])
@pytest.mark.parametrize("act_name", ["silu", "gelu"])
def test_gated_gradients_against_differences(harness, rows, fmt, act_name):      # noqa: F811
    """Central differences of sum(c h) of the float64 formula, in single values behind the codes of x, gate and up."""
    in_dim, width = 128, 40
    gen = torch.Generator().manual_seed(rows)
    codes, scales = (t.cuda() for t in rows8(torch.randn(rows, in_dim, generator=gen)))
    x, (gate, up) = rows8_values(codes, scales), [weights(width, in_dim, fmt, 128, "fp32", gen) for _ in range(2)]
    c = torch.randn(rows, width, generator=gen).bfloat16().cuda()
    unit = harness.GatedUnit(rows, in_dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], fmt=FMT[fmt], act=act_name, training=True)
    unit.forward(codes, scales)
    got = unit.backward(c)
    want = gated_exact(x, gate[2], up[2], act_name, c)
    f = lambda x, g, u: (c.double() * act(x @ g.t(), act_name)[0] * (x @ u.t())).sum()      # noqa: E731
    operands = [x, gate[2], up[2]]
    for k, name in enumerate(("grad_input", "grad_0", "grad_1")):
        for at in [(0, 0), (1, 77), (2, 127)]:
            d = 2.0 ** -9
            slopes = []
            for sign in (1, -1):
                moved = [t.clone() for t in operands]
                moved[k][at] += sign * d
                slopes.append(f(*moved))
            slope = (slopes[0] - slopes[1]) / (2 * d)
            # d^2 / 6 = 6.4e-7 of third derivatives: of x, rows' sums of c b w^3 and c w^2 u, below 1; of gate, a row's x^3 b c, and up's are 0: below 100 a row
            assert abs(slope - got[k][at].double()) <= want[name + "_tol"][at] + got[k][at].double().abs() * 2.0 ** -8 + 6.4e-7 * 100 * rows, (name, at)


@pytest.mark.parametrize("rows,out_dim", [(3, 40), (70, 100)])
def test_linear_gradients_against_differences(harness, rows, out_dim):      # noqa: F811
    """sum(c x W^T) is linear in either: its differences are the gradients but for float64's roundings."""
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, 128, out_dim, 128, "fp8", "fp32")
    c = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    unit = harness.Linear(rows, 128, out_dim, weights=w, scales=ws, training=True)
    unit.forward(codes, code_scales)
    got = unit.backward(c)
    want = gradients_exact([c.double()], [values], x, [torch.zeros(rows, out_dim, dtype=torch.float64, device="cuda")])
    f = lambda x, w: (c.double() * (x @ w.t())).sum()      # noqa: E731
    for k, name in enumerate(("grad_input", "grad_0")):
        for at in [(0, 0), (1, 77), (2, 127)]:
            slopes = []
            for sign in (1, -1):
                moved = [x.clone(), values.clone()]
                moved[k][at] += sign
                slopes.append(f(*moved))
            slope, size = (slopes[0] - slopes[1]) / 2, (c.double().abs() * (x.abs() @ values.abs().t() + 2)).sum()
            assert abs(slope - got[k][at].double()) <= want[name + "_tol"][at] + got[k][at].double().abs() * 2.0 ** -8 + size * 2.0 ** -40, (name, at)
