"""The feed-forward half at the edges of its values: infinities next to padding, norms of rows whose squares pass fp32's range."""
import pytest
import torch

from ffn_checks import hold_rows8
from ffn_util import DTYPE, FMT, activations, hold, norm_exact, rows8_values, weights
from test_gpu_ffn import harness      # noqa: F401

pytestmark = pytest.mark.gpu


def as_formula(got, want, name):
    """Infinities and NaN where the formula has them, with their signs."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), f"{name}: {int((got.isnan() != want.isnan()).sum())} of {got.numel()} are NaN in one alone"
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got.isinf() * got.sign(), want.isinf() * want.sign()), f"{name}: infinities"


# out_dim: of rows that are copied, and read where they lie; rows and out_dim leave the inner axes' last steps partly empty
@pytest.mark.parametrize("rows,out_dim", [(70, 100), (70, 104), (6, 72), (190, 328), (700, 840)])
@pytest.mark.parametrize("fmt", ["fp8", "int4"])
def test_infinities_next_to_padding(harness, rows, out_dim, fmt):      # noqa: F811
    """An infinite gradient in the last row and at the start of the last step: its products with the padding's zeros are no part of a sum."""
    in_dim = 144
    gen = torch.Generator().manual_seed(rows + out_dim)
    codes, scales = activations(rows, in_dim, gen)
    codes[codes & 0x7F == 0] = 0x38                           # (no zeros, whose product with an infinity is NaN in the formula too)
    x = rows8_values(codes, scales)
    w, ws, values = weights(out_dim, in_dim, fmt, 144, "fp32", gen)
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, fmt=FMT[fmt], group_size=144, training=True)
    unit.forward(codes, scales)
    grad = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    grad[rows - 1, 7], grad[rows // 2, out_dim // 64 * 64], grad[1, out_dim - 1] = float("inf"), float("-inf"), float("inf")
    grad_input, grad_weights = unit.backward(grad)
    # products of an infinity with each term apart: a sum over the inner axis in a library's blocks has its own padding
    as_formula(grad_input, (grad.double()[:, :, None] * values[None]).sum(1), "grad_input")
    as_formula(grad_weights, (grad.double().t()[:, :, None] * x[None]).sum(1), "grad_weights")


def test_infinities_next_to_padding_of_the_gated_unit(harness):      # noqa: F811
    rows, in_dim, width = 70, 128, 100
    gen = torch.Generator().manual_seed(1)
    codes, scales = activations(rows, in_dim, gen)
    codes[codes & 0x7F == 0] = 0x38
    x = rows8_values(codes, scales)
    gate, up = weights(width, in_dim, "fp8", 128, "fp32", gen), weights(width, in_dim, "fp8", 128, "fp32", gen)
    unit = harness.GatedUnit(rows, in_dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], training=True)
    unit.forward(codes, scales)
    grad = torch.ones(rows, width, dtype=torch.bfloat16, device="cuda")
    grad[rows - 1, 7] = float("inf")
    _, grad_gate, grad_up = unit.backward(grad)
    a, b = x[-1] @ gate[2][7], x[-1] @ up[2][7]
    assert a != 0 and b != 0 and torch.isfinite(grad_gate[torch.arange(width) != 7]).all() and torch.isfinite(grad_up[torch.arange(width) != 7]).all()
    s = torch.sigmoid(a)
    assert torch.equal(grad_gate[7].double(), torch.sign(x[-1] * b * s * (1 + a * (1 - s))) * float("inf"))
    assert torch.equal(grad_up[7].double(), torch.sign(x[-1] * a) * float("inf"))


@pytest.mark.parametrize("dim", [1, 7, 40, 512, 1000, 1152, 2048, 4100, 8192, 8200])
@pytest.mark.parametrize("dtype,residual,quantize", [("bf16", False, False), ("bf16", True, True), ("fp32", True, False), ("fp32", False, True)])
def test_norm_of_rows_whose_squares_pass_the_range(harness, dim, dtype, residual, quantize):      # noqa: F811
    """The type's lowest value, values near its largest, and one such among small ones: normalised as any other row, next to rows of ordinary size and one that is infinite."""
    t = DTYPE[dtype]
    gen = torch.Generator().manual_seed(dim)
    x = torch.randn(7, dim, generator=gen)
    x[0] = torch.finfo(t).min
    x[1] = torch.sign(x[1]) * (1 + torch.rand(dim, generator=gen)) * 1.5e38
    x[2] *= 1e18                                              # sums past the range, of squares that are not
    x[3, 1:], x[3, 0] = x[3, 1:] * 1e20, 3e38
    x[5, dim // 2] = float("inf")
    x = x.to(t).cuda()
    gain, grad = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda(), torch.randn(7, dim, generator=gen).to(t).cuda()
    zeros = torch.zeros_like(x)
    unit = harness.RowNorm(7, dim, gain=gain, dtype=t, eps=1e-6, residual=residual, quantize=quantize, training=True, grad_gain_dtype=torch.float32)
    out, scales, total = unit.forward(x, zeros if residual else None)
    if residual:
        assert torch.equal(total, x)
    rows = torch.tensor([0, 1, 2, 3, 4, 6], device="cuda")
    want = norm_exact(x[rows].double(), gain.double(), 1e-6)
    # 1 / 3.4e38 is held with 21 bits: 2^-22 of it, beside the sums'
    tol = want["y_tol"] + want["y"].abs() * 2.0 ** -22
    if quantize:
        hold_rows8(out[rows], scales[rows], want["y"], tol, "y")
    else:
        hold(out[rows], want["y"], tol, "y")
    assert ((unit.rstd[rows].double() / want["rstd"] - 1).abs() <= (want["rstd_tol"] / want["rstd"]) + 2.0 ** -22).all()
    assert unit.rstd[5] == 0                                  # of an infinite row: zeros, and NaN where the infinity is (of 8 bits its block)
    if not quantize:
        assert out[5, dim // 2].isnan() and out[5].isnan().sum() == 1 and not out[5][~out[5].isnan()].any()
    else:
        assert (scales[5] == 255).sum() == 1
    few = harness.RowNorm(6, dim, gain=gain, dtype=t, eps=1e-6, residual=residual, quantize=quantize, training=True, grad_gain_dtype=torch.float32)
    few.forward(x[rows], zeros[rows] if residual else None)
    grad_input, grad_gain = few.backward(grad[rows])
    want = norm_exact(x[rows].double(), gain.double(), 1e-6, grad[rows])
    hold(grad_gain, want["grad_gain"], want["grad_gain_tol"] + (grad[rows].double().abs() * x[rows].double().abs() * want["rstd"][:, None]).sum(0) * 2.0 ** -22, "grad_gain")
    hold(grad_input, want["grad_input"], want["grad_input_tol"] + want["rstd"][:, None] * 2.0 ** -20 * (1 + grad[rows].double().abs()), "grad_input")


def test_inputs_in_what_a_call_writes(harness):      # noqa: F811
    """Refused where rows would be written that are still to be read, the object left as it was; as elsewhere where they are read first."""
    gen = torch.Generator().manual_seed(6)
    codes, scales = activations(300, 256, gen)
    w, ws, _ = weights(256, 256, "fp8", 256, "fp32", gen)
    unit = harness.GatedUnit(300, 256, 256, gate=w, gate_scales=ws, up=w, up_scales=ws, group_size=256, training=True)
    first = [t.clone() for t in unit.forward(codes, scales)]
    for c, s in ((unit.out, scales), (unit.out[1:], scales[1:]), (codes, unit.scales), (codes[:100], unit.scales[200:])):
        with pytest.raises(ValueError, match="lies in"):
            unit.forward(c, s)
    unit.backward(torch.ones(300, 256, dtype=torch.bfloat16, device="cuda"))
    again = unit.forward(*[t.clone() for t in first])
    assert not torch.equal(again[0], first[0])
    line = harness.Linear(300, 256, 256, weights=w, scales=ws, group_size=256, training=True)
    out = line.forward(codes, scales).clone()
    grad = torch.randn(300, 256, generator=gen).bfloat16().cuda()
    want = line.backward(grad)[0].clone()
    for bad in (line.grad_input, line.grad_input[:300]):
        with pytest.raises(ValueError, match="lies in"):
            line.backward(bad)
    assert torch.equal(line.backward(grad)[0], want)
    with pytest.raises(ValueError, match="lies in"):
        line.forward(codes[1:], scales[1:], add=line.out[1:])
    line.out.copy_(out)
    assert torch.equal(line.forward(codes, scales, add=line.out), line.forward(codes, scales, add=out.clone()))
    x, r = (torch.randn(300, 256, generator=gen).bfloat16().cuda() for _ in range(2))
    for quantize in (True, False):
        norm = harness.RowNorm(300, 256, residual=True, quantize=quantize, training=True, device=x.device)
        want = [t.clone() for t in norm.forward(x, r) if t is not None]
        for a, b in ((norm.sum[1:], r[1:]), (x[:9], norm.sum[3:12])):
            with pytest.raises(ValueError, match="lies in"):
                norm.forward(a, b)
        norm.sum.copy_(x)
        assert all(torch.equal(p, q) for p, q in zip([t for t in norm.forward(norm.sum, r) if t is not None], want))
        if not quantize:
            norm.out.copy_(r)
            assert all(torch.equal(p, q) for p, q in zip([t for t in norm.forward(x, norm.out) if t is not None], want))
            with pytest.raises(ValueError, match="lies in"):
                norm.forward(norm.out[1:], r[1:])
        norm.forward(x, r)
        want = norm.backward(grad, r)[0].clone()
        for a, b in ((norm.grad_input[:, :], r), (grad, norm.grad_input)):
            norm.grad_input.copy_(grad if b is r else r)
            assert torch.equal(norm.backward(a, b)[0], want)
        norm.forward(x[1:], r[1:])
        with pytest.raises(ValueError, match="lies in"):
            norm.backward(norm.grad_input[1:], r[1:])
        with pytest.raises(ValueError, match="lies in"):
            norm.backward(grad[1:], norm.grad_input[1:])


def test_types_of_the_gains_gradient(harness):      # noqa: F811
    with pytest.raises(ValueError, match="grad_gain_dtype"):
        harness.RowNorm(4, 128, gain=torch.ones(128, device="cuda"), training=True, grad_gain_dtype=torch.float16)
