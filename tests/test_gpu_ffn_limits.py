"""The feed-forward half at the limits of its sizes and strides, and the calls with strides that test_gpu_ffn does not make: norm, gated unit and rows to 8 bits."""
import pytest
import torch

from ffn_checks import hold_rows8
from ffn_util import FMT, activations, gated_exact, gradients_exact, hold, norm_exact, product_bound, rows8_values, weights
from test_gpu_ffn import eco, harness, make_gated, make_linear      # noqa: F401

pytestmark = pytest.mark.gpu


def test_strides_near_the_limit(harness):      # noqa: F811
    """Rows 2^23 - 16 codes apart, and the output's gradient 2^22 (read where it lies) and 2^23 - 8 elements (copied): offsets within a tile come up to 2^31."""
    rows, in_dim, out_dim = 300, 144, 104
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, 144, "fp8", "fp32")
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, group_size=144, training=True)
    wide = torch.empty(rows, (1 << 23) - 16, dtype=torch.uint8, device="cuda")[:, :in_dim].copy_(codes)
    y = x @ values.t()
    hold(unit.forward(wide, code_scales), y, product_bound(x, values), "out")
    g = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    want = gradients_exact([g.double()], [values], x, [torch.zeros(rows, out_dim, dtype=torch.float64, device="cuda")])
    for stride in (1 << 22, (1 << 23) - 8):
        far = torch.empty(rows, stride, dtype=torch.bfloat16, device="cuda")[:, :out_dim].copy_(g)
        grad_input, grad_weights = unit.backward(far)
        hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
        hold(grad_weights, want["grad_0"], want["grad_0_tol"], "grad_weights")
        del far
    far = torch.empty(rows, (1 << 23) - 8, dtype=torch.bfloat16, device="cuda")[:, :out_dim].copy_(g)
    hold(unit.forward(codes, code_scales, add=far), y + g.double(), product_bound(x, values) + (y.abs() + g.double().abs()) * 2.0 ** -23, "out + add")


@pytest.mark.parametrize("rows", [3, 40, 70])
@pytest.mark.parametrize("in_dim,out_dim,fmt", [(128, 65536, "fp8"), (65536, 16, "int4"), (16, 65535, "fp8")])
def test_the_widest_products(harness, rows, in_dim, out_dim, fmt):      # noqa: F811
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, in_dim, fmt, "fp32")
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, fmt=FMT[fmt], group_size=in_dim, training=True)
    hold(unit.forward(codes, code_scales), x @ values.t(), product_bound(x, values), "out")
    g = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    grad_input, grad_weights = unit.backward(g)
    want = gradients_exact([g.double()], [values], x, [torch.zeros(rows, out_dim, dtype=torch.float64, device="cuda")])
    hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
    hold(grad_weights, want["grad_0"], want["grad_0_tol"], "grad_weights")


@pytest.mark.parametrize("rows", [3, 70])
def test_the_widest_gated_unit(harness, rows):      # noqa: F811
    gen, codes, code_scales, x, gate, up = make_gated(rows, 128, 65535, 128, "fp8", "fp32")
    unit = harness.GatedUnit(rows, 128, 65535, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], training=True)
    h, h_scales = unit.forward(codes, code_scales)
    g = torch.randn(rows, 65535, generator=gen).bfloat16().cuda()
    grads = unit.backward(g)
    want = gated_exact(x, gate[2], up[2], "silu", g)
    hold_rows8(h, h_scales, want["h"], want["h_tol"], "h")
    for got, name in zip(grads, ("grad_input", "grad_0", "grad_1")):
        hold(got, want[name], want[name + "_tol"], name)


def test_the_widest_norm(harness):      # noqa: F811
    gen = torch.Generator().manual_seed(1)
    x, r, g, gs = (torch.randn(3, 65536, generator=gen).bfloat16().cuda() for _ in range(4))
    gain = (1 + 0.1 * torch.randn(65536, generator=gen)).bfloat16().cuda()
    unit = harness.RowNorm(3, 65536, gain=gain, residual=True, training=True)
    y, scales, total = unit.forward(x, r)
    grad_input, grad_gain = unit.backward(g, gs)
    want = norm_exact(total.double(), gain.double(), 1e-6, g, gs)
    hold_rows8(y, scales, want["y"], want["y_tol"], "y")
    hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
    hold(grad_gain, want["grad_gain"], want["grad_gain_tol"], "grad_gain")


def apart(t, by, shift, fill):
    """The rows of t in a wider array, `by` elements between them, from element `shift` on; and that array."""
    whole = torch.full((t.shape[0], t.shape[1] + by + shift), fill, dtype=t.dtype, device="cuda")
    whole[:, shift:shift + t.shape[1]] = t
    return whole[:, shift:shift + t.shape[1]], whole


def same(p, q):
    return torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8))


def untouched(whole, t, shift, fill):
    left, right = whole[:, :shift], whole[:, shift + t.shape[1]:]
    return bool((left == fill).all()) and bool((right == fill).all())


@pytest.mark.parametrize("dim", [5, 300, 777, 1152, 4100, 8200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("quantize", [True, False])
def test_strides_of_the_norm(eco, dim, dtype, quantize):      # noqa: F811
    """Every array with its own stride and at any alignment of its elements: the bits of packed ones, and nothing written beside the rows."""
    rows = 9
    gen = torch.Generator().manual_seed(dim)
    x, r, g, gs = (torch.randn(rows, dim, generator=gen).to(dtype).cuda() for _ in range(4))
    gain = (1 + 0.1 * torch.randn(dim + 1, generator=gen)).bfloat16().cuda()
    code = eco.ECO_DT_BF16 if dtype == torch.bfloat16 else eco.ECO_DT_FP32
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def run(by, shift):
        a = [apart(t, by + k, shift, 9.0)[0] for k, t in enumerate((x, r, g, gs))]
        empty = torch.zeros(rows, dim, dtype=dtype, device="cuda")
        total, total_whole = apart(empty, 2 * by, shift, 9.0)
        grad, grad_whole = apart(empty, 3 * by, shift, 9.0)
        out, out_whole = apart(torch.zeros(rows, dim, dtype=torch.uint8, device="cuda") if quantize else empty, 5 * by, shift, 9)
        scales = torch.zeros(rows, -(-dim // 128), dtype=torch.uint8, device="cuda") if quantize else None
        rstd, gg = torch.empty(rows, device="cuda"), torch.empty(dim + 1, device="cuda")
        d = eco.make_norm(rows=rows, dim=dim, eps=1e-6, dtype=code, grad_gain_dtype=eco.ECO_DT_FP32, input=a[0], residual=a[1], grad_out=a[2], grad_sum=a[3], sum=total, out=out,
                          scales=scales, gain=gain[1:], rstd=rstd, grad_input=grad, grad_gain=gg[1:], input_stride=a[0].stride(0), residual_stride=a[1].stride(0),
                          grad_out_stride=a[2].stride(0), grad_sum_stride=a[3].stride(0), sum_stride=total.stride(0), out_stride=out.stride(0), grad_input_stride=grad.stride(0))
        assert eco.eco_norm_backward_workspace(d) <= work.numel()
        eco.eco_norm(d)
        eco.eco_norm_backward(d, work, work.numel())
        assert untouched(total_whole, total, shift, 9.0) and untouched(grad_whole, grad, shift, 9.0) and untouched(out_whole, out, shift, 9)
        return [total, out, rstd, grad, gg[1:]] + ([scales] if quantize else [])

    packed = run(0, 0)
    for by, shift in ((1, 0), (1, 1), (2, 3)):
        for k, (p, q) in enumerate(zip(packed, run(by, shift))):
            assert same(p, q), (by, shift, k)


@pytest.mark.parametrize("rows,width,fmt", [(9, 200, "fp8"), (40, 333, "int4"), (150, 391, "fp8"), (150, 256, "int4")])
def test_strides_of_the_gated_unit(eco, rows, width, fmt):      # noqa: F811
    in_dim = 144
    gen, codes, code_scales, x, gate, up = make_gated(rows, in_dim, width, 144, fmt, "fp32")
    grad = torch.randn(rows, width, generator=gen).bfloat16().cuda()
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def run(by, shift):
        c, _ = apart(codes, 16 * by, 0, 0x7F)
        g, _ = apart(grad, 3 * by, shift, float("nan"))
        out, out_whole = apart(torch.zeros(rows, width, dtype=torch.uint8, device="cuda"), 5 * by, shift, 9)
        gi, gi_whole = apart(torch.zeros(rows, in_dim, dtype=torch.bfloat16, device="cuda"), by, shift, 9.0)
        scales = torch.zeros(rows, -(-width // 128), dtype=torch.uint8, device="cuda")
        gg, gu = (torch.empty(width, in_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        d = eco.make_gated(rows=rows, in_dim=in_dim, width=width, group_size=144, fmt=FMT[fmt], codes=c, code_scales=code_scales, gate=gate[0], gate_scales=gate[1], up=up[0],
                           up_scales=up[1], out=out, out_scales=scales, grad_out=g, grad_input=gi, grad_gate=gg, grad_up=gu, codes_stride=c.stride(0), out_stride=out.stride(0),
                           grad_out_stride=g.stride(0), grad_input_stride=gi.stride(0))
        assert max(eco.eco_gated_workspace(d, False), eco.eco_gated_workspace(d, True)) <= work.numel()
        eco.eco_gated(d, work, work.numel())
        eco.eco_gated_backward(d, work, work.numel())
        assert untouched(out_whole, out, shift, 9) and untouched(gi_whole, gi, shift, 9.0)
        return out, scales, gi, gg, gu

    packed = run(0, 0)
    for by, shift in ((1, 0), (1, 1), (4, 4), (3, 5)):
        for k, (p, q) in enumerate(zip(packed, run(by, shift))):
            assert same(p, q), (by, shift, k)


@pytest.mark.parametrize("dim", [3, 130, 1152, 9000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_of_rows_to_8_bits(harness, dim, dtype):      # noqa: F811
    gen = torch.Generator().manual_seed(dim)
    x = torch.randn(7, dim, generator=gen).to(dtype).cuda()
    codes, scales = harness.quantize_rows(x)
    for by, shift in ((1, 0), (1, 1), (5, 3)):
        out, whole = apart(torch.zeros_like(codes), 2 * by, shift, 0x5A)
        got, got_scales = harness.quantize_rows(apart(x, by, shift, float("nan"))[0], codes=out, scales=torch.zeros_like(scales))
        assert got is out and same(got, codes) and same(got_scales, scales) and untouched(whole, out, shift, 0x5A)


@pytest.mark.parametrize("rows", [5, 200])
def test_rows_of_one_value_and_zeros(harness, rows):      # noqa: F811
    """Rows whose codes are all zeros, and a scale byte at either end of what rows are given: products, h and gradients of zeros and of ordinary values beside them."""
    gen = torch.Generator().manual_seed(rows)
    codes, scales = activations(rows, 256, gen)
    codes[1], scales[1] = 0, 27
    scales[2], scales[3] = 27, 127 + 40
    w, ws, values = weights(100, 256, "fp8", 128, "fp32", gen)
    x = rows8_values(codes, scales)
    unit = harness.Linear(rows, 256, 100, weights=w, scales=ws, out_dtype=torch.float32, training=True)
    out = unit.forward(codes, scales)
    hold(out, x @ values.t(), product_bound(x, values, exact=True), "out")
    assert not out[1].any()
    gated = harness.GatedUnit(rows, 256, 100, gate=w, gate_scales=ws, up=w, up_scales=ws, training=True)
    h, h_scales = gated.forward(codes, scales)
    assert not (h[1] & 0x7F).any() and h_scales[1, 0] == 27
    grads = gated.backward(torch.ones(rows, 100, dtype=torch.bfloat16, device="cuda"))
    assert not grads[0][1].float().any() and all(torch.isfinite(g).all() for g in grads)
