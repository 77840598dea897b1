"""The feed-forward half of a layer on the GPU against float64: the norm with the residual's addition and 8-bit rows, the 8-bit linear product, the gated unit, forward
and backward, over formats, scale groups, odd sizes and strides, and a layer's half as a whole.  The bounds are those of ffn_util."""
import pytest
import torch

from ffn_util import DTYPE, FMT, activations, gated_exact, gradients_exact, hold, hold_rows8, norm_exact, product_bound, rows8, rows8_values, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eco():
    from paper_2601_22101_amd import binding
    return binding


@pytest.fixture(scope="module")
def harness():
    from paper_2601_22101_amd import harness
    return harness


NORMS = [(1, 512), (1, 1), (2, 7), (3, 127), (5, 128), (4, 129), (33, 520), (7, 777), (65, 1152), (9, 1537), (300, 2048), (3, 2049), (5, 4100), (2, 8192), (3, 8200), (2, 20011)]


@pytest.mark.parametrize("rows,dim", NORMS)
@pytest.mark.parametrize("dtype,residual,quantize,gain", [("bf16", True, True, "bf16"), ("fp32", False, True, "fp32"), ("bf16", False, False, "fp32"), ("fp32", True, False, None)])
def test_norm(harness, rows, dim, dtype, residual, quantize, gain):
    gen = torch.Generator().manual_seed(rows * 10007 + dim)
    normal = lambda *shape: torch.randn(*shape, generator=gen)                     # noqa: E731
    t = DTYPE[dtype]
    x, r = (normal(rows, dim) * torch.exp2(3 * normal(rows, 1))).to(t).cuda(), normal(rows, dim).to(t).cuda()
    g = None if gain is None else (1 + 0.3 * normal(dim)).to(DTYPE[gain]).cuda()
    grad_out, grad_sum = (normal(rows, dim) / rows).to(t).cuda(), (normal(rows, dim) / rows).to(t).cuda()
    unit = harness.RowNorm(rows, dim, gain=g, dtype=t, eps=1e-5, residual=residual, quantize=quantize, training=True, grad_gain_dtype=torch.float32,
                           device=x.device)
    out, scales, total = unit.forward(x, r if residual else None)
    grad_input, grad_gain = unit.backward(grad_out, grad_sum if residual else None)
    s = (x.float() + r.float()).to(t) if residual else x
    if residual:
        assert torch.equal(total, s)
    want = norm_exact(s.double(), torch.ones(dim, device="cuda", dtype=torch.float64) if g is None else g.double(), 1e-5, grad_out, grad_sum if residual else None)
    hold(unit.rstd, want["rstd"], want["rstd_tol"], "rstd")
    if quantize:
        hold_rows8(out, scales, want["y"], want["y_tol"], "y")
    else:
        hold(out, want["y"], want["y_tol"], "y")
    hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
    if g is not None:
        hold(grad_gain, want["grad_gain"], want["grad_gain_tol"], "grad_gain")


def test_norm_gradient_against_differences(harness):
    """The gradient of sum(c y) in fp32 against central differences of the float64 formula."""
    gen = torch.Generator().manual_seed(3)
    x, c, gain = torch.randn(3, 40, generator=gen), torch.randn(3, 40, generator=gen), 1 + 0.2 * torch.randn(40, generator=gen)
    unit = harness.RowNorm(3, 40, gain=gain.cuda(), dtype=torch.float32, eps=1e-3, quantize=False, training=True, grad_gain_dtype=torch.float32)
    unit.forward(x.cuda())
    grad_input, grad_gain = (t.double().cpu() for t in unit.backward(c.cuda()))
    f = lambda x, g: (c.double() * norm_exact(x, g, 1e-3)["y"]).sum()            # noqa: E731
    d = 2.0 ** -12
    for at in [(0, 0), (1, 17), (2, 39)]:
        e = torch.zeros(3, 40, dtype=torch.float64)
        e[at] = d
        slope = (f(x.double() + e, gain.double()) - f(x.double() - e, gain.double())) / (2 * d)
        assert abs(slope - grad_input[at]) <= 1e-5 * grad_input.abs().max()     # d^2 / 6 = 1e-8 of third derivatives of some hundreds, fp32 beside it
        e = torch.zeros(40, dtype=torch.float64)
        e[at[1]] = d
        slope = (f(x.double(), gain.double() + e) - f(x.double(), gain.double() - e)) / (2 * d)
        assert abs(slope - grad_gain[at[1]]) <= 1e-5 * grad_gain.abs().max()


@pytest.mark.parametrize("rows,dim,stride", [(1, 1, 1), (3, 130, 130), (70, 1000, 1011), (2, 9000, 9000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_quantize(harness, rows, dim, stride, dtype):
    """Exact: the scale is a power of two, and the value times it is rounded once."""
    gen = torch.Generator().manual_seed(rows + dim)
    x = (torch.randn(rows, stride, generator=gen) * torch.exp2(8 * torch.randn(rows, stride, generator=gen))).to(DTYPE[dtype]).cuda()[:, :dim]
    codes, scales = harness.quantize_rows(x)
    want_codes, want_scales = rows8(x.double())
    assert torch.equal(scales, want_scales)
    assert torch.equal(codes.view(torch.float8_e4m3fn).float(), want_codes.view(torch.float8_e4m3fn).float())


def test_rows_quantize_borders(harness):
    """Blocks of zeros, of the smallest and largest values, a largest of 448 2^k exactly and just above, ties, and values that are not finite."""
    x = torch.zeros(9, 256, device="cuda")
    x[1, 5], x[2, 5] = 448.0, 448.0 * (1 + 2.0 ** -20)
    x[3, :4] = torch.tensor([256.0, 17.0, 19.0, 21.0], device="cuda")           # ties go to even
    x[4, 0], x[4, 200] = 3e38, 1e-38                                             # 1.763 2^127, above 448 2^119 = 1.75 2^127
    x[5, 7], x[6, 130], x[7, 255] = float("nan"), float("inf"), float("-inf")
    x[5, 8] = x[6, 131] = 1.0
    x[8, 0] = 2.0 ** -91                                                         # 448 2^-100 = 1.75 2^-92 is the smallest block's largest
    codes, scales = harness.quantize_rows(x)
    assert scales[0].tolist() == [27, 27] and int(codes[0].sum()) == 0
    assert scales[1].tolist() == [127, 27] and scales[2].tolist() == [128, 27]
    v = rows8_values(codes, scales)
    assert v[1, 5] == 448 and v[2, 5] == 448
    assert v[3, :4].tolist() == [256, 16, 20, 20]
    assert scales[4].tolist() == [127 + 120, 27] and abs(v[4, 0].item() / 3e38 - 1) <= 2.0 ** -4 and v[4, 200] == 0
    for row, block in ((5, 0), (6, 1), (7, 1)):
        assert scales[row, block] == 255 and (codes[row, 128 * block:128 * block + 128] == 0x7F).all()
        assert scales[row, 1 - block] == 27 and int(codes[row, 128 - 128 * block:256 - 128 * block].sum()) == 0
    assert scales[8, 0] == 28 and v[8, 0] == 2.0 ** -91


LINEARS = [
    # rows, in_dim, out_dim, group, fmt, scales
    (1, 128, 1, 128, "fp8", "fp32"), (1, 512, 2048, 128, "fp8", "bf16"), (2, 16, 33, 16, "fp8", "fp32"), (3, 576, 2304, 576, "fp8", "fp32"),
    (16, 1024, 1000, 256, "int4", "bf16"), (17, 6912, 257, 128, "fp8", "fp32"), (64, 2304, 129, 2304, "int4", "fp32"), (65, 1408, 2048, 128, "int4", "bf16"),
    (127, 1152, 300, 384, "fp8", "bf16"), (200, 272, 777, 272, "int4", "bf16"), (257, 640, 1153, 128, "fp8", "fp32"), (513, 48, 96, 10 ** 9, "fp8", "fp32"),
    (1025, 1152, 640, 1152, "fp8", "bf16"), (700, 2048, 1408, 2048, "int4", "fp32"),
    # one step of the inner axis, or a piece of one; tiles that are split along it, with odd widths; whole rounds of tiles and a rest
    # few rows: each width of a workgroup with each number of rows
    (9, 256, 12301, 128, "fp8", "fp32"), (30, 144, 12301, 144, "fp8", "bf16"), (20, 272, 6150, 272, "fp8", "fp32"), (50, 2048, 200, 128, "fp8", "fp32"),
    (16, 400, 6150, 400, "int4", "fp32"), (2, 256, 12300, 256, "int4", "bf16"), (32, 256, 12301, 128, "int4", "fp32"), (60, 256, 12301, 256, "int4", "fp32"), (64, 144, 6150, 144, "int4", "bf16"),
    (100, 16, 40, 16, "fp8", "fp32"), (70, 6912, 301, 128, "fp8", "fp32"), (4100, 4096, 1030, 4096, "int4", "fp32"), (8200, 128, 2200, 128, "fp8", "bf16"),
]


def make_linear(rows, in_dim, out_dim, group, fmt, scales):
    gen = torch.Generator().manual_seed(rows * 31 + in_dim * 7 + out_dim)
    codes, code_scales = activations(rows, in_dim, gen)
    w, ws, values = weights(out_dim, in_dim, fmt, group, scales, gen)
    return gen, codes, code_scales, rows8_values(codes, code_scales), w, ws, values


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,in_dim,out_dim,group,fmt,scales", LINEARS)
def test_linear(harness, rows, in_dim, out_dim, group, fmt, scales, out):
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, group, fmt, scales)
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, fmt=FMT[fmt], group_size=group, out_dtype=DTYPE[out])
    y, tol = x @ values.t(), product_bound(x, values, exact=out == "fp32")
    hold(unit.forward(codes, code_scales), y, tol, "out")
    add = torch.randn(rows, out_dim, generator=gen).to(DTYPE[out]).cuda()
    hold(unit.forward(codes, code_scales, add=add), y + add.double(), tol + (y.abs() + add.double().abs()) * 2.0 ** -23, "out + add")


@pytest.mark.parametrize("rows,in_dim,out_dim,group,fmt,scales", LINEARS)
def test_linear_gradients(harness, rows, in_dim, out_dim, group, fmt, scales):
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, group, fmt, scales)
    unit = harness.Linear(rows, in_dim, out_dim, weights=w, scales=ws, fmt=FMT[fmt], group_size=group, training=True)
    grad = (torch.randn(rows, out_dim, generator=gen) * torch.exp2(4 * torch.randn(rows, 1, generator=gen))).bfloat16().cuda()
    unit.forward(codes, code_scales)
    grad_input, grad_weights = unit.backward(grad)
    g = grad.double()
    want = gradients_exact([g], [values], x, [torch.zeros_like(g)])
    hold(grad_input, want["grad_input"], want["grad_input_tol"], "grad_input")
    hold(grad_weights, want["grad_0"], want["grad_0_tol"], "grad_weights")


GATED = [
    # rows, in_dim, width, group, fmt, scales, act
    (1, 128, 128, 128, "fp8", "fp32", "silu"), (1, 1152, 6912, 128, "fp8", "fp32", "gelu"), (2, 16, 1, 16, "fp8", "bf16", "silu"), (5, 576, 130, 576, "int4", "fp32", "gelu"),
    (16, 1024, 1024, 128, "fp8", "fp32", "silu"), (31, 2048, 1408, 128, "int4", "bf16", "silu"), (64, 320, 255, 320, "fp8", "fp32", "gelu"),
    (65, 512, 2048, 256, "fp8", "bf16", "silu"), (130, 1152, 391, 1152, "int4", "bf16", "gelu"), (300, 1024, 1000, 128, "fp8", "fp32", "silu"),
    (513, 144, 4100, 10 ** 9, "fp8", "fp32", "gelu"), (1030, 384, 640, 384, "fp8", "fp32", "silu"),
    (9, 256, 12301, 128, "fp8", "fp32", "silu"), (30, 144, 12301, 144, "fp8", "bf16", "gelu"), (20, 272, 6150, 272, "fp8", "fp32", "silu"), (50, 1024, 200, 128, "fp8", "fp32", "silu"),
    (2, 256, 6150, 256, "int4", "fp32", "gelu"), (32, 256, 12301, 128, "int4", "fp32", "silu"), (60, 256, 12301, 256, "int4", "fp32", "silu"), (64, 144, 6150, 144, "int4", "bf16", "silu"),
    (4100, 128, 2500, 128, "int4", "fp32", "gelu"), (66, 16, 7, 16, "fp8", "fp32", "silu"), (2100, 2048, 130, 256, "fp8", "bf16", "silu"),
]


def make_gated(rows, in_dim, width, group, fmt, scales):
    gen = torch.Generator().manual_seed(rows * 37 + in_dim * 5 + width)
    codes, code_scales = activations(rows, in_dim, gen)
    return gen, codes, code_scales, rows8_values(codes, code_scales), weights(width, in_dim, fmt, group, scales, gen), weights(width, in_dim, fmt, group, scales, gen)


@pytest.mark.parametrize("rows,in_dim,width,group,fmt,scales,act", GATED)
def test_gated(harness, rows, in_dim, width, group, fmt, scales, act):
    gen, codes, code_scales, x, gate, up = make_gated(rows, in_dim, width, group, fmt, scales)
    unit = harness.GatedUnit(rows, in_dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], fmt=FMT[fmt], group_size=group, act=act, training=True)
    h, h_scales = unit.forward(codes, code_scales)
    grad = (torch.randn(rows, width, generator=gen) * torch.exp2(4 * torch.randn(rows, 1, generator=gen))).bfloat16().cuda()
    grads = unit.backward(grad)
    want = gated_exact(x, gate[2], up[2], act, grad)
    hold_rows8(h, h_scales, want["h"], want["h_tol"], "h")
    for got, name in zip(grads, ("grad_input", "grad_0", "grad_1")):
        hold(got, want[name], want[name + "_tol"], name)


@pytest.mark.parametrize("rows,in_dim,width,fmt", [(40, 256, 133, "fp8"), (200, 256, 391, "int4"), (1100, 384, 640, "int4"), (700, 128, 2000, "fp8"), (20, 512, 100, "int4")])
def test_one_gradient_alone(harness, rows, in_dim, width, fmt):
    """The others are NULL in the descriptor: theirs are left alone."""
    gen, codes, code_scales, x, gate, up = make_gated(rows, in_dim, width, 128, fmt, "fp32")
    grad = torch.randn(rows, width, generator=gen).bfloat16().cuda()
    unit = harness.GatedUnit(rows, in_dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], fmt=FMT[fmt], training=True)
    line = harness.Linear(rows, in_dim, width, weights=gate[0], scales=gate[1], fmt=FMT[fmt], training=True)
    of_unit = gated_exact(x, gate[2], up[2], "silu", grad)
    of_line = gradients_exact([grad.double()], [gate[2]], x, [torch.zeros(rows, width, dtype=torch.float64, device="cuda")])
    for u, d, want, names in ((unit, unit.gated, of_unit, ("grad_input", "grad_gate", "grad_up")), (line, line.linear, of_line, ("grad_input", "grad_weights"))):
        u.forward(codes, code_scales)
        for input_alone in (True, False):
            keep = {n: getattr(d, n) for n in names}
            for n in names:
                getattr(u, n).fill_(77.0)
                if (n == "grad_input") != input_alone:
                    setattr(d, n, None)
            u.backward(grad)
            torch.cuda.synchronize()
            for i, n in enumerate(names):
                name = "grad_input" if i == 0 else f"grad_{i - 1}"
                if (n == "grad_input") == input_alone:
                    hold(getattr(u, n), want[name], want[name + "_tol"], n)
                else:
                    assert (getattr(u, n) == 77.0).all(), n
                setattr(d, n, keep[n])


def run_layer(harness, rows, device="cuda"):
    """The feed-forward half of a layer, forward and backward: a dict of everything that it makes."""
    dim, width = 576, 1152
    gen = torch.Generator().manual_seed(rows)
    gate, up, down = weights(width, dim, "fp8", 576, "fp32", gen), weights(width, dim, "fp8", 576, "fp32", gen), weights(dim, width, "fp8", 128, "bf16", gen)
    x, r = (torch.randn(rows, dim, generator=gen).bfloat16().cuda() for _ in range(2))
    gain = (1 + 0.1 * torch.randn(dim, generator=gen)).bfloat16().cuda()
    grad = (torch.randn(rows, dim, generator=gen) / 8).bfloat16().cuda()
    norm = harness.RowNorm(rows, dim, gain=gain, residual=True, training=True)
    unit = harness.GatedUnit(rows, dim, width, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], group_size=576, training=True)
    last = harness.Linear(rows, width, dim, weights=down[0], scales=down[1], group_size=128, training=True)

    def step():
        y, ys, total = norm.forward(x, r)
        h, hs = unit.forward(y, ys)
        out = last.forward(h, hs, add=total)
        grad_h, grad_down = last.backward(grad)
        grad_y, grad_gate, grad_up = unit.backward(grad_h)
        grad_x, grad_gain = norm.backward(grad_y, grad)
        return dict(y=y, ys=ys, total=total, h=h, hs=hs, out=out, grad_h=grad_h, grad_down=grad_down, grad_y=grad_y, grad_gate=grad_gate, grad_up=grad_up,
                    grad_x=grad_x, grad_gain=grad_gain)
    return step, dict(x=x, r=r, gain=gain, grad=grad, gate=gate[2], up=up[2], down=down[2])


@pytest.mark.parametrize("rows", [1, 77, 600])
def test_a_layers_half(harness, rows):
    """Each output against float64 from what was really its input."""
    step, s = run_layer(harness, rows)
    got = step()
    want = norm_exact(got["total"].double(), s["gain"].double(), 1e-6, got["grad_y"], s["grad"])
    hold_rows8(got["y"], got["ys"], want["y"], want["y_tol"], "y")
    hold(got["grad_x"], want["grad_input"], want["grad_input_tol"], "grad_x")
    hold(got["grad_gain"], want["grad_gain"], want["grad_gain_tol"], "grad_gain")
    y, h = rows8_values(got["y"], got["ys"]), rows8_values(got["h"], got["hs"])
    want = gated_exact(y, s["gate"], s["up"], "silu", got["grad_h"])
    hold_rows8(got["h"], got["hs"], want["h"], want["h_tol"], "h")
    for name, key in (("grad_y", "grad_input"), ("grad_gate", "grad_0"), ("grad_up", "grad_1")):
        hold(got[name], want[key], want[key + "_tol"], name)
    t = got["total"].double()
    p = h @ s["down"].t()
    hold(got["out"], p + t, product_bound(h, s["down"]) + (p.abs() + t.abs()) * 2.0 ** -23, "out")
    g = s["grad"].double()
    want = gradients_exact([g], [s["down"]], h, [torch.zeros_like(g)])
    hold(got["grad_h"], want["grad_input"], want["grad_input_tol"], "grad_h")
    hold(got["grad_down"], want["grad_0"], want["grad_0_tol"], "grad_down")


@pytest.mark.parametrize("rows", [3, 300])
def test_captured_layers_half(harness, rows):
    """Captured into a graph and replayed between eager work: the bits of the eager pass every time."""
    step, s = run_layer(harness, rows)
    want = {k: v.clone() for k, v in step().items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        for t in got.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in got.items():
            assert torch.equal(t.view(torch.uint8), want[name].view(torch.uint8)), (k, name)
        (s["x"].float() * 2).sum().item()


def test_runs_are_the_same_bits(harness):
    step, _ = run_layer(harness, 333)
    first = {k: v.clone() for k, v in step().items()}
    for name, t in step().items():
        assert torch.equal(t.view(torch.uint8), first[name].view(torch.uint8)), name


def test_another_stream(harness):
    step, s = run_layer(harness, 200)
    want = {k: v.clone() for k, v in step().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    for name, t in got.items():
        assert torch.equal(t.view(torch.uint8), want[name].view(torch.uint8)), name


def test_fewer_rows_leave_the_others_alone(harness):
    """Units made for more rows, called with fewer and with none: what lies behind the last row is neither read nor written."""
    gen, codes, code_scales, x, gate, up = make_gated(90, 256, 200, 256, "fp8", "fp32")
    down = weights(256, 208, "fp8", 208, "fp32", gen)
    unit = harness.GatedUnit(90, 256, 200, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], group_size=256, training=True)
    last = harness.Linear(90, 208, 256, weights=down[0], scales=down[1], group_size=208, training=True)
    norm = harness.RowNorm(90, 256, gain=torch.ones(256, device="cuda"), residual=True, training=True)
    many = [codes.clone(), code_scales.clone()]
    for n in (41, 1, 0):
        for t in (unit.out, unit.scales, unit.grad_input, last.out, last.grad_input, norm.out, norm.scales, norm.sum, norm.grad_input):
            t.view(torch.uint8).fill_(0x5A)
        codes[n:].fill_(0x7F)                                # NaN: not read
        code_scales[n:].fill_(0xFF)
        grad = torch.full((90, 200), float("nan"), dtype=torch.bfloat16, device="cuda")
        grad[:n] = 0.5
        h, hs = unit.forward(codes[:n], code_scales[:n])
        grads = unit.backward(grad[:n])
        assert h.shape == (n, 200) and hs.shape == (n, 2) and grads[0].shape == (n, 256)
        want = gated_exact(rows8_values(many[0][:n], many[1][:n]), gate[2], up[2], "silu", grad[:n])
        if n:
            hold_rows8(h, hs, want["h"], want["h_tol"], "h")
            hold(grads[0], want["grad_input"], want["grad_input_tol"], "grad_input")
        hold(grads[1], want["grad_0"], want["grad_0_tol"] + 1e-30, "grad_gate")
        hold(grads[2], want["grad_1"], want["grad_1_tol"] + 1e-30, "grad_up")
        wide = torch.full((90, 208), 0x7F, dtype=torch.uint8, device="cuda")
        wide[:n] = 0x38                                       # ones
        ones = torch.full((90, 2), 0xFF, dtype=torch.uint8, device="cuda")
        ones[:n] = 127
        out = last.forward(wide[:n], ones[:n])
        g = torch.full((90, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
        g[:n] = 1.0
        grad_input, grad_weights = last.backward(g[:n])
        assert out.shape == (n, 256) and (grad_weights == n).all() and torch.isfinite(grad_input).all()
        z = torch.full((90, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
        z[:n] = 1.0
        norm.forward(z[:n], z[:n])
        grad_z, grad_gain = norm.backward(z[:n])
        assert grad_z.shape == (n, 256) and torch.isfinite(grad_gain).all() and (n or not grad_gain.any())
        for t in (unit.out, unit.scales, unit.grad_input, last.out, last.grad_input, norm.out, norm.scales, norm.sum, norm.grad_input):
            assert (t[n:].view(torch.uint8) == 0x5A).all()


@pytest.mark.parametrize("out_dim", [256, 136, 133])
def test_strides_and_alignments(eco, out_dim):
    """Rows that lie apart, at any alignment that is allowed, in the C calls: the same bits as packed ones, and nothing written between the rows."""
    rows, in_dim = 70, 272
    gen, codes, code_scales, x, w, ws, values = make_linear(rows, in_dim, out_dim, 272, "fp8", "fp32")
    grad = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    add = torch.randn(rows, out_dim, generator=gen).bfloat16().cuda()
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    sizes = dict(rows=rows, in_dim=in_dim, out_dim=out_dim, group_size=272)

    def run(pad, shift):
        wide = lambda t, by: torch.full((rows, t.shape[1] + by + shift), 0x5A, dtype=t.dtype, device="cuda")[:, shift:shift + t.shape[1]].copy_(t)   # noqa: E731
        c = torch.full((rows, in_dim + 16 * pad), 0x7F, dtype=torch.uint8, device="cuda")
        c[:, :in_dim] = codes
        a, g = wide(add, 3 * pad), wide(grad, 5 * pad)
        out = torch.full((rows, out_dim + 7 * pad + shift), 9.0, dtype=torch.bfloat16, device="cuda")
        gi = torch.full((rows, in_dim + pad + shift), 9.0, dtype=torch.bfloat16, device="cuda")
        gw = torch.empty(out_dim, in_dim, dtype=torch.bfloat16, device="cuda")
        d = eco.make_linear(**sizes, codes=c, code_scales=code_scales, weights=w, scales=ws, add=a, out=out[:, shift:], grad_out=g, grad_input=gi[:, shift:], grad_weights=gw,
                            codes_stride=c.stride(0), add_stride=a.stride(0), out_stride=out.stride(0), grad_out_stride=g.stride(0), grad_input_stride=gi.stride(0))
        assert max(eco.eco_linear_workspace(d, False), eco.eco_linear_workspace(d, True)) <= work.numel()
        eco.eco_linear(d, work, work.numel())
        eco.eco_linear_backward(d, work, work.numel())
        for t, n in ((out, out_dim), (gi, in_dim)):
            assert (t[:, :shift] == 9).all() and (t[:, shift + n:] == 9).all()
        return out[:, shift:shift + out_dim].clone(), gi[:, shift:shift + in_dim].clone(), gw

    packed = run(0, 0)
    for pad, shift in ((1, 0), (1, 1), (3, 5)):
        for k, (p, q) in enumerate(zip(packed, run(pad, shift))):
            assert torch.equal(p, q), (pad, shift, k)


def test_in_place(eco):
    """sum over the residual or the input, grad_input over grad_out or grad_sum, out over add: as elsewhere."""
    rows, dim = 37, 1160
    gen = torch.Generator().manual_seed(2)
    x, r, g, gs = (torch.randn(rows, dim, generator=gen).bfloat16().cuda() for _ in range(4))
    gain = torch.ones(dim, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def run(over_sum, over_grad):
        a = {k: t.clone() for k, t in (("input", x), ("residual", r), ("grad_out", g), ("grad_sum", gs))}
        total = a.get(over_sum, torch.empty_like(x))
        gi = a.get(over_grad, torch.empty_like(x))
        out, scales, rstd = torch.empty(rows, dim, dtype=torch.uint8, device="cuda"), torch.empty(rows, 10, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
        gg = torch.empty(dim, dtype=torch.bfloat16, device="cuda")
        d = eco.make_norm(rows=rows, dim=dim, eps=1e-6, sum=total, gain=gain, out=out, scales=scales, rstd=rstd, grad_input=gi, grad_gain=gg, **a)
        eco.eco_norm(d)
        eco.eco_norm_backward(d, work, work.numel())
        return total.clone(), out, scales, rstd, gi.clone(), gg
    want = run(None, None)
    for where in (("input", "grad_out"), ("residual", "grad_sum")):
        for k, (p, q) in enumerate(zip(want, run(*where))):
            assert torch.equal(p, q), (where, k)


def test_values_that_are_not_finite_stay_in_their_rows(harness):
    """NaN and infinities of a row reach that row's results alone and, of the gradients of weights, what depends on it."""
    gen, codes, code_scales, x, gate, up = make_gated(40, 144, 100, 144, "fp8", "fp32")
    unit = harness.GatedUnit(40, 144, 100, gate=gate[0], gate_scales=gate[1], up=up[0], up_scales=up[1], group_size=144)
    last = harness.Linear(40, 144, 100, weights=gate[0], scales=gate[1], group_size=144, training=True)
    clean = [t.clone() for t in (*unit.forward(codes, code_scales), last.forward(codes, code_scales))]
    codes[7, 143] = 0x7F                                     # in the last piece, whose block is short
    code_scales[9, 0] = 0xFF
    codes[9, :128] = 0x7F
    got = [*unit.forward(codes, code_scales), last.forward(codes, code_scales)]
    there = torch.ones(40, dtype=torch.bool, device="cuda")
    there[[7, 9]] = False
    for p, q in zip(clean, got):
        assert torch.equal(p[there], q[there])
    assert (got[0][~there] == 0x7F).all() and (got[1][~there] == 0xFF).all() and got[2][~there].isnan().all()
    grad = torch.ones(40, 100, dtype=torch.bfloat16, device="cuda")
    grad_input, grad_weights = last.backward(grad)
    assert torch.isfinite(grad_input).all() and grad_weights[:, 143].isnan().all() and torch.isfinite(grad_weights[:, 128:143]).all()
    grad[39, 99] = float("inf")                               # the last row, which the inner axis' last step repeats
    grad_input, _ = last.backward(grad)
    assert torch.isfinite(grad_input[:39]).all() and not torch.isfinite(grad_input[39]).any()


def test_extreme_activations(harness):
    """Gates far past the activations' ends: finite, and the limits where they are limits."""
    codes = torch.full((2, 128), 0x7E, dtype=torch.uint8, device="cuda")       # 448
    scales = torch.tensor([[127 + 20], [127 + 60]], dtype=torch.uint8, device="cuda")
    gate = torch.full((4, 128), 0x38, dtype=torch.uint8, device="cuda")
    gate[1], gate[3] = 0xB8, 0xB8                             # -1
    s = torch.full((4,), 1.0, device="cuda")
    up = torch.full((4, 128), 0x38, dtype=torch.uint8, device="cuda")
    for act in ("silu", "gelu"):
        unit = harness.GatedUnit(2, 128, 4, gate=gate, gate_scales=s, up=up, up_scales=s * 2.0 ** -60, group_size=128, act=act, training=True)
        h, hs = unit.forward(codes, scales)
        v = rows8_values(h, hs)
        assert torch.isfinite(v).all() and (v[:, 1] == 0).all() and (v[:, 3] == 0).all()
        for k, e in enumerate((20, 60)):
            want = (448.0 * 128 * 2.0 ** e) ** 2 * 2.0 ** -60
            assert abs(v[k, 0].item() / want - 1) <= 2.0 ** -4 and v[k, 2] == v[k, 0]
        grads = unit.backward(torch.full((2, 4), 2.0 ** -20, dtype=torch.bfloat16, device="cuda"))
        assert all(torch.isfinite(g).all() for g in grads)


def test_offsets_past_32_bits(harness):
    """More than 2^32 codes: the last rows come out as they do by themselves."""
    rows, dim, width = 65600, 65536, 16
    gen = torch.Generator().manual_seed(5)
    end = torch.randn(8, dim, generator=gen).bfloat16().cuda()
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    x[-8:] = end
    codes, scales = harness.quantize_rows(x)
    want_codes, want_scales = harness.quantize_rows(end)
    assert torch.equal(codes[-8:], want_codes) and torch.equal(scales[-8:], want_scales) and not codes[:-8].any()
    norm = harness.RowNorm(rows, dim, quantize=False)
    assert torch.equal(norm.forward(x)[0][-8:], harness.RowNorm(8, dim, quantize=False).forward(end)[0])
    del x, norm
    w, ws, values = weights(width, dim, "fp8", 128, "fp32", gen)
    unit = harness.Linear(rows, dim, width, weights=w, scales=ws, training=True)
    v = rows8_values(want_codes, want_scales)
    hold(unit.forward(codes, scales)[-8:], v @ values.t(), product_bound(v, values), "out")
    grad = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    grad[-8:] = torch.randn(8, width, generator=gen).bfloat16().cuda()
    grad_input, grad_weights = unit.backward(grad)
    g = grad[-8:].double()
    want = gradients_exact([g], [values], v, [torch.zeros_like(g)])
    hold(grad_input[-8:], want["grad_input"], want["grad_input_tol"], "grad_input")
    assert not grad_input[:-8].any()
    hold(grad_weights, want["grad_0"], want["grad_0_tol"] + 1e-30, "grad_weights")


def test_units_at_once_on_two_streams(harness):
    """Each with its own workspace, and what the allocator is told where a stream is given: the bits of one after the other."""
    layers = [run_layer(harness, rows) for rows in (300, 500)]
    want = [{k: v.clone() for k, v in step().items()} for step, _ in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(3):
        got = []
        for (step, _), s in zip(layers, streams):
            with torch.cuda.stream(s):
                got.append(step())
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for name, t in g.items():
                assert torch.equal(t.view(torch.uint8), w[name].view(torch.uint8)), name


def test_a_stream_that_is_given(harness):
    gen, codes, code_scales, x, w, ws, values = make_linear(90, 256, 130, 256, "fp8", "fp32")
    unit = harness.Linear(90, 256, 130, weights=w, scales=ws, group_size=256, training=True)
    grad = torch.ones(90, 130, dtype=torch.bfloat16, device="cuda")
    want = [unit.forward(codes, code_scales).clone(), *(t.clone() for t in unit.backward(grad))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (side, side.cuda_stream):
        got = [unit.forward(codes, code_scales, stream=s), *unit.backward(grad, stream=s)]
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_refusals(harness):
    """A refused call leaves the object as it was."""
    gen, codes, code_scales, x, w, ws, values = make_linear(9, 256, 130, 256, "fp8", "fp32")
    unit = harness.Linear(9, 256, 130, weights=w, scales=ws, group_size=256, training=True)
    with pytest.raises(RuntimeError, match="forward"):
        unit.backward(torch.ones(9, 130, dtype=torch.bfloat16, device="cuda"))
    first = unit.forward(codes, code_scales).clone()
    more = torch.zeros(10, 256, dtype=torch.uint8, device="cuda")
    for bad in ((codes.int(), code_scales), (codes[:, :240], code_scales), (codes, code_scales[:, :1]), (codes.cpu(), code_scales), (codes, code_scales[:5]), (None, code_scales),
                (codes, None), (more, more[:, :2]), (codes.t().contiguous().t(), code_scales), (codes[0], code_scales)):
        with pytest.raises(ValueError):
            unit.forward(*bad)
    for bad in (torch.ones(9, 130, device="cuda"), torch.ones(9, 130, dtype=torch.bfloat16), torch.ones(8, 130, dtype=torch.bfloat16, device="cuda"), None):
        with pytest.raises(ValueError):
            unit.backward(bad)
    grad = torch.ones(9, 130, dtype=torch.bfloat16, device="cuda")
    unit.backward(grad)
    assert torch.equal(unit.forward(codes, code_scales), first)
    plain = harness.Linear(9, 256, 130, weights=w, scales=ws, group_size=256)
    plain.forward(codes, code_scales)
    with pytest.raises(RuntimeError, match="training"):
        plain.backward(grad)
    with pytest.raises(ValueError):
        harness.Linear(9, 256, 130, weights=w[:-1], scales=ws, group_size=256)
    with pytest.raises(ValueError):
        harness.Linear(9, 256, 130, weights=w, scales=ws[:-1], group_size=256)
    with pytest.raises(ValueError):
        harness.GatedUnit(9, 256, 130, gate=w, gate_scales=ws, up=w, up_scales=ws.bfloat16(), group_size=256)
    with pytest.raises(ValueError):
        harness.GatedUnit(9, 256, 130, gate=w, gate_scales=ws, up=w, up_scales=ws, group_size=256, act="relu")
    norm = harness.RowNorm(9, 256, gain=torch.ones(256, device="cuda"))
    with pytest.raises(ValueError):
        norm.forward(torch.ones(9, 256, dtype=torch.bfloat16, device="cuda"), torch.ones(9, 256, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        harness.RowNorm(9, 256, gain=torch.ones(255, device="cuda"))


@pytest.mark.parametrize("fmt,act", [("fp8", "silu"), ("int4", "gelu")])
def test_the_example_runs(fmt, act):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_ffn.py")
    spec = importlib.util.spec_from_file_location("train_ffn", path)
    train_ffn = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(train_ffn)
    losses, layer = train_ffn.train(steps=2, rows=130, fmt=fmt, act=act)
    assert len(losses) == 2 and all(l > 0 and l == l for l in losses)
    for m, v in layer.state:
        assert torch.isfinite(m).all() and m.any() and (v >= 0).all() and v.any()
