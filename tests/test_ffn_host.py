"""The feed-forward half of a layer without a GPU: refusals before any device work, workspaces, and the tests' own formulas against autograd."""
import ctypes as C
import os

import pytest
import torch

import ffn_util


@pytest.fixture(scope="module")
def eco():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if not os.path.exists(os.path.join(root, "paper_2601_22101_amd", "libeco.so")):
        from paper_2601_22101_amd import build
        build.build()
    from paper_2601_22101_amd import binding
    return binding


def status(eco, fn, *args):
    try:
        fn(*args)
    except eco.EcoError as e:
        assert eco.eco_last_error()
        return e.status
    return 0


def norm(eco, **kw):
    return eco.make_norm(**{**dict(rows=4, dim=512, eps=1e-6, input=0x1000, residual=0x2000, sum=0x3000, gain=0x4000, out=0x5000, scales=0x6000, rstd=0x7000, grad_out=0x8000,
                                   grad_sum=0x9000, grad_input=0xA000, grad_gain=0xB000), **kw})


def linear(eco, **kw):
    return eco.make_linear(**{**dict(rows=4, in_dim=512, out_dim=256, group_size=128, codes=0x1000, code_scales=0x2000, weights=0x3000, scales=0x4000, add=0x5000, out=0x6000,
                                     grad_out=0x7000, grad_input=0x8000, grad_weights=0x9000), **kw})


def gated(eco, **kw):
    return eco.make_gated(**{**dict(rows=4, in_dim=512, width=256, group_size=128, codes=0x1000, code_scales=0x2000, gate=0x3000, gate_scales=0x4000, up=0x5000, up_scales=0x6000,
                                    out=0x7000, out_scales=0x8000, grad_out=0x9000, grad_input=0xA000, grad_gate=0xB000, grad_up=0xC000), **kw})


def test_struct_layouts(eco):
    assert (C.sizeof(eco.eco_norm_t), C.sizeof(eco.eco_linear_t), C.sizeof(eco.eco_gated_t)) == (184, 160, 176)


def test_norm_refusals(eco):
    both = [(dict(dim=0), eco.ECO_EINVAL), (dict(eps=0.0), eco.ECO_EINVAL), (dict(eps=float("nan")), eco.ECO_EINVAL), (dict(eps=-1.0), eco.ECO_EINVAL), (dict(eps=1e-60), eco.ECO_EINVAL),
            (dict(dtype=7), eco.ECO_EINVAL), (dict(gain_dtype=7), eco.ECO_EINVAL), (dict(gain=0x4001), eco.ECO_EALIGN), (dict(rows=(1 << 23) + 1), eco.ECO_EUNSUPPORTED),
            (dict(dim=(1 << 16) + 1), eco.ECO_EUNSUPPORTED), (dict(sum_stride=511), eco.ECO_EINVAL), (dict(sum_stride=1 << 23), eco.ECO_EUNSUPPORTED)]
    forward = [(dict(input=None), eco.ECO_EINVAL), (dict(sum=None), eco.ECO_EINVAL), (dict(residual=None), eco.ECO_EINVAL), (dict(out=None), eco.ECO_EINVAL),
               (dict(input=0x1001), eco.ECO_EALIGN), (dict(out=0x5001, scales=None), eco.ECO_EALIGN), (dict(rstd=0x7002), eco.ECO_EALIGN), (dict(input_stride=1), eco.ECO_EINVAL),
               (dict(residual_stride=100), eco.ECO_EINVAL), (dict(out_stride=100), eco.ECO_EINVAL)]
    backward = [(dict(grad_out=None), eco.ECO_EINVAL), (dict(rstd=None), eco.ECO_EINVAL), (dict(sum=None, input=None), eco.ECO_EINVAL),
                (dict(grad_input=None, grad_gain=None), eco.ECO_EINVAL), (dict(grad_gain_dtype=9), eco.ECO_EINVAL), (dict(grad_gain=0xB001), eco.ECO_EALIGN),
                (dict(grad_out=0x8001), eco.ECO_EALIGN), (dict(grad_input_stride=7), eco.ECO_EINVAL), (dict(grad_sum_stride=7), eco.ECO_EINVAL)]
    for kw, want in both + forward:
        assert status(eco, eco.eco_norm, norm(eco, **kw), 0) == want, kw
    for kw, want in both + backward:
        assert status(eco, eco.eco_norm_backward, norm(eco, **kw), 0x10000, 1 << 30, 0) == want, kw
    need = eco.eco_norm_backward_workspace(norm(eco))
    assert need == 4 * 512
    assert status(eco, eco.eco_norm_backward, norm(eco), None, 0, 0) == eco.ECO_EINVAL
    assert status(eco, eco.eco_norm_backward, norm(eco), 0x10000, need - 1, 0) == eco.ECO_EINVAL and str(need) in eco.eco_last_error()
    assert status(eco, eco.eco_norm_backward, norm(eco), 0x10080, need, 0) == eco.ECO_EALIGN
    q = lambda **kw: status(eco, eco.eco_rows_quantize, *{**dict(src=0x1000, t=0, rows=4, dim=100, stride=0, codes=0x2000, cs=0, scales=0x3000, stream=0), **kw}.values())   # noqa: E731
    assert q(src=None) == q(codes=None) == q(scales=None) == q(dim=0) == q(t=5) == q(stride=99) == q(cs=99) == eco.ECO_EINVAL
    assert q(src=0x1002) == eco.ECO_EALIGN and q(dim=70000) == eco.ECO_EUNSUPPORTED


@pytest.mark.parametrize("which", ["linear", "gated"])
def test_product_refusals(eco, which):
    make, run, back = {"linear": (linear, eco.eco_linear, eco.eco_linear_backward), "gated": (gated, eco.eco_gated, eco.eco_gated_backward)}[which]
    width = "out_dim" if which == "linear" else "width"
    w, ws = ("weights", "scales") if which == "linear" else ("up", "up_scales")
    both = [(dict(in_dim=0), eco.ECO_EINVAL), ({width: 0}, eco.ECO_EINVAL), (dict(in_dim=520, group_size=520), eco.ECO_EUNSUPPORTED), (dict(group_size=0), eco.ECO_EINVAL),
            (dict(group_size=64), eco.ECO_EUNSUPPORTED), (dict(group_size=384), eco.ECO_EUNSUPPORTED), (dict(group_size=1024), eco.ECO_EUNSUPPORTED),
            (dict(in_dim=576), eco.ECO_EUNSUPPORTED), (dict(fmt=2), eco.ECO_EUNSUPPORTED), (dict(fmt=3), eco.ECO_EUNSUPPORTED), (dict(fmt=4), eco.ECO_EINVAL),
            (dict(fmt=-1), eco.ECO_EINVAL), (dict(scale_dtype=3), eco.ECO_EINVAL), ({w: None}, eco.ECO_EINVAL), ({ws: None}, eco.ECO_EINVAL), ({w: 0x3008}, eco.ECO_EALIGN),
            ({ws: 0x4004}, eco.ECO_EALIGN), (dict(codes=None), eco.ECO_EINVAL), (dict(code_scales=None), eco.ECO_EINVAL), (dict(codes=0x1008), eco.ECO_EALIGN),
            (dict(codes_stride=520), eco.ECO_EALIGN), (dict(codes_stride=256), eco.ECO_EINVAL), (dict(codes_stride=1 << 23), eco.ECO_EUNSUPPORTED),
            (dict(rows=(1 << 23) + 1), eco.ECO_EUNSUPPORTED), (dict(rows=1 << 23, **{width: 1 << 16}), eco.ECO_EUNSUPPORTED)]
    if which == "linear":
        forward = [(dict(out=None), eco.ECO_EINVAL), (dict(out=0x6001), eco.ECO_EALIGN), (dict(out=0x6002, out_dtype=0), eco.ECO_EALIGN), (dict(add=0x5001), eco.ECO_EALIGN),
                   (dict(out_dtype=2), eco.ECO_EINVAL), (dict(add_stride=255), eco.ECO_EINVAL), (dict(out_stride=255), eco.ECO_EINVAL)]
        backward = [(dict(grad_input=None, grad_weights=None), eco.ECO_EINVAL), (dict(grad_weights=0x9008), eco.ECO_EALIGN)]
    else:
        forward = [(dict(out=None), eco.ECO_EINVAL), (dict(out_scales=None), eco.ECO_EINVAL), (dict(act=2), eco.ECO_EINVAL), (dict(act=-1), eco.ECO_EINVAL), (dict(out_stride=255), eco.ECO_EINVAL)]
        backward = [(dict(grad_input=None, grad_gate=None, grad_up=None), eco.ECO_EINVAL), (dict(grad_gate=None), eco.ECO_EINVAL), (dict(grad_up=None), eco.ECO_EINVAL),
                    (dict(grad_up=0x9008), eco.ECO_EALIGN), (dict(act=5), eco.ECO_EINVAL)]
    backward += [(dict(grad_out=None), eco.ECO_EINVAL), (dict(grad_out=0x7001), eco.ECO_EALIGN), (dict(grad_out_stride=3), eco.ECO_EINVAL), (dict(grad_input=0x8001), eco.ECO_EALIGN),
                 (dict(grad_input_stride=511), eco.ECO_EINVAL)]
    for kw, want in both + forward:
        assert status(eco, run, make(eco, **kw), 0x100000, 1 << 40, 0) == want, kw
    for kw, want in both + backward:
        assert status(eco, back, make(eco, **kw), 0x100000, 1 << 40, 0) == want, kw
    size = eco.eco_linear_workspace if which == "linear" else eco.eco_gated_workspace
    assert status(eco, back, make(eco), None, 0, 0) == eco.ECO_EINVAL
    assert status(eco, back, make(eco), 0x100080, 1 << 40, 0) == eco.ECO_EALIGN
    assert status(eco, back, make(eco), 0x100000, 1024, 0) == eco.ECO_EINVAL and "workspace" in eco.eco_last_error()
    assert status(eco, size, make(eco, group_size=64), False) == eco.ECO_EUNSUPPORTED


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_workspace_is_enough_for_fewer_rows(eco, fmt):
    """A call whose workspace is too small is refused before any device work: with the size for the most rows none is (what follows it here is the lack of a GPU, or rows = 0)."""
    for in_dim, width in ((128, 100), (6912, 1152), (1152, 6912), (2048, 1408)):
        most = 3000
        l, g = linear(eco, rows=most, in_dim=in_dim, out_dim=width, fmt=fmt), gated(eco, rows=most, in_dim=in_dim, width=width, fmt=fmt)
        sizes = [eco.eco_linear_workspace(l, b) for b in (False, True)] + [eco.eco_gated_workspace(g, b) for b in (False, True)]
        last = [0] * 4
        for rows in [0, 1, 2, 16, 17, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 640, 1000, 1025, 2047, 2049, most]:
            l.rows = g.rows = rows
            now = [eco.eco_linear_workspace(l, b) for b in (False, True)] + [eco.eco_gated_workspace(g, b) for b in (False, True)]
            assert all(a <= b for a, b in zip(last, now)), rows
            last = now
            if not torch.cuda.is_available():
                for call, d, n in ((eco.eco_linear, l, 0), (eco.eco_linear_backward, l, 1), (eco.eco_gated, g, 2), (eco.eco_gated_backward, g, 3)):
                    status(eco, call, d, 0x100000, now[n], 0)
                    assert "workspace" not in eco.eco_last_error(), (rows, n)
        assert last == sizes


@pytest.mark.parametrize("kind,fmt,in_dim,width,rows", [("gated", 1, 1216, 7167, 169), ("gated", 0, 1280, 7162, 131), ("linear", 0, 1024, 211, 28608), ("linear", 1, 1184, 166, 17051)])
def test_a_workspace_is_enough_for_tiles_of_192(eco, kind, fmt, in_dim, width, rows):
    """Few tiles of 192 columns, split in fifteen or sixteen parts, which end further behind the last column than those of 256."""
    make, size, back = {"linear": (linear, eco.eco_linear_workspace, eco.eco_linear_backward), "gated": (gated, eco.eco_gated_workspace, eco.eco_gated_backward)}[kind]
    d = make(eco, rows=rows, in_dim=in_dim, group_size=in_dim, fmt=fmt, **{"out_dim" if kind == "linear" else "width": width})
    if torch.cuda.is_available():
        pytest.skip("the pointers are none")
    status(eco, back, d, 0x100000, size(d, True), 0)
    assert "workspace" not in eco.eco_last_error()


def test_in_place_with_another_stride_is_refused(eco):
    """A row would be written over others that are still to be read."""
    for kw in (dict(sum=0x1000, sum_stride=600), dict(sum=0x2000, residual_stride=520), dict(sum=0x1000, input_stride=1024)):
        assert status(eco, eco.eco_norm, norm(eco, **kw), 0) == eco.ECO_EINVAL and "stride" in eco.eco_last_error()
    for kw in (dict(grad_input=0x8000, grad_out_stride=520), dict(grad_input=0x9000, grad_input_stride=600)):
        assert status(eco, eco.eco_norm_backward, norm(eco, **kw), 0x10000, 1 << 30, 0) == eco.ECO_EINVAL and "stride" in eco.eco_last_error()
    for kw in (dict(add=0x6000, add_stride=264), dict(add=0x6000, out_stride=512)):
        assert status(eco, eco.eco_linear, linear(eco, **kw), 0x100000, 1 << 40, 0) == eco.ECO_EINVAL and "stride" in eco.eco_last_error()
    if not torch.cuda.is_available():                         # (the same, given once as 0 and once as a number, gets past the checks)
        for d, run in ((norm(eco, sum=0x1000, sum_stride=512), lambda d: eco.eco_norm(d, 0)), (linear(eco, add=0x6000, add_stride=256), lambda d: eco.eco_linear(d, 0x100000, 1 << 40, 0))):
            assert status(eco, run, d) not in (eco.ECO_EINVAL, eco.ECO_EALIGN, eco.ECO_EUNSUPPORTED)


def test_harness_refusals():
    from paper_2601_22101_amd import harness
    w, s = torch.zeros(256, 128, dtype=torch.uint8), torch.ones(256)
    with pytest.raises(ValueError, match="GPU"):
        harness.Linear(4, 128, 256, weights=w, scales=s)
    with pytest.raises(ValueError, match="GPU"):
        harness.GatedUnit(4, 128, 256, gate=w, gate_scales=s, up=w, up_scales=s)
    with pytest.raises(ValueError, match="GPU"):
        harness.RowNorm(4, 128, gain=torch.ones(128))
    with pytest.raises(ValueError, match="GPU"):
        harness.quantize_rows(torch.zeros(4, 128))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_formulas_against_autograd(kind):
    """The tests' own gradients, in float64, on the CPU."""
    gen = torch.Generator().manual_seed(1)
    normal = lambda *shape: torch.randn(*shape, generator=gen, dtype=torch.float64)      # noqa: E731
    x, gate, up, grad = normal(5, 16).requires_grad_(), normal(7, 16).requires_grad_(), normal(7, 16).requires_grad_(), normal(5, 7)
    a = x @ gate.t()
    f = torch.nn.functional.silu(a) if kind == "silu" else torch.nn.functional.gelu(a, approximate="tanh")
    (f * (x @ up.t())).backward(grad)
    want = ffn_util.gated_exact(x.detach(), gate.detach(), up.detach(), kind, grad)
    for t, name in ((x, "grad_input"), (gate, "grad_0"), (up, "grad_1")):
        assert torch.allclose(t.grad, want[name], rtol=1e-12, atol=1e-12)
    s, gain, more = normal(3, 9).requires_grad_(), normal(9).requires_grad_(), normal(3, 9)
    g = normal(3, 9)
    (s * (s.square().mean(1, keepdim=True) + 1e-3).rsqrt() * gain).backward(g)
    want = ffn_util.norm_exact(s.detach(), gain.detach(), 1e-3, g, more)
    assert torch.allclose(s.grad + more, want["grad_input"], rtol=1e-12, atol=1e-12) and torch.allclose(gain.grad, want["grad_gain"], rtol=1e-12, atol=1e-12)


def test_rows8_of_the_tests():
    """Every E4M3 value times a power of two comes back as itself; ties go to even."""
    v = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double()
    v = v[torch.isfinite(v)]
    assert torch.equal(ffn_util.round_e4m3(v), v)
    assert ffn_util.round_e4m3(torch.tensor([17.0, 19.0, 21.0, 2.0 ** -10, 3 * 2.0 ** -10], dtype=torch.float64)).tolist() == [16, 20, 20, 0, 2 * 2.0 ** -9]
    row = torch.nn.functional.pad(v, (0, 300 - v.numel())).view(1, 300) * 2.0 ** 5
    codes, scales = ffn_util.rows8(row)
    assert torch.equal(ffn_util.rows8_values(codes, scales)[:, :128], row[:, :128])
    assert ffn_util.exponent(torch.tensor([0.0, 448.0, 449.0, 1e-40, 2.9e38, 3e38])).tolist() == [-100, 0, 1, -100, 119, 120]      # 448 2^119 = 2.98e38
