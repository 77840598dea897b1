"""Outputs of the feed-forward half that are inputs, where other workgroups still read them: refused before any device work."""
import pytest

from test_ffn_host import eco, gated, linear, norm, status      # noqa: F401


def test_outputs_over_inputs_are_refused(eco):      # noqa: F811
    calls = [(lambda: eco.eco_rows_quantize(0x1000, 0, 4, 128, 0, 0x1000, 0, 0x3000, 0), "codes is src"),
             (lambda: eco.eco_norm(norm(eco, out=0x1000), 0), "out is input"), (lambda: eco.eco_norm(norm(eco, out=0x2000), 0), "out is residual"),
             (lambda: eco.eco_norm(norm(eco, out=0x3000), 0), "out is sum"),
             (lambda: eco.eco_linear(linear(eco, out=0x1000), 0x100000, 1 << 40, 0), "out is codes"),
             (lambda: eco.eco_linear_backward(linear(eco, grad_input=0x7000), 0x100000, 1 << 40, 0), "grad_input is grad_out"),
             (lambda: eco.eco_gated(gated(eco, out=0x1000), 0x100000, 1 << 40, 0), "out is codes"),
             (lambda: eco.eco_gated(gated(eco, out_scales=0x2000), 0x100000, 1 << 40, 0), "out_scales is code_scales")]
    for call, message in calls:
        with pytest.raises(eco.EcoError, match=message) as e:
            call()
        assert e.value.status == eco.ECO_EINVAL
