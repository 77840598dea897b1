"""The checks of the feed-forward half's results find what they are there for: NaN codes, a wrong scale, a code one step off, one lost term of thousands.  On the CPU, with the mistakes
planted in results made from float64."""
import pytest
import torch

import ffn_checks
from ffn_checks import hold_moved, hold_rows8, hold_whole, root
from ffn_util import rows8


def rows(n=40, dim=300):
    gen = torch.Generator().manual_seed(4)
    y = torch.randn(n, dim, generator=gen, dtype=torch.float64) * torch.exp2(3 * torch.randn(n, 1, generator=gen, dtype=torch.float64))
    return y, *rows8(y)


def test_right_rows_are_taken():
    y, codes, scales = rows()
    hold_rows8(codes, scales, y, torch.zeros_like(y), "y")
    hold_moved(codes, scales, y, "y")


@pytest.mark.parametrize("nan", [0x7F, 0xFF])
@pytest.mark.parametrize("share", ["one", "block", "all"])
def test_codes_that_are_nan_are_refused(nan, share):
    y, codes, scales = rows()
    if share == "one":
        codes[3, 299] = nan
    elif share == "block":
        codes[5, 128:256] = nan
    else:
        codes[:] = nan
    with pytest.raises(AssertionError, match="not finite"):
        hold_rows8(codes, scales, y, y.abs() * 2.0 ** -20, "y")


def test_a_wrong_scale_and_a_code_one_step_off_are_refused():
    y, codes, scales = rows()
    d = y.abs() * 2.0 ** -20
    wrong = scales.clone()
    wrong[7, 1] += 1
    with pytest.raises(AssertionError, match="a scale"):
        hold_rows8(codes, wrong, y, d, "y")
    # away from a border between codes, so that no error of 2^-20 explains a step
    z = codes.view(torch.float8_e4m3fn).double()
    at = (z.abs() > 1) & (z.abs() < 400)
    i = at.nonzero()[at.sum().item() // 2]
    y = y.clone()
    s = torch.exp2(scales[i[0], i[1] // 128].double() - 127)
    y[i[0], i[1]] = z[i[0], i[1]] * s
    codes[i[0], i[1]] += 1
    with pytest.raises(AssertionError, match="codes"):
        hold_rows8(codes, scales, y, y.abs() * 2.0 ** -20, "y")
    _, codes, scales = rows()
    codes[:, ::20] ^= 1
    with pytest.raises(AssertionError, match="codes"):
        hold_moved(codes, scales, rows()[0], "y")


def test_one_lost_term_of_thousands_is_refused():
    gen = torch.Generator().manual_seed(5)
    g, w = torch.randn(64, 6912, generator=gen, dtype=torch.float64), torch.randn(6912, 128, generator=gen, dtype=torch.float64)
    rounded = w.bfloat16().double()
    want, parts = g @ w, [root(g, w) * ffn_checks.ROUND]
    hold_whole((g @ rounded).bfloat16(), parts, want, "all terms")
    g[:, 4000] = 0
    with pytest.raises(AssertionError, match="of the result"):
        hold_whole((g @ rounded).bfloat16(), parts, want, "one less")
