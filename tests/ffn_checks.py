"""Checks of the feed-forward half's results beside the element-wise ones of ffn_util: 8-bit rows that hold no NaN, and the size of a whole array's error.

An element's bound allows for the worst signs of a few thousand roundings, which is some per cent of a result, and a lost term among thousands hides in it.  The whole array's error does
not: roundings have independent signs, so that
  * a rounding to nearest is, over many values, at most ROUND = 2^-8 / sqrt(3) of them for bf16 (uniform in half a step, 2^-8 of the value's power of two);
  * a sum of products whose one factor is rounded is off by ROUND of the root of the sum of its squared products;
  * the 8-bit instruction leaves out of eight neighbouring products what lies below 2^-13 of the largest: at most sqrt(7) 2^-13 of that root.
The square root of the sum of their squares is the error that is expected at most, and TWICE it the bound.  A term that is lost of n makes an error of 1 / sqrt(n) of the result:
the bound of 2 sqrt(2) ROUND (two roundings) shows one of 24000.  That is so for many results: arrays of less than MANY are left to the element-wise bounds.

Codes: an error of sqrt(7) 2^-13 = 3.2e-4 of a product's typical size moves a code, whose steps are 1/16 to 1/8 of its value, in 0.5 % of the cases; values ten times smaller than typical, a
tenth of all, have ten times the relative error and so add as much, for the three and a half decades down to the smallest code: at most 2 % in all.
"""
import torch

import ffn_util

ROUND = 2.0 ** -8 / 3 ** 0.5
LEFT_OUT = 7 ** 0.5 * 2.0 ** -13
TWICE, MANY = 2.0, 4096
MOVED = 0.02


def root(x, w):
    """The root of the sum of squared products, of each result of x w."""
    return (x.square() @ w.square()).sqrt()


def hold_whole(got, parts, want, name):
    """`parts`: arrays whose norms are those of errors with independent signs."""
    if want.numel() < MANY:
        return
    assert got.dtype == torch.bfloat16
    bound = TWICE * sum(p.double().norm().item() ** 2 for p in [want * ROUND, *parts]) ** 0.5
    error = (got.double() - want).norm().item()
    assert error <= bound, f"{name}: an error of {error / want.norm().item():.3g} of the result, {error / bound:.3g} times its bound"


def hold_rows8(codes, scales, y, d, name):
    """As ffn_util's, of rows in which no code may be NaN: no comparison is true of one, so that its bounds let it through."""
    assert torch.isfinite(codes.view(torch.float8_e4m3fn).double()).all(), f"{name}: a code that is not finite"
    ffn_util.hold_rows8(codes, scales, y, d, name)


def hold_moved(codes, scales, y, name):
    """Of all codes in blocks with the right scale, and of all scales, hardly any are not those of y."""
    want_codes, want_scales = ffn_util.rows8(y)
    right = scales == want_scales
    there = right.repeat_interleave(128, 1)[:, :y.shape[1]]
    if y.numel() < MANY:
        return
    moved = (codes.view(torch.float8_e4m3fn).double() != want_codes.view(torch.float8_e4m3fn).double()) & there
    assert moved.sum().item() <= MOVED * y.numel(), f"{name}: {moved.sum().item()} of {y.numel()} codes"
    assert (~right).sum().item() <= MOVED * right.numel() + 1, f"{name}: {(~right).sum().item()} of {right.numel()} scales"
