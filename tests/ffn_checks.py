"""Checks of the feed-forward half's results beside the element-wise ones of ffn_util: 8-bit rows that hold no NaN."""
import torch

import ffn_util


def hold_rows8(codes, scales, y, d, name):
    """As ffn_util's, of rows in which no code may be NaN: no comparison is true of one, so that its bounds let it through."""
    assert torch.isfinite(codes.view(torch.float8_e4m3fn).double()).all(), f"{name}: a code that is not finite"
    ffn_util.hold_rows8(codes, scales, y, d, name)
