"""Figures that include/mosaic_layer.h gives a caller to reckon with."""
import re

import torch

from test_layer_host_api import header


def test_what_a_rounding_to_bf16_adds():
    """The bound stated for a term's rounding holds for the worst number there is, and no smaller power of two does."""
    v = 1 + torch.arange(1, 1 << 15, dtype=torch.float64) / (1 << 15)          # a whole binade
    worst = ((v.to(torch.bfloat16).double() - v).abs() / v).max().item()
    text = re.sub(r"\s+\*?\s*", " ", header())
    stated = [float(2 ** -int(n)) for n in re.findall(r"2\^-(\d+) relative", text)]
    assert stated and all(s / 2 < worst <= s for s in stated)
