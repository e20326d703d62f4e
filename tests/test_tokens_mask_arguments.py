"""A dropout's site and first row as Python numbers: past the range of the library's they are refused, not taken for others (4294967296
for site 0)."""
import pytest
import torch

from paper_2601_06562_amd import binding as b


@pytest.mark.parametrize("bad", [dict(site=-1), dict(site=2 ** 31 - 1), dict(site=2 ** 32), dict(site=2 ** 32 + 5), dict(first_row=-1),
                                 dict(first_row=2 ** 63), dict(first_row=2 ** 64), dict(site=-2 ** 32)])
def test_numbers_past_the_range_are_refused(bad):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="site must lie"):
        b.mosaic_dropout_forward(x, None, x, 0.1, 1, **bad)
    with pytest.raises(ValueError, match="site must lie"):
        b.mosaic_dropout_backward(x, x, 0.1, 1, **bad)


def test_the_ends_of_the_range_are_taken():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    for good in (dict(site=0), dict(site=2 ** 31 - 2), dict(first_row=2 ** 63 - 8)):
        with pytest.raises(ValueError, match="device memory"):
            b.mosaic_dropout_forward(x, None, x, 0.1, 1, **good)
