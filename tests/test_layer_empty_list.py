"""A list of rows without entries: it lists no rows, and never stands for all of them."""
import pytest
import torch

from paper_2601_06562_amd import binding as b

NONE = torch.zeros(0, dtype=torch.int32)


def test_half_a_list_is_refused():
    """An empty tensor has no address, and without either address the library takes all rows."""
    x, gamma = torch.zeros((4, 64), dtype=torch.bfloat16), torch.ones(64)
    for idx, count in ((NONE, None), (None, NONE)):
        with pytest.raises(ValueError, match="go together"):
            b.mosaic_rmsnorm_forward(x, None, gamma, 1e-5, x, idx=idx, count=count)
    with pytest.raises(ValueError, match="count must hold"):
        b.mosaic_rmsnorm_forward(x, None, gamma, 1e-5, x, idx=NONE, count=NONE)


@pytest.mark.gpu
def test_no_entries():
    dev = "cuda:0"
    x = torch.ones((4, 64), dtype=torch.bfloat16, device=dev)
    y, gamma = torch.full_like(x, -5.0), torch.ones(64, device=dev)
    for n in (0, 3):                                                           # whatever the count says
        b.mosaic_rmsnorm_forward(x, None, gamma, 1e-5, y, idx=NONE.to(dev),
                                 count=torch.tensor([n], dtype=torch.int32, device=dev))
    assert (y == -5.0).all()
