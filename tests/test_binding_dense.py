"""Lists, counts, results and workspaces reach the library as an address and a length, so the binding refuses the views whose
elements do not lie side by side: the library would read, or write, other places than theirs."""
import pytest
import torch

from paper_2601_06562_amd import binding as b

INTS = torch.arange(16, dtype=torch.int32)
VIEWS = {"strided": INTS[::2], "column": INTS.view(4, 4)[:, 1], "expanded": INTS[:1].expand(8)}


@pytest.mark.parametrize("view", VIEWS)
def test_a_list_of_rows(view):
    x, gamma = torch.zeros((16, 64), dtype=torch.bfloat16), torch.ones(64)
    with pytest.raises(ValueError, match="idx must be contiguous"):
        b.mosaic_rmsnorm_forward(x, None, gamma, 1e-5, x, idx=VIEWS[view], count=INTS[:1])
    with pytest.raises(ValueError, match="count must be contiguous"):
        b._dev_ptr(VIEWS[view], "count", torch.int32)


@pytest.mark.parametrize("view", VIEWS)
def test_the_other_calls(view):
    v, one, mask = VIEWS[view], INTS[:1], torch.zeros(8, dtype=torch.uint8)
    with pytest.raises(ValueError, match="idx must be contiguous"):
        b.mosaic_shift_indices(v, one, 4, INTS[:2], INTS[:8].clone())
    with pytest.raises(ValueError, match="conf must be contiguous"):
        b.mosaic_unmask_topn(torch.zeros(16)[::2], INTS[:8], INTS[:8], one, 8, INTS[:2], one,
                             INTS[:8], mask)
    with pytest.raises(ValueError, match="workspace must be contiguous"):
        b._workspace_args(v)


def test_dense_views_and_one_element_pass():
    """They get as far as the check that comes next."""
    for t in (INTS, INTS[4:12], INTS[3:4], INTS[::16], INTS[:0], INTS[:1].expand(1)):
        with pytest.raises(ValueError, match="device memory"):
            b._dev_ptr(t, "idx", torch.int32)
    assert b._dev_ptr(None, "idx") == 0
