"""Lists of nearly 2^31 rows: the kernels number rows in 32 bits and in whole tiles of up to 256, so the last tile has to end below
2^31.  Bounds past that are refused (workspaces of no bytes: nothing is enqueued)."""
import pytest

from paper_2601_06562_amd import binding as b
from test_tokens_host_api import SHAPE, SMALL, logprobs, logprobs_backward

MOST = (1 << 31) - 256


@pytest.mark.parametrize("d,V", [(64, 256), (8, 5), (512, 32000)])
@pytest.mark.parametrize("rows,taken", [(MOST - 1, True), (MOST, True), (MOST + 1, False), (MOST + 193, False), ((1 << 31) - 1, False)])
def test_the_longest_list(rows, taken, d, V):
    wide = dict(T=9, d=d, V=V, max_rows=rows, ld_h=d, ld_w=d, bytes=0)
    assert logprobs(**wide) == (SMALL if taken else SHAPE)
    assert logprobs_backward(ld_dx=d, ld_dw=d, **wide) == (SMALL if taken else SHAPE)
    assert logprobs(**dict(wide, T=rows, idx=0, count=0)) == (SMALL if taken else SHAPE)
    assert (b.mosaic_masked_logprobs_workspace_bytes(9, rows, d, V, 2) > 0) is taken
    assert (b.mosaic_masked_logprobs_backward_workspace_bytes(rows, d, V, 1) > 0) is taken
