"""A workspace query answers for exactly the sizes that its call takes: 0 for those it refuses, never 0 for the others."""
import itertools

from paper_2601_06562_amd import binding as b
from test_layer_host_api import SHAPE, SMALL, ffn_backward, norm_backward, q8

SIZES = (8, 16384, 16392, 1 << 17, (1 << 17) + 8)


def test_the_block():
    for d, F in itertools.product(SIZES, SIZES):
        wide = dict(d=d, F=F, ld_x=1 << 20, ld_w=1 << 20, ld_dx=1 << 20, ld_dw=1 << 20, ld_dout=1 << 20, ld_out=1 << 20, bytes=0)
        rows = q8(ld_values=1 << 20, ld_scales=1 << 13)
        for eight in (False, True):
            need = b.mosaic_gated_ffn_backward_workspace_bytes(4, d, F, eight)
            status = ffn_backward(x=0, q8=rows, **wide) if eight else ffn_backward(**wide)
            assert (need, status) == (0, SHAPE) or (need > 0 and status == SMALL), (d, F, eight)


def test_the_norm():
    for d in SIZES:
        need = b.mosaic_rmsnorm_backward_workspace_bytes(4, d)
        status = norm_backward(d=d, ld_dy=1 << 20, ld_h=1 << 20, ld_in=1 << 20, ld_dsum=1 << 20, bytes=0)
        assert (need, status) == (0, SHAPE) or (need > 0 and status == SMALL), d
