"""`accumulate` speaks of the weights' gradients alone: a call that asks for none takes it either way."""
from paper_2601_06562_amd import binding as b
from test_layer_host_api import INVALID, OK, SMALL, ffn_backward, norm_backward


def test_without_weight_gradients():
    for dw_type in (b.BF16, b.F32):
        for accumulate in (0, 1):
            assert ffn_backward(dwg=0, dwu=0, dw_type=dw_type, accumulate=accumulate, bytes=0) == SMALL   # the last check
            assert ffn_backward(T=0, dwg=0, dwu=0, dw_type=dw_type, accumulate=accumulate, ws=0) == OK
    assert ffn_backward(dx=0, dwg=0, dwu=0, out=0, accumulate=1) == INVALID


def test_with_them():
    assert ffn_backward(dw_type=b.BF16, accumulate=1) == INVALID and ffn_backward(dw_type=b.F32, accumulate=1, bytes=0) == SMALL


def test_the_norm():
    assert norm_backward(T=0, dgamma=0, dy=0, h=0, accumulate=1) == OK
