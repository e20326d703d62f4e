"""Dropout from a counter-based generator, whose mask is never stored, against a plain statement of the same."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
SEED = 0xFEDCBA9876543210


def matrix(T, d, dtype, seed, pad=0):
    full = torch.full((T, d + pad), 777.0, dtype=dtype, device=DEV)
    full[:, :d] = torch.randn((T, d), generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)
    return full[:, :d], full


SIZES = [(1, 8), (1, 4096), (3, 24), (37, 3584), (255, 512), (5, 2056), (1237, 1024), (9000, 1000), (2, 16384)]


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("stream_type", [BF16, F32])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5])
def test_forward(T, d, stream_type, p):
    """A product in 32 bits with a factor rounded to 32, a sum, and one rounding."""
    x, _ = matrix(T, d, BF16, 1, pad=8)
    r, _ = matrix(T, d, stream_type, 2, pad=16)
    mask, grow = ref.kept(T, d, p, SEED, site=5, first_row=77)
    for residual in (r, None):
        out, full = matrix(T, d, stream_type, 3, pad=24)
        b.mosaic_dropout_forward(x, residual, out, p, SEED, site=5, first_row=77)
        torch.cuda.synchronize()
        part = torch.where(mask, x.cpu().double() * grow, 0.0)
        want = part + (residual.cpu().double() if residual is not None else 0.0)
        before = 3 * ref.U[F32] * (part.abs() + want.abs())
        assert ((out.cpu().double() - want).abs() <= before + ref.U[stream_type] * (want.abs() + before)).all()
        assert bool((full[:, d:] == 777.0).all())
        if residual is None:
            assert torch.equal(out.cpu() != 0, mask & (x.cpu() != 0))


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("stream_type", [BF16, F32])
def test_backward_makes_the_same_mask(T, d, stream_type):
    g, _ = matrix(T, d, stream_type, 4, pad=8)
    dx, full = matrix(T, d, BF16, 5, pad=8)
    mask, grow = ref.kept(T, d, 0.3, SEED, site=0, first_row=1 << 33)
    b.mosaic_dropout_backward(g, dx, 0.3, SEED, first_row=1 << 33)
    torch.cuda.synchronize()
    want = torch.where(mask, g.cpu().double() * grow, 0.0)
    assert ((dx.cpu().double() - want).abs() <= (ref.U[BF16] + 3 * ref.U[F32]) * want.abs()).all()
    assert torch.equal(dx.cpu() != 0, mask & (want.to(BF16) != 0)) and bool((full[:, d:] == 777.0).all())


def test_the_gradient_by_differences():
    """The forward pass is linear: a step in one direction changes it by the backward pass's transpose."""
    T, d = 65, 520
    x, _ = matrix(T, d, BF16, 6)
    v = torch.ones((T, d), dtype=BF16, device=DEV)
    g, _ = matrix(T, d, F32, 7)
    y0, y1 = torch.empty((T, d), device=DEV), torch.empty((T, d), device=DEV)
    dx = torch.empty((T, d), dtype=BF16, device=DEV)
    half = (x.float() * 0.5).to(BF16)
    b.mosaic_dropout_forward(half, None, y0, 0.25, 3)
    b.mosaic_dropout_forward(v, None, y1, 0.25, 3)
    b.mosaic_dropout_backward(g, dx, 0.25, 3)
    for y, at in ((y0, half), (y1, v)):
        left, right = (y.double() * g.double()).sum(), (at.double() * dx.double()).sum()
        size = (y.double() * g.double()).abs().sum()
        assert abs((left - right).item()) <= (ref.U[BF16] + 4 * ref.U[F32]) * size.item()


def test_parts_make_the_whole():
    T, d = 300, 1024
    x, _ = matrix(T, d, BF16, 8)
    whole, parts = torch.empty((T, d), dtype=BF16, device=DEV), torch.empty((T, d), dtype=BF16, device=DEV)
    b.mosaic_dropout_forward(x, None, whole, 0.2, SEED, site=9, first_row=5)
    for lo, hi in ((0, 1), (1, 130), (130, 300)):
        b.mosaic_dropout_forward(x[lo:hi], None, parts[lo:hi], 0.2, SEED, site=9, first_row=5 + lo)
    assert torch.equal(whole, parts)
    b.mosaic_dropout_forward(x, None, parts, 0.2, SEED, site=8, first_row=5)
    assert not torch.equal(whole, parts)


def test_in_place():
    T, d = 130, 264
    for kind in (BF16, F32):
        x, _ = matrix(T, d, BF16, 9)
        r, _ = matrix(T, d, kind, 10)
        out = torch.empty_like(r)
        b.mosaic_dropout_forward(x, r, out, 0.4, 1)
        b.mosaic_dropout_forward(x, r, r, 0.4, 1)
        assert torch.equal(r, out)
    x, _ = matrix(T, d, BF16, 9)
    out = torch.empty_like(x)
    b.mosaic_dropout_forward(x, None, out, 0.4, 1)
    b.mosaic_dropout_backward(x, x, 0.4, 1)          # the same operation
    assert torch.equal(x, out)


def test_a_dropped_element_is_zero_whatever_it_was():
    T, d = 64, 512
    x = torch.full((T, d), float("nan"), dtype=BF16, device=DEV)
    x[:, ::2] = float("inf")
    out = torch.empty((T, d), device=DEV)
    b.mosaic_dropout_forward(x, None, out, 0.5, 77)
    mask, _ = ref.kept(T, d, 0.5, 77)
    assert torch.equal(out.cpu() == 0, ~mask) and bool((out.cpu().isnan() | out.cpu().isinf())[mask].all())


def test_the_border_of_p():
    """Nearly all dropped: what is kept grows by 2^16."""
    x = torch.ones((2000, 4096), dtype=BF16, device=DEV)
    out = torch.empty((2000, 4096), device=DEV)
    b.mosaic_dropout_forward(x, None, out, 1 - 2.0 ** -16, 5)
    kept = out[out != 0]
    assert bool((kept == 65536.0).all()) and 60 < kept.numel() < 200      # 125 expected
    b.mosaic_dropout_forward(x, None, out, 2.0 ** -18, 5)                 # rounds to none
    assert bool((out == 1).all())


def test_replayed_from_a_graph():
    x, _ = matrix(700, 512, BF16, 12)
    r, _ = matrix(700, 512, F32, 13)
    out = torch.empty_like(r)
    b.mosaic_dropout_forward(x, r, out, 0.1, 99)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.mosaic_dropout_forward(x, r, out, 0.1, 99)
    for _ in range(3):
        x.normal_()
        r.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        b.mosaic_dropout_forward(x, r, out, 0.1, 99)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
