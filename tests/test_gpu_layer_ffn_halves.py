"""Gradients of the feed-forward block for few rows: dg and du are carried in two numbers an element up to 32 rows, so that the
gradients are as exact as their own rounding, where the rounding of a few large terms would show."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_layer_ffn import ACT, DEV, inputs, matrix
from test_gpu_layer_ffn_tiles import blank, gradient_bounds, rounded

pytestmark = pytest.mark.gpu
ROWS = [1, 2, 3, 7, 8, 15, 16, 17, 31, 32]
# Of a term's rounding remains 2^-8 of 2^-8; gradient_bounds has 1.02 of 2^-8 for it.
LEFT = 2.0 ** -8


def exact_bounds(dout, x, wg, wu, act):
    """As gradient_bounds, for terms of twice the bits: its bound for a rounding is taken down to what remains of one, by the
    magnitudes of the terms."""
    whole = list(gradient_bounds(dout, x, wg, wu, act))
    do, xd, g, u = dout.double(), x.double(), x.double() @ wg.double().t(), x.double() @ wu.double().t()
    gg = g.clone().requires_grad_(True)
    a = ref.activation(gg, act)
    a.backward(torch.ones_like(g))
    dg, du = (do * u * gg.grad).abs(), (do * a.detach()).abs()
    sizes = [dg @ wg.double().abs() + du @ wu.double().abs(), dg.t() @ xd.abs(), du.t() @ xd.abs()]
    return [(want, off - (1 - LEFT) * 1.02 * ref.U_BF16 * size) for (want, off), size in zip(whole, sizes)]


@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("d,F,act,kept", [(72, 136, "silu", "bf16"), (512, 2048, "gelu", "bf16"), (520, 1288, "silu", "int8"),
                                          (1032, 2744, "silu", "e4m3"), (3600, 4128, "silu", "bf16"), (136, 16392, "gelu", "int8"),
                                          (8, 8, "silu", "bf16"), (2056, 72, "gelu", "bf16")])
def test_as_exact_as_their_rounding(T, d, F, act, kept):
    print(f"T {T} d {d} F {F} {act} {kept}", flush=True)
    gen, x_all, wg, wu = inputs(T + 40, d, F, T + 3 * d + 5 * F, 8)
    dout_all, _ = matrix(T + 40, F, gen, 8, 0.01)
    x_all[T:] = float("nan")                                                   # rows that are not the call's
    dout_all[T:] = float("nan")
    x, dout = x_all[:T], dout_all[:T]
    source, x_exact = x, x
    if kept != "bf16":
        source = b.Q8Rows.empty(T, d, torch.int8 if kept == "int8" else torch.float8_e4m3fn, 32, DEV)
        b.mosaic_checkpoint_store(x, source)
        x_exact = ref.restored(source.values, source.scales, 32)
    (dx, dx_full), (dx_alone, _) = blank(T, d), blank(T, d)
    (dw, dw_full), (dw_alone, _) = blank(2 * F, d), blank(2 * F, d)
    sums = torch.full((2 * F, d), 3.0, device=DEV)
    out, _ = blank(T, F)
    need = b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, kept != "bf16")
    work = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)       # NaN in every type
    work[need:] = 0xAB

    def backward(dx, dw, **more):
        parts = (None, None) if dw is None else (dw[:F], dw[F:])
        b.mosaic_gated_ffn_backward(dout, source, wg, wu, dx, *parts, work[:need], activation=ACT[act], **more)

    backward(dx, dw, out=out)
    backward(dx_alone, None)
    backward(None, dw_alone)
    backward(None, sums)
    (want_x, off_x), *weights = exact_bounds(dout, x_exact, wg, wu, act)
    assert ((dx.double() - want_x).abs() <= rounded(off_x, want_x)).all()
    for i, (want, off) in enumerate(weights):
        at = slice(i * F, (i + 1) * F)
        assert ((dw[at].double() - want).abs() <= rounded(off, want)).all()
        assert ((sums[at].double() - want).abs() <= off + ref.U_F32 * want.abs() + 1e-38).all()
    exact, bound = ref.ffn_bound(x_exact, wg, wu, act)
    assert ((out.double() - exact).abs() <= bound).all()
    assert torch.equal(dx_alone, dx) and torch.equal(dw_alone, dw)
    assert (dx_full[:, d:] == 777.0).all() and (dw_full[:, d:] == 777.0).all() and (work[need:] == 0xAB).all()


@pytest.mark.parametrize("T", [1, 5, 32, 33])
def test_infinite_gradients_stay_infinite(T):
    """An element whose gradient is infinite has no low half: the results are not NaN for it."""
    d, F = 64, 128
    gen, x, wg, wu = inputs(T, d, F, 5)
    x[0], wg[:], wu[:] = 0.0, 0.0, 0.0
    x[0, 0] = 1.0
    wg[0, 0], wu[0, 0] = 100.0, 1.0                                            # silu(100) = 100, slope 1
    dout = torch.zeros((T, F), dtype=torch.bfloat16, device=DEV)
    for value in (float("inf"), 3.3895313892515355e38):                        # du = 100 times either
        dout[0, 0] = value
        dx, dw = torch.empty((T, d), dtype=torch.bfloat16, device=DEV), torch.empty((2 * F, d), device=DEV)
        work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
        b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dw[:F], dw[F:], work)
        assert dx[0, 0].item() == float("inf") and dw[F, 0].item() == float("inf")


def test_a_workspace_for_more_rows_serves():
    """Sized for any number of rows it serves every smaller number, across the bound on few rows."""
    d, F = 136, 264
    for size in (32, 33, 40, 64, 100):
        gen, x, wg, wu = inputs(size, d, F, size)
        dout, _ = matrix(size, F, gen, 0, 0.01)
        need = b.mosaic_gated_ffn_backward_workspace_bytes(size, d, F)
        work = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        for T in sorted({1, 16, 31, 32, size}):
            dx, dw = torch.empty((T, d), dtype=torch.bfloat16, device=DEV), torch.empty((2 * F, d), device=DEV)
            b.mosaic_gated_ffn_backward(dout[:T], x[:T], wg, wu, dx, dw[:F], dw[F:], work[:need])
            for got, (want, off) in zip((dx, dw[:F], dw[F:]), gradient_bounds(dout[:T], x[:T], wg, wu, "silu")):
                assert ((got.double() - want).abs() <= rounded(off, want)).all()
        assert (work[need:] == 0xFF).all()
