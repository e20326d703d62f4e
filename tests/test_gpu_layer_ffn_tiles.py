"""The feed-forward block and its gradients at sizes that take every tile of every product, one tile a block and several, ragged
in every direction; test_ffn_choice_host.py holds the list to that.  Plain statements in 64 bits, on the device."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_layer_ffn import ACT, DEV, inputs, matrix

pytestmark = pytest.mark.gpu

SIZES = [  # rows, d, F
    (1, 72, 136), (1, 72, 25432), (16839, 72, 136), (17, 3600, 4128), (473, 528, 3192), (258, 1184, 7944), (1255, 6624, 264),
    (261, 288, 10952), (3124, 72, 1248), (13, 1256, 19592), (16570, 144, 304), (215, 1608, 2456), (36, 1176, 3208),
    (9248, 1760, 408), (262, 72, 17864), (257, 72, 21920), (16671, 72, 400), (414, 72, 18888), (415, 72, 24712),
    (550, 7136, 280), (49, 72, 144), (1599, 4952, 136), (17063, 792, 136), (133, 5384, 3216), (8467, 2856, 136),
    (1, 5024, 1632),
    # several tiles a block and a K of many steps, which ends inside one: projections; dw; dx
    (8190, 200, 2040), (4730, 1032, 6984), (8200, 1032, 8200), (8200, 2056, 1032),
]


def gradient_bounds(dout, x, wg, wu, act, rows=None):
    """dx, dw_gate and dw_up, each with an elementwise bound on its error before its own rounding.  A term is rounded to bf16 once (1.02 of that, with what its 32-bit factors are off); both activations' second
    derivatives are below 1.13, so a projection's error of `off` moves a term by at most the slack; a sum of K terms in 32
    bits is off by 2 K units of the sum of their magnitudes.  `rows`: of the whole batch, where these are a part of it."""
    do, x, wg, wu = (t.double() for t in (dout, x, wg, wu))
    T, F = do.shape
    d = x.shape[1]
    g, u = x @ wg.t(), x @ wu.t()
    gg = g.clone().requires_grad_(True)
    a = ref.activation(gg, act)
    a.backward(torch.ones_like(g))
    dg, du = do * u * gg.grad, do * a.detach()
    off = 2 * d * ref.U_F32 * (x.abs() @ (wg.abs() + wu.abs()).t())
    slack = do.abs() * 1.13 * (u.abs() + off) * (off + 2.0 ** -20 * (1 + g.abs())) + do.abs() * 1.13 * (off + 2.0 ** -20 * g.abs())
    tg, tu = 1.02 * ref.U_BF16 * dg.abs() + slack, 1.02 * ref.U_BF16 * du.abs() + slack
    off_x = tg @ wg.abs() + tu @ wu.abs() + 4 * F * ref.U_F32 * (dg.abs() @ wg.abs() + du.abs() @ wu.abs())
    yield dg @ wg + du @ wu, off_x
    for t, terms in ((tg, dg), (tu, du)):
        yield terms.t() @ x, t.t() @ x.abs() + 2 * (rows or T) * ref.U_F32 * (terms.abs().t() @ x.abs())


def blank(T, d):
    full = torch.full((T, d + 8), 777.0, dtype=torch.bfloat16, device=DEV)
    return full[:, :d], full


def rounded(bound, want):
    """With one rounding of the result to bf16."""
    return (1 + ref.U_BF16) * bound + ref.U_BF16 * want.abs() + 1e-38


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,d,F", SIZES)
def test_every_tile(T, d, F, act):
    print(f"T {T} d {d} F {F} {act}", flush=True)
    gen, x, wg, wu = inputs(T, d, F, T + 3 * d + 5 * F, 8, packed=True)
    dout, _ = matrix(T, F, gen, 8, 0.01)
    (out, out_full), (again, again_full) = blank(T, F), blank(T, F)
    (dx, dx_full), (dw, dw_full) = blank(T, d), blank(2 * F, d)
    (dx_alone, dxa_full), (dw_alone, dwa_full) = blank(T, d), blank(2 * F, d)
    sums, sums_full = matrix(2 * F, d, gen, 8, 0.01, torch.float32)
    start = sums.clone()
    need = b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F)
    work = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)

    def backward(dx, dw, **more):
        parts = (None, None) if dw is None else (dw[:F], dw[F:])
        b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, *parts, work[:need], activation=ACT[act], **more)

    b.mosaic_gated_ffn_forward(x, wg, wu, out, activation=ACT[act])
    backward(dx, dw, out=again)
    backward(dx_alone, None)
    backward(None, dw_alone)
    backward(None, sums, accumulate=True)
    exact, bound = ref.ffn_bound(x, wg, wu, act)
    assert ((out.double() - exact).abs() <= bound).all() and ((again.double() - exact).abs() <= bound).all()
    del exact, bound
    (want_x, off_x), *weights = gradient_bounds(dout, x, wg, wu, act)
    assert ((dx.double() - want_x).abs() <= rounded(off_x, want_x)).all()
    for i, (want, off) in enumerate(weights):
        at = slice(i * F, (i + 1) * F)
        assert ((dw[at].double() - want).abs() <= rounded(off, want)).all()
        total = start[at].double() + want                                       # added in 32 bits, one rounding more
        assert ((sums[at].double() - total).abs() <= off + ref.U_F32 * (total.abs() + off)).all()
    # each gradient alone has the bits that it has beside the other
    assert torch.equal(dx_alone, dx) and torch.equal(dw_alone, dw)
    for full, cols in ((out_full, F), (again_full, F), (dx_full, d), (dxa_full, d), (dw_full, d), (dwa_full, d), (sums_full, d)):
        assert (full[:, cols:] == 777.0).all()
    assert (work[need:] == 0xAB).all()
