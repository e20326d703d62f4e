"""The gated feed-forward block and its gradients against plain 64-bit statements of the same."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACT = {"silu": b.ACT_SILU, "gelu": b.ACT_GELU_TANH}


def generator(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def matrix(T, d, gen, pad=0, scale=1.0, dtype=torch.bfloat16):
    full = torch.full((T, d + pad), 777.0, dtype=dtype, device=DEV)
    full[:, :d] = (torch.randn((T, d), generator=gen) * scale).to(dtype).to(DEV)
    return full[:, :d], full


def inputs(T, d, F, seed, pad=0, packed=False):
    gen = generator(seed)
    x, _ = matrix(T, d, gen, pad)
    if packed:
        w, _ = matrix(2 * F, d, gen, pad, d ** -0.5)
        return gen, x, w[:F], w[F:]
    return gen, x, matrix(F, d, gen, pad, d ** -0.5)[0], matrix(F, d, gen, pad, d ** -0.5)[0]


SIZES = [  # rows, d, F: one row; rows around the tiles; K shorter than, equal to and past whole steps; ragged features
    (1, 8, 8), (1, 512, 2048), (1, 1032, 264), (2, 64, 128), (15, 72, 136), (16, 128, 16), (17, 520, 120), (33, 256, 256),
    (48, 1000, 520), (63, 64, 1024), (64, 192, 384), (65, 200, 392), (127, 128, 128), (129, 136, 248), (200, 320, 640),
    (255, 64, 64), (256, 256, 256), (257, 1032, 776), (300, 8, 2056), (513, 704, 1288), (1000, 512, 512),
]


@pytest.mark.parametrize("T,d,F", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_forward(T, d, F, act):
    pad = (0, 8, 64)[(T + d) % 3]
    gen, x, wg, wu = inputs(T, d, F, T + 3 * d + 5 * F, pad, packed=T % 2 == 1)
    out, full = matrix(T, F, gen, pad=8)
    b.mosaic_gated_ffn_forward(x, wg, wu, out, activation=ACT[act])
    exact, bound = ref.ffn_bound(x.cpu(), wg.cpu(), wu.cpu(), act)
    assert ((out.cpu().double() - exact).abs() <= bound).all()
    assert (full[:, F:] == 777.0).all()


@pytest.mark.parametrize("T,d,F", SIZES)
@pytest.mark.parametrize("kept", ["bf16", "int8", "e4m3"])
def test_gradients(T, d, F, kept):
    act = "gelu" if (T + F) % 16 else "silu"
    pad = (0, 8, 64)[(T + d) % 3]
    gen, x, wg, wu = inputs(T, d, F, T + 3 * d + 5 * F, pad, packed=T % 2 == 1)
    dout, _ = matrix(T, F, gen, pad, 0.01)
    source, x_exact = x, x.cpu()
    if kept != "bf16":
        source = b.Q8Rows.empty(T, d, torch.int8 if kept == "int8" else torch.float8_e4m3fn, 32, DEV)
        b.mosaic_checkpoint_store(x, source)
        x_exact = ref.restored(source.values.cpu(), source.scales.cpu(), 32)
    dx, dx_full = matrix(T, d, gen, 8)
    out, out_full = matrix(T, F, gen, 8)
    dw, dw_full = matrix(2 * F, d, gen, 8)
    need = b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, kept != "bf16")
    work = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_backward(dout, source, wg, wu, dx, dw[:F], dw[F:], work[:need], activation=ACT[act], out=out)
    exact, bound = ref.ffn_bound(x_exact, wg.cpu(), wu.cpu(), act)
    assert ((out.cpu().double() - exact).abs() <= bound).all()
    want = ref.ffn_gradients(dout.cpu(), x_exact, wg.cpu(), wu.cpu(), act)
    # Elementwise: the terms are rounded to bf16 once (with what their 32-bit factors are off, 1.02 of that), the result
    # again; their sum in 32 bits over K terms.
    g, u = x_exact.double() @ wg.cpu().double().t(), x_exact.double() @ wu.cpu().double().t()
    gg = g.clone().requires_grad_(True)
    ref.activation(gg, act).backward(torch.ones_like(g))
    do = dout.cpu().double()
    dg, du = do * u * gg.grad, do * ref.activation(g, act)
    off = 2 * d * ref.U_F32 * (x_exact.double().abs() @ (wg.cpu().double().abs() + wu.cpu().double().abs()).t())
    # second derivatives of both activations are below 1.13, so a projection's error moves a term by at most this
    slack = do.abs() * 1.13 * (u.abs() + off) * (off + 2.0 ** -20 * (1 + g.abs())) + do.abs() * 1.13 * (off + 2.0 ** -20 * g.abs())
    tg, tu = 1.02 * ref.U_BF16 * dg.abs() + slack, 1.02 * ref.U_BF16 * du.abs() + slack
    sums = lambda k: 2 * k * ref.U_F32   # noqa: E731
    bound = tg @ wg.cpu().double().abs() + tu @ wu.cpu().double().abs()
    bound += sums(2 * F) * (dg.abs() @ wg.cpu().double().abs() + du.abs() @ wu.cpu().double().abs())
    assert ((dx.cpu().double() - want[0]).abs() <= (1 + ref.U_BF16) * bound + ref.U_BF16 * want[0].abs() + 1e-38).all()
    for got, w_, t, terms in ((dw[:F], want[1], tg, dg), (dw[F:], want[2], tu, du)):
        bound = t.t() @ x_exact.double().abs() + sums(T) * (terms.abs().t() @ x_exact.double().abs())
        assert ((got.cpu().double() - w_).abs() <= (1 + ref.U_BF16) * bound + ref.U_BF16 * w_.abs() + 1e-38).all()
    # In the 2-norm two independent roundings of at most 2^-8 / sqrt 3 each; few terms may line up, so only where there are many.
    if min(T, d, F) >= 48:
        for got, w_ in ((dx, want[0]), (dw[:F], want[1]), (dw[F:], want[2])):
            assert ref.relative(got, w_) <= ref.U_BF16
    assert (dx_full[:, d:] == 777.0).all() and (out_full[:, F:] == 777.0).all() and (dw_full[:, d:] == 777.0).all()
    assert (work[need:] == 0xAB).all()
    # the same bits on a second call, and each result alone
    dx2 = torch.empty_like(dx)
    b.mosaic_gated_ffn_backward(dout, source, wg, wu, dx2, None, None, work[:need], activation=ACT[act])
    assert torch.equal(dx2, dx)
    dw2 = torch.empty((2 * F, d), dtype=torch.bfloat16, device=DEV)
    b.mosaic_gated_ffn_backward(dout, source, wg, wu, None, dw2[:F], dw2[F:], work[:need], activation=ACT[act])
    assert torch.equal(dw2, dw)


@pytest.mark.parametrize("T,d,F", [(4100, 4104, 4104), (8201, 4104, 2056), (700, 2200, 5000), (9000, 264, 1032), (1100, 5000, 1096)])
def test_more_tiles_than_blocks(T, d, F):
    """Sizes of several tiles a block, ragged in every direction; the plain statement in 64 bits on the device, with the bounds
    of the sizes above."""
    gen, x, wg, wu = inputs(T, d, F, T + 3 * d + 5 * F, 8)
    dout, _ = matrix(T, F, gen, 8, 0.01)
    out, out_full = matrix(T, F, gen, 8)
    dx, dx_full = matrix(T, d, gen, 8)
    dw, dw_full = matrix(2 * F, d, gen, 8)
    work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_forward(x, wg, wu, out)
    b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dw[:F], dw[F:], work)
    exact, bound = ref.ffn_bound(x, wg, wu, "silu")
    assert ((out.double() - exact).abs() <= bound).all()
    del exact, bound
    want = ref.ffn_gradients(dout, x, wg, wu, "silu")
    for got, w in zip((dx, dw[:F], dw[F:]), want):
        assert ref.relative(got, w) <= ref.U_BF16
        # The elements are sums of many terms of the same spread, each rounded to bf16: an element's error has about 2^-8 / sqrt 3
        # of the elements' root mean square as its spread; sixteen of those, and the result's own rounding.
        rms = w.square().mean().sqrt()
        assert ((got.double() - w).abs() <= 16 * ref.U_BF16 / 3 ** 0.5 * rms + ref.U_BF16 * w.abs()).all()
    assert (out_full[:, F:] == 777.0).all() and (dx_full[:, d:] == 777.0).all() and (dw_full[:, d:] == 777.0).all()


@pytest.mark.parametrize("T,d,F", [(40, 264, 18952), (64, 1032, 12296), (20, 136, 24584), (9, 520, 20008), (3, 200, 30008), (100, 72, 5000), (23, 2056, 5704)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_few_rows_of_wide_blocks(T, d, F, act):
    """Few rows of many features, K ragged: every way that takes them, forward and again in the backward pass."""
    gen, x, wg, wu = inputs(T, d, F, T + 3 * d + 5 * F, 8, packed=T % 2 == 1)
    dout, _ = matrix(T, F, gen, 8, 0.01)
    out, out_full = matrix(T, F, gen, 8)
    again, again_full = matrix(T, F, gen, 8)
    dx, dw = torch.empty_like(x), torch.empty((2 * F, d), dtype=torch.bfloat16, device=DEV)
    work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_forward(x, wg, wu, out, activation=ACT[act])
    b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dw[:F], dw[F:], work, activation=ACT[act], out=again)
    exact, bound = ref.ffn_bound(x, wg, wu, act)
    assert ((out.double() - exact).abs() <= bound).all() and ((again.double() - exact).abs() <= bound).all()
    for got, w in zip((dx, dw[:F], dw[F:]), ref.ffn_gradients(dout, x, wg, wu, act)):
        # a result's rounding, 2^-8 / sqrt 3, and its terms', as much again, where there are few of them not averaged
        assert ref.relative(got, w) <= 2 * ref.U_BF16
    assert (out_full[:, F:] == 777.0).all() and (again_full[:, F:] == 777.0).all()
    first = out.clone()
    b.mosaic_gated_ffn_forward(x, wg, wu, out, activation=ACT[act])
    assert torch.equal(out, first)


@pytest.mark.parametrize("T,d,F,act", [(290, 200, 12200, "silu"), (300, 1032, 12280, "gelu"), (1000, 72, 12280, "silu"),
                                       (120, 328, 18952, "gelu"), (200, 136, 18936, "silu"), (2040, 520, 5632, "gelu")])
def test_rows_by_features_between_the_tiles(T, d, F, act):
    """Numbers of features that neither 64 nor 128 a tile divide well among the compute units; see test_few_rows_of_wide_blocks."""
    test_few_rows_of_wide_blocks(T, d, F, act)


@pytest.mark.parametrize("T,d,F", [(1, 64, 64), (90, 136, 264), (700, 512, 384)])
def test_weight_gradients_in_parts(T, d, F):
    """32-bit weight gradients, a batch taken in parts: the parts add up to what the whole gives."""
    gen, x, wg, wu = inputs(T, d, F, 77 + T)
    dout, _ = matrix(T, F, gen, 0, 0.01)
    dx = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    whole = torch.full((2 * F, d), 5.0, device=DEV)
    work = torch.empty(max(16, b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F)), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, whole[:F], whole[F:], work)
    want = ref.ffn_gradients(dout.cpu(), x.cpu(), wg.cpu(), wu.cpu(), "silu")
    if T >= 90:   # one rounding to bf16 of every term
        assert ref.relative(whole[:F], want[1]) <= 0.6 * ref.U_BF16 and ref.relative(whole[F:], want[2]) <= 0.6 * ref.U_BF16
    start = torch.randn((2 * F, d), generator=gen).to(DEV) * 0.01
    parts = start.clone()
    cut = T // 3
    for lo, hi in ((0, cut), (cut, T)):
        b.mosaic_gated_ffn_backward(dout[lo:hi], x[lo:hi], wg, wu, None, parts[:F], parts[F:], work, accumulate=True)
    size = dout.cpu().double().abs().max() * 8 * T
    assert ((parts - start - whole).abs().cpu().double() <= 4 * (T + 4) * ref.U_F32 * size).all()


def test_gradients_against_differences():
    """Along their own direction the gradients are what central differences of the 64-bit block give."""
    T, d, F = 40, 128, 192
    for act in ("silu", "gelu"):
        gen, x, wg, wu = inputs(T, d, F, 9)
        dout, _ = matrix(T, F, gen)
        dx = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
        dwg, dwu = (torch.empty((F, d), device=DEV) for _ in range(2))
        work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
        b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dwg, dwu, work, activation=ACT[act])
        at = [t.cpu().double() for t in (x, wg, wu)]
        for k, grad in enumerate((dx, dwg, dwu)):
            v = grad.cpu().double()
            size = v.norm()
            v = v / size
            e = 1e-4
            ends = []
            for sign in (1, -1):
                moved = list(at)
                moved[k] = at[k] + sign * e * v
                ends.append((ref.ffn(*moved, act) * dout.cpu().double()).sum())
            slope = ((ends[0] - ends[1]) / (2 * e)).item()
            assert abs(slope - size.item()) <= ref.U_BF16 * abs(slope)


@pytest.mark.parametrize("T", [3, 100])
def test_large_and_non_finite_values(T):
    """Saturated activations are exact zeros and identities; a NaN or infinity reaches its own row alone."""
    d, F = 64, 128
    gen, x, wg, wu = inputs(T, d, F, 4)
    x[0] = 0
    x[0, 0] = 300.0
    wg[:, 0] = torch.tensor([1.0, -1.0], device=DEV).repeat(F // 2).to(torch.bfloat16)
    wu[:, 0] = 1.0
    clean = x.clone()
    x[1, 5] = float("nan")
    x[2, 5] = float("inf")
    for act in ("silu", "gelu"):
        out, ref_out = (torch.empty((T, F), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        b.mosaic_gated_ffn_forward(x, wg, wu, out, activation=ACT[act])
        b.mosaic_gated_ffn_forward(clean, wg, wu, ref_out, activation=ACT[act])
        assert (out[0, 0::2].float() == 90112.0).all()                # 300 * 300, to bf16
        assert (out[0, 1::2].float().abs() < 1e-30).all()
        assert out[1].isnan().all() and not out[2].isfinite().any()
        assert torch.equal(out[3:], ref_out[3:])
        dout = torch.ones((T, F), dtype=torch.bfloat16, device=DEV)
        dx = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
        work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
        b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, None, None, work, activation=ACT[act])
        assert dx[1].isnan().all() and dx[0].isfinite().all() and dx[3:].isfinite().all()


def test_offsets_past_32_bits():
    """Rows that lie further apart than 32-bit byte offsets reach: a wide row stride, first and last rows checked."""
    T, d, F = 2100, 64, 128
    stride = 1 << 20                                                           # 2 MiB a row, 4.1 GiB in all
    gen = generator(8)
    room = torch.zeros((T, stride), dtype=torch.bfloat16, device=DEV)
    x = room[:, :d]
    x.copy_(torch.randn((T, d), generator=gen).to(DEV))
    out = room[:, 4096:4096 + F]
    _, _, wg, wu = inputs(1, d, F, 12)
    b.mosaic_gated_ffn_forward(x, wg, wu, out)
    exact, bound = ref.ffn_bound(x.cpu(), wg.cpu(), wu.cpu(), "silu")
    assert ((out.cpu().double() - exact).abs() <= bound).all()
    dout, dx = room[:, 8192:8192 + F], room[:, 16384:16384 + d]
    dout.copy_(torch.randn((T, F), generator=gen).to(DEV))
    dw = torch.empty((2 * F, d), device=DEV)
    work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dw[:F], dw[F:], work)
    want = ref.ffn_gradients(dout.cpu(), x.cpu(), wg.cpu(), wu.cpu(), "silu")
    for got, w_ in zip((dx, dw[:F], dw[F:]), want):
        assert ref.relative(got, w_) <= ref.U_BF16


def test_no_rows():
    d, F = 64, 128
    _, _, wg, wu = inputs(1, d, F, 3)
    x, out = torch.empty((0, d), dtype=torch.bfloat16, device=DEV), torch.empty((0, F), dtype=torch.bfloat16, device=DEV)
    b.mosaic_gated_ffn_forward(x, wg, wu, out)
    dw = torch.full((2 * F, d), 3.0, device=DEV)
    b.mosaic_gated_ffn_backward(out, x, wg, wu, x, dw[:F], dw[F:], None, accumulate=True)
    assert (dw == 3.0).all()
    b.mosaic_gated_ffn_backward(out, x, wg, wu, x, dw[:F], dw[F:], None)
    assert (dw == 0.0).all()


def test_another_stream_and_a_graph():
    T, d, F = 77, 256, 512
    gen, x, wg, wu = inputs(T, d, F, 19)
    dout, _ = matrix(T, F, gen)
    out, again = (torch.empty((T, F), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dx, dx2 = (torch.empty((T, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dw, dw2 = (torch.empty((2 * F, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_forward(x, wg, wu, out)
    b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx, dw[:F], dw[F:], work)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b.mosaic_gated_ffn_forward(x, wg, wu, again, stream=side)
    side.synchronize()
    assert torch.equal(out, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.mosaic_gated_ffn_forward(x, wg, wu, again)
        b.mosaic_gated_ffn_backward(dout, x, wg, wu, dx2, dw2[:F], dw2[F:], work)
    for _ in range(3):
        for t in (again, dx2, dw2):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
