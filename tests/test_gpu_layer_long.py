"""The layer operators beyond one launch's rows, one round of blocks and 32-bit byte offsets: 131072 rows of the block, 2^20 blocks
of the norms and checkpoints, 4 GiB of a matrix.  Plain statements in 64 bits, on the device, in parts of the rows."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_layer_ffn_tiles import gradient_bounds, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
PART = 1 << 16


def device_generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def matrix(T, d, gen, dtype=torch.bfloat16, scale=1.0):
    out = torch.empty((T, d), dtype=dtype, device=DEV)
    for r in range(0, T, PART):
        n = min(T - r, PART)
        out[r:r + n] = torch.randn((n, d), generator=gen, device=DEV) * scale
    return out


def parts(T):
    return [slice(r, min(T, r + PART)) for r in range(0, T, PART)]


@pytest.mark.parametrize("d,F,kept", [(72, 136, "bf16"), (72, 136, "e4m3"), (72, 8200, "int8")])
def test_block_of_several_launches(d, F, kept):
    """dg | du of the widest lie further apart than 32-bit byte offsets reach."""
    T = 131072 + 70
    gen = device_generator(d + F)
    x, dout = matrix(T, d, gen), matrix(T, F, gen, scale=0.01)
    w = matrix(2 * F, d, gen, scale=d ** -0.5)
    wg, wu = w[:F], w[F:]
    source, x_exact = x, x
    if kept != "bf16":
        source = b.Q8Rows.empty(T, d, torch.int8 if kept == "int8" else torch.float8_e4m3fn, 32, DEV)
        b.mosaic_checkpoint_store(x, source)
        x_exact = ref.restored(source.values, source.scales, 32)
    out, again, dx = (torch.full((T, n), 777.0, dtype=torch.bfloat16, device=DEV) for n in (F, F, d))
    dw = torch.empty((2 * F, d), device=DEV)
    work = torch.empty(b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, kept != "bf16"), dtype=torch.uint8, device=DEV)
    b.mosaic_gated_ffn_forward(x, wg, wu, out)
    b.mosaic_gated_ffn_backward(dout, source, wg, wu, dx, dw[:F], dw[F:], work, out=again)
    want_w, off_w = (torch.zeros((2 * F, d), dtype=torch.float64, device=DEV) for _ in range(2))
    for at in parts(T):
        for got, rows in ((out, x), (again, x_exact)):
            exact, bound = ref.ffn_bound(rows[at], wg, wu, "silu")
            assert ((got[at].double() - exact).abs() <= bound).all()
        (want, off), *weights = gradient_bounds(dout[at], x_exact[at], wg, wu, "silu", rows=T)
        assert ((dx[at].double() - want).abs() <= rounded(off, want)).all()
        for i, (want, off) in enumerate(weights):
            want_w[i * F:(i + 1) * F] += want
            off_w[i * F:(i + 1) * F] += off
    assert ((dw.double() - want_w).abs() <= off_w + ref.U_F32 * want_w.abs()).all()
    # the elementwise bound of so many terms is wide; in the 2-norm each term's rounding is 2^-8 / sqrt 3 at most
    assert ref.relative(dw, want_w) <= 0.6 * ref.U_BF16


def check_norm(y, h, gamma):
    want = ref.norm(h, gamma, EPS)
    bound = (ref.U_BF16 + (h.shape[1] + 16) * ref.U_F32) * want.abs() + 1e-38
    assert ((y.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("T,d", [((1 << 20) + 300, 1032), ((1 << 22) + 77, 8)])
def test_norm_of_more_rows_than_a_round(T, d):
    """Blocks take a second row: both halves of what the waves of a row exchange in, and rows past 4 GiB."""
    gen = device_generator(d)
    x, r = matrix(T, d, gen), matrix(T, d, gen, torch.float32, 2.0)
    gamma = 1 + 0.2 * torch.randn(d, generator=gen, device=DEV)
    y, total = torch.empty_like(x), torch.empty_like(r)
    q8 = b.Q8Rows.empty(T, d, torch.int8, 128, DEV)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, sum=total, q8=q8)
    for at in parts(T):
        h = x[at].double() + r[at].double()
        assert ((total[at].double() - h).abs() <= 2 * ref.U_F32 * h.abs()).all()
        check_norm(y[at], h, gamma)
        want = ref.norm(h, gamma, EPS)
        scales = q8.scales[at].double().repeat_interleave(128, dim=1)[:, :d]
        assert ((q8.values[at].double() * scales - want).abs() <= 0.5 * scales + (d + 16) * ref.U_F32 * want.abs() + 1e-45).all()


@pytest.mark.parametrize("T,d", [((1 << 20) + 300, 1032), ((1 << 22) + 77, 8)])
def test_listed_rows_of_a_second_round(T, d):
    """Entries of the first round, of the second, and of both are skipped for the same block; the others are as they would be
    alone."""
    gen = device_generator(d + 1)
    x = matrix(T, d, gen)
    gamma = torch.ones(d, device=DEV)
    y = torch.full_like(x, -5.0)
    order = torch.randperm(T, generator=gen, device=DEV)
    idx = order.to(torch.int32)
    skip = torch.zeros(T, dtype=torch.bool, device=DEV)
    skip[0:T:3] = True
    skip[T - 40:T - 20] = True
    idx[skip] = torch.where(torch.arange(int(skip.sum()), device=DEV) % 2 == 0, -7, T).to(torch.int32)
    b.mosaic_rmsnorm_forward(x, None, gamma, EPS, y, idx=idx, count=torch.tensor([T], dtype=torch.int32, device=DEV))
    listed = torch.zeros(T, dtype=torch.bool, device=DEV)
    listed[order[~skip]] = True
    for at in parts(T):
        rows = listed[at]
        check_norm(y[at][rows], x[at][rows].double(), gamma)
        assert (y[at][~rows] == -5.0).all()


def test_norm_gradient_past_32_bit_offsets():
    T, d = (1 << 20) + 300, 1032
    gen = device_generator(5)
    h, dy = matrix(T, d, gen, torch.float32, 2.0), matrix(T, d, gen, scale=0.01)
    gamma = 1 + 0.2 * torch.randn(d, generator=gen, device=DEV)
    dsum, dgamma = torch.empty_like(h), torch.empty(d, device=DEV)
    work = torch.empty(b.mosaic_rmsnorm_backward_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    b.mosaic_rmsnorm_backward(dy, h, gamma, EPS, dsum, dgamma, work)
    want_gamma, size_gamma = torch.zeros(d, dtype=torch.float64, device=DEV), torch.zeros(d, dtype=torch.float64, device=DEV)
    for at in parts(T):
        rows, g = h[at].double(), dy[at].double()
        rms = torch.sqrt(rows.square().mean(dim=1, keepdim=True) + EPS)
        n, c = rows / rms, g * gamma.double()
        along = (c * n).mean(dim=1, keepdim=True)
        want = (c - n * along) / rms
        size = (c.abs() + n.abs() * (c * n).abs().mean(dim=1, keepdim=True)) / rms
        assert ((dsum[at].double() - want).abs() <= ref.U_F32 * want.abs() + (d + 32) * ref.U_F32 * size + 1e-38).all()
        want_gamma += (g * n).sum(dim=0)
        size_gamma += (g * n).abs().sum(dim=0)
    # 512 partial sums of every 512th row; 64 strips of them, joined in a few steps more; a row's root as above
    depth = T / 512 + 512 / 64 + 32
    assert ((dgamma.double() - want_gamma).abs() <= (depth + d + 32) * ref.U_F32 * size_gamma).all()


@pytest.mark.parametrize("T,d", [((1 << 20) + 300, 1032), ((1 << 22) + 77, 8)])
def test_checkpoints_of_more_rows_than_a_round(T, d):
    gen = device_generator(d + 2)
    x = matrix(T, d, gen, torch.float32)
    q8 = b.Q8Rows.empty(T, d, torch.int8, 64, DEV)
    out = torch.full((T, d), 777.0, device=DEV)
    b.mosaic_checkpoint_store(x, q8)
    b.mosaic_checkpoint_load(q8, out)
    for at in parts(T):
        scales = q8.scales[at].double().repeat_interleave(64, dim=1)[:, :d]
        back = q8.values[at].double() * scales
        want = x[at].double()
        assert ((back - want).abs() <= 0.5 * scales + 4 * ref.U_F32 * want.abs()).all()
        assert torch.equal(out[at], ref.restored(q8.values[at], q8.scales[at], 64).float())


@pytest.mark.parametrize("T,d", [(1500, 4104), (1101, 8192), (1030, 8200), (1030, 12296), (1027, 16384)])
@pytest.mark.parametrize("kept", ["bf16", "f32", "int8", "e4m3"])
def test_norms_of_wide_rows(T, d, kept):
    """Rows of more than 4096 columns, several a block in the backward pass, where the next row is not asked for ahead."""
    gen = device_generator(T + d)
    stream = torch.float32 if kept == "f32" else torch.bfloat16
    x, r = matrix(T, d, gen), matrix(T, d, gen, stream, 2.0)
    dy, dsum_in = matrix(T, d, gen, scale=0.01), matrix(T, d, gen, stream, 0.01)
    gamma = 1 + 0.2 * torch.randn(d, generator=gen, device=DEV)
    y, total, dsum = torch.empty_like(x), torch.empty_like(r), torch.empty_like(r)
    dgamma = torch.empty(d, device=DEV)
    work = torch.empty(b.mosaic_rmsnorm_backward_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, sum=total)
    check_norm(y, x.double() + r.double(), gamma)
    source, h = total, total
    if kept in ("int8", "e4m3"):
        source = b.Q8Rows.empty(T, d, torch.int8 if kept == "int8" else torch.float8_e4m3fn, 64, DEV)
        b.mosaic_checkpoint_store(total, source)
        h = ref.restored(source.values, source.scales, 64)
    b.mosaic_rmsnorm_backward(dy, source, gamma, EPS, dsum, dgamma, work, dsum_in=dsum_in)
    want, want_gamma = ref.norm_gradients(dy, h, gamma, EPS, dsum_in)
    rms = torch.sqrt(h.double().square().mean(dim=1, keepdim=True) + EPS)
    n, c = h.double() / rms, dy.double() * gamma.double()
    size = (c.abs() + n.abs() * (c * n).abs().mean(dim=1, keepdim=True)) / rms + dsum_in.double().abs()
    unit = ref.U_BF16 if stream == torch.bfloat16 else ref.U_F32
    assert ((dsum.double() - want).abs() <= unit * want.abs() + (d + 32) * ref.U_F32 * size + 1e-38).all()
    size = (dy.double() * n).abs().sum(dim=0)
    assert ((dgamma.double() - want_gamma).abs() <= (T + d + 32) * ref.U_F32 * size + 1e-38).all()
