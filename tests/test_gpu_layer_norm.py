"""Root-mean-square norm with the residual's addition, its 8-bit output and its gradient, and 8-bit rows, against plain
64-bit statements of the same."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


def matrix(T, d, dtype, gen, pad=0, scale=1.0):
    """A [T, d] view with `pad` columns behind every row, which hold a sentinel."""
    full = torch.full((T, d + pad), 777.0, dtype=dtype, device=DEV)
    full[:, :d] = (torch.randn((T, d), generator=gen) * scale).to(dtype).to(DEV)
    return full[:, :d], full


def untouched(full, d):
    return bool((full[:, d:] == 777.0).all())


def generator(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def check_y(y, h, gamma):
    """One rounding to bf16, and the sum of squares in 32 bits: off by at most d units, halved by the root; a few more."""
    want = ref.norm(h, gamma, EPS)
    bound = (ref.U_BF16 + (h.shape[1] + 16) * ref.U_F32) * want.abs() + 1e-38
    assert ((y.double().cpu() - want).abs() <= bound).all()


def check_q8(q8, y_exact, dtype, group, slack):
    """Scales of the groups, and every value within half a step of the format (plus what 32-bit inputs may be off)."""
    scales = q8.scales.cpu().double()
    want = ref.group_scales(y_exact, dtype, group)
    assert ((scales - want).abs() <= slack * want + 1e-45).all()
    wide = ref.widen(scales, group, y_exact.shape[1])
    back = q8.values.cpu().double() * wide
    if dtype == torch.int8:
        step = wide
    else:   # 3 fraction bits: the step is a sixteenth to an eighth of the magnitude, and 2^-9 below 2^-6
        step = torch.maximum(y_exact.abs() / 8 * (1 + 1e-6), wide * 2.0 ** -9)
    assert ((back - y_exact).abs() <= 0.5 * step + slack * y_exact.abs() + 1e-45).all()


@pytest.mark.parametrize("T,d", [(1, 8), (1, 4096), (3, 24), (5, 512), (7, 520), (9, 1000), (4, 1032), (6, 2048), (5, 2056),
                                 (1003, 3584), (33, 4104), (3, 8192), (2, 16384)])
@pytest.mark.parametrize("stream_type", [torch.bfloat16, torch.float32])
def test_norm_of_a_sum(T, d, stream_type):
    gen = generator(T * 100003 + d)
    x, _ = matrix(T, d, torch.bfloat16, gen, pad=8)
    r, _ = matrix(T, d, stream_type, gen, pad=16, scale=3.0)
    gamma_type = torch.float32 if (T + d) % 16 else torch.bfloat16
    gamma = (1 + 0.2 * torch.randn(d, generator=gen)).to(gamma_type).to(DEV)
    total, total_full = matrix(T, d, stream_type, gen, pad=24)
    y, y_full = matrix(T, d, torch.bfloat16, gen, pad=8)
    group = (32, 64, 128)[(T + d // 8) % 3]
    fmt = torch.int8 if d % 16 else torch.float8_e4m3fn
    q8 = b.Q8Rows.empty(T, d, fmt, group, DEV)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, sum=total, q8=q8)
    torch.cuda.synchronize()
    h = x.cpu().double() + r.cpu().double()
    unit = ref.U_BF16 if stream_type == torch.bfloat16 else ref.U_F32
    assert ((total.cpu().double() - h).abs() <= (unit + ref.U_F32) * h.abs()).all()
    check_y(y, h, gamma.cpu())
    check_q8(q8, ref.norm(h, gamma.cpu(), EPS), fmt, group, slack=(d + 16) * ref.U_F32)
    assert untouched(total_full, d) and untouched(y_full, d)


def test_one_input_alone_and_in_place():
    gen = generator(5)
    T, d = 37, 1024
    for stream_type in (torch.bfloat16, torch.float32):
        r, _ = matrix(T, d, stream_type, gen)
        x, _ = matrix(T, d, torch.bfloat16, gen)
        gamma = torch.rand(d, generator=gen).to(DEV)
        y = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
        b.mosaic_rmsnorm_forward(None, r, gamma, EPS, y)                       # a residual stream's own norm
        check_y(y, r.cpu().double(), gamma.cpu())
        h = x.cpu().double() + r.cpu().double()
        b.mosaic_rmsnorm_forward(x, r, gamma, EPS, x, sum=r)                   # y over x, the sum over the residual
        check_y(x, h, gamma.cpu())
        b.mosaic_rmsnorm_forward(x, None, gamma, EPS, y)
        check_y(y, x.cpu().double(), gamma.cpu())


@pytest.mark.parametrize("T,d", [(64, 512), (1000, 4096), (333, 1032)])
def test_listed_rows_only(T, d):
    """Only rows of the list are read (the others hold NaN) and written; entries outside the matrix are skipped."""
    gen = generator(T + d)
    x, _ = matrix(T, d, torch.bfloat16, gen)
    r, _ = matrix(T, d, torch.bfloat16, gen)
    gamma = torch.rand(d, generator=gen).to(DEV)
    mask = (torch.rand(T, generator=gen) < 0.4).to(torch.uint8).to(DEV)
    idx = torch.full((T,), 12345678, dtype=torch.int32, device=DEV)
    count = torch.zeros(1, dtype=torch.int32, device=DEV)
    scratch = torch.empty(b.mosaic_compact_scratch_bytes(T), dtype=torch.uint8, device=DEV)
    b.mosaic_mask_compact(mask, idx, count, scratch)
    kept = mask.cpu().bool()
    clean_x, clean_r = x.cpu(), r.cpu()
    x[~kept.to(DEV)] = float("nan")
    r[~kept.to(DEV)] = float("inf")
    y = torch.full((T, d), -5.0, dtype=torch.bfloat16, device=DEV)
    q8 = b.Q8Rows.empty(T, d, torch.int8, 128, DEV)
    q8.values.fill_(99)
    q8.scales.fill_(99.0)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, idx=idx, count=count, q8=q8)
    h = clean_x[kept].double() + clean_r[kept].double()
    check_y(y.cpu()[kept], h, gamma.cpu())
    assert (y.cpu()[~kept] == -5.0).all() and (q8.values.cpu()[~kept] == 99).all() and (q8.scales.cpu()[~kept] == 99).all()
    n = int(kept.sum())
    y.fill_(-5.0)
    bad = idx.clone()
    bad[0], bad[1] = -1, T                                                     # skipped
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, idx=bad, count=count, max_rows=n - 1)   # the bound cuts the last
    written = (y.cpu() != -5.0).any(dim=1)
    want = torch.zeros(T, dtype=torch.bool)
    want[idx.cpu()[2:n - 1].long()] = True
    assert torch.equal(written, want)
    count.zero_()
    y.fill_(-5.0)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y, idx=idx, count=count)
    assert (y == -5.0).all()


def test_special_rows():
    """A row of zeros gives zeros; NaN and infinities stay in their row; an 8-bit group with one restores as NaN."""
    T, d = 6, 640
    gen = generator(11)
    x, _ = matrix(T, d, torch.bfloat16, gen)
    x[1] = 0
    x[3, 17] = float("nan")
    x[5, 600] = float("inf")
    gamma = torch.ones(d, device=DEV)
    y = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    q8 = b.Q8Rows.empty(T, d, torch.float8_e4m3fn, 128, DEV)
    b.mosaic_rmsnorm_forward(x, None, gamma, EPS, y, q8=q8)
    assert (y[1] == 0).all() and (q8.scales[1] == 0).all() and (q8.values[1].float() == 0).all()
    assert y[3].isnan().all() and q8.scales[3].isnan().all()
    assert y[5, 600].isnan() and q8.scales[5, 4].isnan()       # inf / inf; the rest of the row is x / inf = 0
    for t in (0, 2, 4):
        assert y[t].isfinite().all() and q8.scales[t].isfinite().all()
    q8 = b.Q8Rows.empty(T, d, torch.int8, 128, DEV)
    b.mosaic_checkpoint_store(x, q8)
    out = torch.empty((T, d), dtype=torch.float32, device=DEV)
    b.mosaic_checkpoint_load(q8, out)
    bad = torch.zeros((T, d), dtype=torch.bool)
    bad[3, 0:128] = True
    bad[5, 512:640] = True
    assert torch.equal(out.cpu().isnan(), bad)


@pytest.mark.parametrize("T,d", [(1, 8), (3, 40), (257, 512), (65, 1000), (9, 3584), (2, 16384)])
@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_eight_bit_rows(T, d, fmt, group):
    gen = generator(T + 7 * d + group)
    for dtype in (torch.bfloat16, torch.float32):
        x, _ = matrix(T, d, dtype, gen, pad=8)
        x[:, d // 2] *= 40
        x[T // 2, :group] = 1e-36 if dtype == torch.float32 else 0.0          # below 2^-112: stored as zeros
        x[0, d - 8:] *= 1e-20
        values = torch.full((T, d + 8), 3, dtype=torch.uint8, device=DEV)
        scales = torch.full((T, -(-d // group) + 3), -1.0, device=DEV)
        q8 = b.Q8Rows(values[:, :d].view(fmt), scales[:, :-3], group)
        b.mosaic_checkpoint_store(x, q8)
        exact = x.cpu().double()
        exact[T // 2, :group] = 0
        check_q8(q8, exact, fmt, group, slack=4 * ref.U_F32)
        assert (values[:, d:] == 3).all() and (scales[:, -3:] == -1).all()
        out, full = matrix(T, d, torch.bfloat16, gen, pad=16)
        b.mosaic_checkpoint_load(q8, out)
        assert torch.equal(out.cpu(), ref.restored(q8.values.cpu(), q8.scales.cpu(), group))
        assert untouched(full, d)
        wide = torch.empty((T, d), device=DEV)
        b.mosaic_checkpoint_load(q8, wide)
        assert torch.equal(wide.cpu(), out.cpu().float())


def test_rounding_of_eight_bits():
    """Ties go to the even number, and the largest magnitude takes the format's largest number."""
    x = torch.zeros((1, 32), device=DEV)
    x[0, :8] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -127.0, 126.5])
    q8 = b.Q8Rows.empty(1, 32, torch.int8, 32, DEV)
    b.mosaic_checkpoint_store(x, q8)
    assert q8.scales.item() == 1.0 and q8.values[0, :8].tolist() == [127, 0, 2, 2, 0, -2, -127, 126]
    x[0, :8] = torch.tensor([448.0, 17.0, 19.0, -17.0, 1.0625, 1.1875, -448.0, 2.0 ** -10])
    q8 = b.Q8Rows.empty(1, 32, torch.float8_e4m3fn, 32, DEV)
    b.mosaic_checkpoint_store(x, q8)
    assert q8.scales.item() == 1.0
    assert q8.values[0, :8].float().tolist() == [448.0, 16.0, 20.0, -16.0, 1.0, 1.25, -448.0, 0.0]


@pytest.mark.parametrize("T,d", [(1, 8), (3, 512), (5, 520), (130, 1000), (9, 2056), (1003, 3584), (4099, 1024), (17, 4096),
                                 (3, 8200), (2, 16384)])
@pytest.mark.parametrize("kept", ["bf16", "f32", "int8", "e4m3"])
def test_norm_gradient(T, d, kept):
    gen = generator(3 * T + d)
    stream = torch.float32 if kept == "f32" or (T + d) % 3 == 0 and kept != "bf16" else torch.bfloat16
    h, _ = matrix(T, d, stream, gen, pad=8, scale=2.0)
    dy, _ = matrix(T, d, torch.bfloat16, gen, pad=16, scale=0.01)
    dsum_in, _ = matrix(T, d, stream, gen, scale=0.01)
    gamma = (1 + 0.2 * torch.randn(d, generator=gen)).to(DEV)
    dsum, full = matrix(T, d, stream, gen, pad=8)
    dgamma = torch.randn(d, generator=gen).to(DEV)
    start = dgamma.cpu().double()
    work = torch.full((b.mosaic_rmsnorm_backward_workspace_bytes(T, d) + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    source, h_exact = h, h.cpu()
    if kept in ("int8", "e4m3"):
        source = b.Q8Rows.empty(T, d, torch.int8 if kept == "int8" else torch.float8_e4m3fn, 64, DEV)
        b.mosaic_checkpoint_store(h, source)
        h_exact = ref.restored(source.values.cpu(), source.scales.cpu(), 64)
    b.mosaic_rmsnorm_backward(dy, source, gamma, EPS, dsum, dgamma, work[:-64], dsum_in=dsum_in)
    want, want_gamma = ref.norm_gradients(dy.cpu(), h_exact, gamma.cpu(), EPS, dsum_in.cpu())
    # 32-bit sums of d (rows) and T (columns) terms; what cancels is bounded by the terms' magnitudes
    rms = torch.sqrt(h_exact.double().square().mean(dim=1, keepdim=True) + EPS)
    n, c = h_exact.double() / rms, dy.cpu().double() * gamma.cpu().double()
    size = (c.abs() + n.abs() * (c * n).abs().mean(dim=1, keepdim=True)) / rms + dsum_in.cpu().double().abs()
    unit = ref.U_BF16 if stream == torch.bfloat16 else ref.U_F32
    assert ((dsum.cpu().double() - want).abs() <= unit * want.abs() + (d + 32) * ref.U_F32 * size + 1e-38).all()
    size = (dy.cpu().double() * n).abs().sum(dim=0)
    bound = (T + d + 32) * ref.U_F32 * size + 1e-38
    assert ((dgamma.cpu().double() - want_gamma).abs() <= bound).all()
    assert untouched(full, d) and (work[-64:] == 0xAB).all()
    first = dgamma.clone()
    dgamma.copy_(start.float())
    alone = torch.empty_like(dsum)
    b.mosaic_rmsnorm_backward(dy, source, gamma, EPS, alone, dgamma, work[:-64], accumulate=True)
    want2, _ = ref.norm_gradients(dy.cpu(), h_exact, gamma.cpu(), EPS)
    assert ((dgamma.cpu().double() - start - first.cpu().double()).abs() <= 2 * ref.U_F32 * (start.abs() + first.cpu().double().abs())).all()
    assert ref.relative(alone, want2) <= max(unit, (d + 32) * ref.U_F32)
    only = torch.empty_like(first)
    b.mosaic_rmsnorm_backward(dy, source, gamma, EPS, None, only, work[:-64])
    assert torch.equal(only, first)                                            # the same sums on every call


def test_norm_gradient_against_differences():
    """Along its own direction the gradient is what central differences of the 64-bit norm give."""
    gen = generator(21)
    T, d = 7, 512
    h, _ = matrix(T, d, torch.float32, gen)
    dy, _ = matrix(T, d, torch.bfloat16, gen)
    gamma = (1 + 0.2 * torch.randn(d, generator=gen)).to(DEV)
    dsum, dgamma = torch.empty_like(h), torch.empty(d, device=DEV)
    work = torch.empty(b.mosaic_rmsnorm_backward_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    b.mosaic_rmsnorm_backward(dy, h, gamma, EPS, dsum, dgamma, work)
    h0, g0, w = h.cpu().double(), gamma.cpu().double(), dy.cpu().double()
    for grad, at in ((dsum, 0), (dgamma, 1)):
        v = grad.cpu().double()
        v /= v.norm()
        e = 1e-4
        up = ref.norm(h0 + e * v, g0, EPS) if at == 0 else ref.norm(h0, g0 + e * v, EPS)
        down = ref.norm(h0 - e * v, g0, EPS) if at == 0 else ref.norm(h0, g0 - e * v, EPS)
        slope = ((up - down) * w).sum().item() / (2 * e)
        assert abs(slope - grad.double().norm().item()) <= 1e-5 * abs(slope)


def test_no_rows():
    d = 256
    empty = torch.empty((0, d), dtype=torch.bfloat16, device=DEV)
    gamma = torch.ones(d, device=DEV)
    b.mosaic_rmsnorm_forward(empty, empty, gamma, EPS, empty)
    dgamma = torch.full((d,), 3.0, device=DEV)
    b.mosaic_rmsnorm_backward(empty, empty, gamma, EPS, empty, dgamma, None, accumulate=True)
    assert (dgamma == 3.0).all()
    b.mosaic_rmsnorm_backward(empty, empty, gamma, EPS, empty, dgamma, None)
    assert (dgamma == 0.0).all()


def test_another_stream_and_a_graph():
    """Calls run on the stream they are given, and a captured call gives the eager result on every replay."""
    gen = generator(31)
    T, d = 129, 1024
    x, _ = matrix(T, d, torch.bfloat16, gen)
    r, _ = matrix(T, d, torch.bfloat16, gen)
    gamma = torch.rand(d, generator=gen).to(DEV)
    y, again = (torch.empty((T, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dgamma, dgamma2 = (torch.empty(d, device=DEV) for _ in range(2))
    dsum = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    work = torch.empty(b.mosaic_rmsnorm_backward_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, y)
    b.mosaic_rmsnorm_backward(y, x, gamma, EPS, dsum, dgamma, work)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b.mosaic_rmsnorm_forward(x, r, gamma, EPS, again, stream=side)
    side.synchronize()
    assert torch.equal(y, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.mosaic_rmsnorm_forward(x, r, gamma, EPS, again)
        b.mosaic_rmsnorm_backward(again, x, gamma, EPS, dsum, dgamma2, work)
    for _ in range(3):
        again.zero_()
        dgamma2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, again) and torch.equal(dgamma, dgamma2)
