"""Log probabilities, entropies and alternatives at sizes that take every width and tile of their kernels, with one tile a unit and several,
with weights that are streamed, and with several units a block; test_tokens_choice_host.py holds the list to that.  Plain statements in 64
bits, on the device."""
import pytest
import torch

import token_reference as ref
from test_gpu_tokens_logprobs import BF16, DEV, F32, bounds, run

pytestmark = pytest.mark.gpu

SIZES = [  # rows, d, V
    # the 4-wave loop, one tile a unit
    (1, 64, 256), (36, 640, 270), (81, 64, 33280), (99, 64, 36864), (142, 64, 39680), (164, 64, 48384), (196, 64, 47872),
    (766, 64, 16640),
    # several tiles a unit, up to 14; ragged last tiles; several units a block
    (1, 64, 67584), (35, 64, 67328), (72, 64, 69120), (107, 64, 98560), (155, 64, 79360), (353, 64, 49920), (772, 64, 29184),
    (486, 64, 51968), (35, 320, 67300), (72, 320, 69001), (107, 384, 98505), (155, 320, 79350), (353, 320, 49900), (772, 320, 29100),
    (486, 320, 51969), (8329, 64, 2816), (8471, 64, 3584), (16640, 64, 8192), (1289, 384, 64768), (1151, 384, 43520), (7306, 256, 13056),
    (8312, 256, 14592),
    # a lone row tile under weights past the memory-side cache
    (1, 1408, 107264), (33, 1536, 98560), (65, 1536, 98561), (97, 1536, 98560), (129, 1536, 98700), (161, 1472, 102656),
    (193, 1472, 102656), (225, 1536, 98560), (225, 1536, 98815),
    # more rows than any but the widest tile is offered for
    (1048577, 64, 512), (1050001, 320, 270),
    # the kernel of eight waves
    (2, 16, 218), (1, 8, 97792), (80, 40, 201), (77, 16, 71424), (156, 8, 37632), (139, 32, 251), (130, 64, 66945), (8815, 136, 3314),
    (8544, 144, 1792), (1534, 248, 21760), (7281, 176, 8704), (1050001, 8, 300),
]
TOPS = (0, 2, 16)


def whole(shape, gen, step):
    """Multiples of `step`, as test_gpu_tokens_logprobs.grid: every sum of products is exact in 32 bits, in any order."""
    out = torch.empty(shape, dtype=BF16, device=DEV)
    for r in range(0, shape[0], 16384):
        n = min(shape[0], r + 16384) - r
        out[r:r + n] = (torch.randn((n, shape[1]), generator=gen, device=DEV) * 16).round().clamp(-127, 127) * step
    return out


def check(got, rows, w, targets, n_top):
    """As test_gpu_tokens_logprobs.check with exact logits, a part of the rows at a time."""
    M, V = rows.shape[0], w.shape[0]
    wt = w.double().t().contiguous()
    for r in range(0, M, max(1, (1 << 26) // V)):
        part = slice(r, min(M, r + max(1, (1 << 26) // V)))
        x = rows[part].double() @ wt
        lse = torch.logsumexp(x, dim=1)
        t = targets[part].long()
        has = (t >= 0) & (t < V)
        own = torch.where(has, x.gather(1, torch.where(has, t, 0)[:, None])[:, 0] - lse, 0.0)
        logp = x - lse[:, None]
        entropy = -(logp.exp() * logp).sum(dim=1)
        del logp
        off, off_lse = bounds(x, rows.shape[1], 0.0)
        spread = (x.amax(dim=1) - x.amin(dim=1)) + 1
        mine = {k: v[part].to(DEV).double() for k, v in got.items()}
        assert ((mine["lse"] - lse).abs() <= off_lse).all()
        assert ((mine["logprob"] - own).abs() <= off_lse + 2.0 ** -20 * own.abs()).all()
        assert ((mine["entropy"] - entropy).abs() <= 2 * off_lse * spread).all()
        if n_top:
            order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :n_top]
            tops = x.gather(1, order) - lse[:, None]
            assert torch.equal(mine["top_id"].long(), order)
            assert ((mine["top_logprob"] - tops).abs() <= off_lse[:, None] + 2.0 ** -20 * tops.abs()).all()
    for k, v in got.items():
        assert bool((v[M:] == -7).all()), k


def problem(M, d, V, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T = M + 5
    hidden = torch.full((T, d + 8), 777.0, dtype=BF16, device=DEV)[:, :d]
    hidden.copy_(whole((T, d), gen, 1 / 8))
    w = whole((V, d), gen, 2.0 ** -(4 + (d.bit_length() + 1) // 2))
    idx = torch.randint(0, T, (M,), generator=gen, device=DEV, dtype=torch.int32)
    targets = torch.randint(0, V, (M,), generator=gen, device=DEV, dtype=torch.int32)
    targets[M // 2] = V - 1
    if M > 4:
        targets[1], targets[2], idx[4] = -1, V, idx[0]
    return hidden, w, idx, targets


@pytest.mark.parametrize("M,d,V", SIZES)
def test_every_width(M, d, V):
    hidden, w, idx, targets = problem(M, d, V, M + d + V)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    for n_top in TOPS:
        check(run(hidden, w, idx, count, M, targets, n_top), hidden[idx.long()], w, targets, n_top)


@pytest.mark.parametrize("bound", [16640, 100000])
@pytest.mark.parametrize("M,d,V", [(36, 640, 2304), (196, 64, 47872), (766, 64, 16640), (772, 320, 29100), (155, 64, 79360), (77, 16, 71424)])
def test_rows_far_below_the_bound(M, d, V, bound):
    hidden, w, idx, targets = problem(bound, d, V, M + bound)
    idx[M:] = 10 ** 9                      # never looked at
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    for n_top in (0, 5):
        got = run(hidden, w, idx, count, bound, targets, n_top)
        check({k: v[:bound] for k, v in got.items()}, hidden[idx[:M].long()], w, targets[:M], n_top)
