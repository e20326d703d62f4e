"""Gradients of the log probabilities at sizes that take every width and tile of their kernels and of the products behind them, one a block
and several, with the targets' rows added; test_tokens_choice_host.py holds the list to that.  Plain statements in 64 bits, on the
device."""
import pytest
import torch

import token_reference as ref
from test_gpu_tokens_logprobs_backward import BF16, DEV, F32, REST, TERMS, run

pytestmark = pytest.mark.gpu

SIZES = [  # rows, d, V, whether dw has 32 bits
    (1, 64, 260, True), (39, 64, 34687, False), (1177, 1728, 5, True), (69, 2048, 1125, False), (2097, 2048, 5, False),
    (1, 64, 98560, True), (70, 256, 32860, True), (3231, 1216, 6, False), (4652, 1688, 5, True), (13216, 1056, 5, False),
    (6526, 1200, 12, True), (12804, 2048, 5, True), (13893, 1720, 6, False), (35, 192, 105091, True), (69, 64, 33979, False),
    (66, 64, 40192, True), (33, 64, 76345, False), (107, 64, 33931, True), (66, 32, 65849, True), (121, 64, 34816, False),
    (68, 64, 68864, False), (72, 64, 67353, True), (129, 64, 43788, True), (113, 24, 68757, False), (134, 64, 47104, False),
    (322, 64, 22118, False), (331, 64, 24231, True), (11652, 64, 5796, True), (134, 64, 66048, True), (207, 64, 43776, True),
    (101, 128, 67328, False), (196, 64, 48128, False), (185, 8, 72801, True), (145, 8, 93010, False), (100, 128, 72680, True),
    (137, 64, 81920, False), (1133, 64, 11008, False), (708, 64, 18452, True), (487, 64, 33756, False), (13586, 64, 1280, False),
    (13642, 64, 1280, True), (14718, 64, 1487, False),
    # more rows than dx takes in one launch
    (140003, 64, 300, True), (140003, 72, 257, False), (262145, 64, 512, False),
    # K of many steps in every product
    (1500, 1032, 9003, False), (1500, 1024, 9003, True),
]


def check(dx, dw, rows, w, targets, g, h, bound=None):
    """As test_gpu_tokens_logprobs_backward.check, with the terms of dw held in two numbers where it has 32 bits or the rows are few.
    That goes by the bound, all that the host knows: for one row found of a bound of 1133 a term is off by 2^-8 as for 1133 rows."""
    M = rows.shape[0]
    few = (bound or M) <= 32
    rows, w = rows.double(), w.double()
    x = rows @ w.t().contiguous()
    logp = x - torch.logsumexp(x, dim=1)[:, None]
    del x
    p = logp.exp()
    entropy = -(p * logp).sum(dim=1)[:, None]
    t = targets.long()
    has = (t >= 0) & (t < w.shape[0])
    g = torch.where(has, g.double(), 0.0)[:, None]
    h = (torch.zeros(M, device=DEV) if h is None else h).double()[:, None]
    dl = -p * (g + h * (logp + entropy))
    dl[has, t[has]] += g[has, 0]
    rest = 2.0 ** -14 * p * (g.abs() + h.abs() * (1 + logp.abs() + entropy))
    del logp, p
    for got, exact, times in ((dx[:M], lambda: dl @ w, lambda off: off @ w.abs()),
                              (dw, lambda: dl.t().contiguous() @ rows, lambda off: off.t().contiguous() @ rows.abs())):
        terms = 2.0 ** -16 if few or got.dtype == F32 else TERMS
        want = exact()
        slack = times(terms * dl.abs() + rest)
        assert (got.double() - want).norm().item() <= (terms + ref.U[got.dtype] + REST) * want.norm().item()
        assert ((got.double() - want).abs() <= slack + (ref.U[got.dtype] + REST) * (want.abs() + slack) + 1e-30).all()


@pytest.mark.parametrize("M,d,V,wide", SIZES)
def test_every_tile(M, d, V, wide):
    gen = torch.Generator(device=DEV).manual_seed(M + d + V)
    T = M + 3
    hidden = torch.full((T, d + 8), 777.0, dtype=BF16, device=DEV)[:, :d]
    hidden.copy_(torch.randn((T, d), generator=gen, device=DEV))
    w = (torch.randn((V, d), generator=gen, device=DEV) * 2 * d ** -0.5).to(BF16)
    idx = torch.randint(0, T, (M,), generator=gen, device=DEV, dtype=torch.int32)
    targets = torch.randint(0, V, (M,), generator=gen, device=DEV, dtype=torch.int32)
    targets[M // 2] = V - 1
    targets[M // 4:M // 3] = V // 3            # one id's rows reach over pieces of their sum
    if M > 4:
        targets[1], targets[2] = -1, V
    g = -3 * (0.1 + torch.rand(M, generator=gen, device=DEV))
    h = torch.randn(M, generator=gen, device=DEV) * 0.2 if (M + V) % 2 else None
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    dx, dw = run(hidden, w, idx, count, M, targets, g, h, F32 if wide else BF16)
    check(dx, dw, hidden[idx.long()], w, targets, g, h)


@pytest.mark.parametrize("wide", [False, True])
def test_parts_of_the_vocabulary(wide):
    """More than the default workspace holds of dl: further parts are added in 32 bits to dx."""
    test_every_tile(2048, 192, 140003, wide)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("found", [0, 1, 257, 700])
@pytest.mark.parametrize("M,d,V", [(1133, 64, 11008), (1500, 1032, 9003), (708, 320, 29100)])
def test_rows_below_the_bound(M, d, V, found, wide):
    gen = torch.Generator(device=DEV).manual_seed(M + found)
    hidden = torch.randn((M, d), generator=gen, device=DEV).to(BF16)
    w = (torch.randn((V, d), generator=gen, device=DEV) * 2 * d ** -0.5).to(BF16)
    idx = torch.randint(0, M, (M,), generator=gen, device=DEV, dtype=torch.int32)
    targets = torch.randint(0, V, (M,), generator=gen, device=DEV, dtype=torch.int32)
    g, h = (torch.rand(M, generator=gen, device=DEV) for _ in range(2))
    idx[found:], g[found:], h[found:] = 10 ** 9, float("nan"), float("nan")          # never looked at
    count = torch.tensor([found], dtype=torch.int32, device=DEV)
    dx, dw = run(hidden, w, idx, count, M, targets, g, h, F32 if wide else BF16)
    assert bool((dx[found:] == 777.0).all())
    if found:
        check(dx, dw, hidden[idx[:found].long()], w, targets[:found], g[:found], h[:found], bound=M)
        if wide:
            _, more = run(hidden, w, idx, count, M, targets, g, h, F32, dw_start=0.25)
            assert torch.equal(more, dw + 0.25)
    else:
        assert bool((dw == 0).all())
