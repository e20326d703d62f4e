"""The LM head's gradient in 32 bits is a sum in 32 bits: its terms carry what their rounding to 16 bits leaves over, for any number of
rows.  Against automatic differentiation in 64 bits."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_tokens_logprobs import problem
from test_gpu_tokens_logprobs_backward import BF16, DEV, F32, REST, run, upstream

pytestmark = pytest.mark.gpu


def check(dw, rows, w, targets, dlogprob, dentropy):
    """Two numbers of 16 bits hold a term to 2^-8 of 2^-8.  Of the rest, as for few rows: p is off by 2^-14 relative (REST covers it in
    the 2-norm), log p + H by 2^-14; the sum's order and its 32 bits are below that."""
    zero = torch.zeros(rows.shape[0])
    _, want = ref.logprob_gradients(rows, w, targets, zero if dlogprob is None else dlogprob, dentropy)
    assert ref.relative(dw, want) <= 2.0 ** -16 + ref.U[F32] + REST
    x = ref.logits(rows, w)
    logp = x - torch.logsumexp(x, dim=1)[:, None]
    p = logp.exp()
    entropy = -(p * logp).sum(dim=1)[:, None]
    t = targets.cpu().long()
    has = (t >= 0) & (t < x.shape[1])
    g = torch.where(has, (zero if dlogprob is None else dlogprob).cpu().double(), 0.0)[:, None]
    h = (zero if dentropy is None else dentropy).cpu().double()[:, None]
    dl = -p * (g + h * (logp + entropy))
    dl[has, t[has]] += g[has, 0]
    off = 2.0 ** -16 * dl.abs() + 2.0 ** -14 * p * (g.abs() + h.abs() * (1 + logp.abs() + entropy))
    slack = off.t() @ rows.cpu().double().abs()
    assert ((dw.double().cpu() - want).abs() <= slack + (ref.U[F32] + REST) * (want.abs() + slack) + 1e-30).all()


SIZES = [  # T, d, V, M
    (40, 64, 300, 33), (65, 512, 1000, 65), (40, 1032, 3001, 37), (129, 200, 2056, 129), (300, 64, 513, 256), (700, 128, 8003, 500),
    (1100, 96, 1500, 1024), (900, 320, 5120, 777), (16, 2048, 2000, 16), (3000, 64, 700, 2900),
]


@pytest.mark.parametrize("T,d,V,M", SIZES)
@pytest.mark.parametrize("kind", ["logprob", "both", "entropy"])
def test_a_sum_in_32_bits(T, d, V, M, kind):
    hidden, w, idx, targets = problem(T, d, V, M, T + d + V + 1, kind="any")
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    dl, de = upstream(M, M)
    dl, de = (dl if kind != "entropy" else None), (de if kind != "logprob" else None)
    dx, dw = run(hidden, w, idx, count, M, targets, dl, de, F32)
    check(dw, hidden[idx.long()], w, targets, dl, de)
    alone, _ = run(hidden, w, idx, count, M, targets, dl, de, want=("dx",))
    assert ref.relative(dx[:M], alone[:M]) <= 2.0 ** -8        # one rounding of sums that differ in their last bits
    again = run(hidden, w, idx, count, M, targets, dl, de, F32)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("found", [1, 63, 64, 199])
def test_fewer_rows_than_the_bound_in_a_small_workspace(found):
    hidden, w, idx, targets = problem(300, 128, 3001, 200, found, kind="any")
    idx[found:] = 10 ** 9                      # never looked at
    count = torch.tensor([found], dtype=torch.int32, device=DEV)
    dl, de = upstream(200, 9)
    dl[found:] = de[found:] = float("nan")
    _, dw = run(hidden, w, idx, count, 200, targets, dl, de, F32, budget=1)
    check(dw, hidden[idx[:found].long()], w, targets[:found], dl[:found], de[:found])


def test_a_batch_in_parts():
    """Halves of the rows, the second added to the first: as close as the whole."""
    hidden, w, idx, targets = problem(700, 128, 3001, 600, 3, kind="any")
    dl, de = upstream(600, 4)
    dw = torch.full((3001, 128), 7.0, device=DEV)
    for half, (a, e) in enumerate(((0, 350), (350, 600))):
        n = e - a
        count = torch.tensor([n], dtype=torch.int32, device=DEV)
        out = [torch.zeros(n, device=DEV) for _ in range(3)]
        ws = torch.empty(max(b.mosaic_masked_logprobs_workspace_bytes(700, n, 128, 3001, ld_h=hidden.stride(0)),
                             b.mosaic_masked_logprobs_backward_workspace_bytes(n, 128, 3001)), dtype=torch.uint8, device=DEV)
        b.mosaic_masked_logprobs(hidden, w, idx[a:e], count, n, targets[a:e], *out, ws)
        b.mosaic_masked_logprobs_backward(hidden, w, idx[a:e], count, n, targets[a:e], *out, dl[a:e], de[a:e], None, dw, ws,
                                          accumulate=half > 0)
    check(dw, hidden[idx.long()], w, targets, dl, de)


def test_the_same_terms_in_16_bits_are_rounded_once():
    """Beside it, for comparison: 16-bit results of few rows come from the same sums."""
    hidden, w, idx, targets = problem(40, 256, 2000, 32, 6, kind="any")
    count = torch.tensor([32], dtype=torch.int32, device=DEV)
    dl, de = upstream(32, 7)
    _, wide = run(hidden, w, idx, count, 32, targets, dl, de, F32)
    _, narrow = run(hidden, w, idx, count, 32, targets, dl, de, BF16)
    assert torch.equal(wide.to(BF16), narrow)
