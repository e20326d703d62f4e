"""The rare calls of the log probabilities at sizes that the 4-wave loop takes: logits in orders that candidates have it hard with, rows
that are no numbers, entries outside the rows, counts below the bound, a captured graph with other counts."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_tokens_logprobs import BF16, DEV, grid, problem, run
from test_gpu_tokens_logprobs import check as check_on_host
from test_gpu_tokens_widths import check
from token_choice import four_waves

pytestmark = pytest.mark.gpu

ORDERS = [(20, 64, 131328), (70, 64, 133120), (70, 64, 20224), (196, 64, 47872), (675, 64, 58368), (353, 320, 49900), (1, 64, 67584),
          (8329, 64, 2816)]


@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "zero rows"])
@pytest.mark.parametrize("M,d,V", ORDERS)
def test_orders_that_candidates_have_it_hard_with(M, d, V, kind):
    """All logits equal, every id better than all before it, the reverse, two values in turn, and zeroed hidden rows: the lower id comes
    first.  An id is 2^14 a + 2^7 b + c, and its logit v / 1024, exactly."""
    assert four_waves(d, V)
    v = torch.arange(V, device=DEV)
    w = torch.zeros((V, d), device=DEV)
    if kind in ("equal", "two"):
        w[:, 0] = 1.0 if kind == "equal" else (v % 2).float()
    else:
        w[:, 0], w[:, 1], w[:, 2] = (v // 16384).float(), (v // 128 % 128).float(), (v % 128).float()
    hidden = torch.zeros((M, d), device=DEV)
    sign = {"falling": -1.0, "zero rows": 0.0}.get(kind, 1.0)
    hidden[:, 0], hidden[:, 1], hidden[:, 2] = sign * 16, sign / 8, sign / 1024
    if kind == "zero rows":
        hidden[::3, :3] = torch.tensor([16, 1 / 8, 1 / 1024], device=DEV)      # beside rows that are not
    hidden, w = hidden.to(BF16), w.to(BF16)
    gen = torch.Generator(device=DEV).manual_seed(M)
    targets = torch.randint(0, V, (M,), generator=gen, device=DEV, dtype=torch.int32)
    for n_top in (1, 5, 16):
        check(run(hidden, w, None, None, M, targets, n_top), hidden, w, targets, n_top)


@pytest.mark.parametrize("n_top", [0, 1, 5, 16])
@pytest.mark.parametrize("T,d,V,M", [(150, 64, 5120, 130), (150, 320, 5000, 130), (150, 64, 70656, 130)])
def test_not_a_number_stays_in_its_row(T, d, V, M, n_top):
    assert four_waves(d, V)
    hidden, w, idx, targets = problem(T, d, V, M, 12)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    idx[7], idx[100] = T - 1, T - 2
    odd = torch.zeros(M, dtype=torch.bool, device=DEV)
    odd[7] = odd[100] = True
    idx[(idx >= T - 2) & ~odd] = 0
    clean = run(hidden, w, idx, count, M, targets, n_top)
    hidden[T - 1, 3], hidden[T - 2, 5] = float("nan"), float("inf")
    got = run(hidden, w, idx, count, M, targets, n_top)
    other = torch.ones(M + 3, dtype=torch.bool)
    other[7] = other[100] = False
    for k in got:
        assert torch.equal(got[k][other], clean[k][other]), k
    for row in (7, 100):
        assert got["lse"][row].isnan() and got["entropy"][row].isnan()
        if n_top:
            assert bool(((got["top_id"][row] >= -1) & (got["top_id"][row] < V)).all())
    assert clean["lse"][:M].isfinite().all()


@pytest.mark.parametrize("T,d,V,M", [(50, 64, 512, 20), (300, 128, 5120, 200), (300, 320, 5001, 290)])
def test_entries_outside_are_clamped(T, d, V, M):
    assert four_waves(d, V)
    hidden, w, idx, targets = problem(T, d, V, M, 8)
    idx[3], idx[5], idx[M - 1], idx[0] = -9, 10 ** 6, T, -2 ** 31
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    for n_top in (0, 3):
        got = run(hidden, w, idx, count, M, targets, n_top)
        check_on_host(got, ref.logits(hidden[idx.long().clamp(0, T - 1)], w), targets, n_top, d, 0.0, M, exact_logits=True)


@pytest.mark.parametrize("M,count", [(200, 0), (200, 1), (200, 63), (200, 200), (200, 1000), (200, -4), (3000, 5), (3000, 70), (3000, 700)])
@pytest.mark.parametrize("n_top", [0, 5])
def test_count_below_the_bound(M, count, n_top):
    hidden, w, idx, targets = problem(500, 128, 5120, M, M + count)
    have = max(0, min(M, count))
    idx[have:] = 10 ** 9
    got = run(hidden, w, idx, torch.tensor([count], dtype=torch.int32, device=DEV), M, targets, n_top)
    if have:
        check_on_host(got, ref.logits(hidden[idx[:have].long()], w), targets[:have], n_top, 128, 0.0, have, exact_logits=True)
    else:
        assert all(bool((v == -7).all()) for v in got.values())


@pytest.mark.parametrize("n_top", [0, 4])
@pytest.mark.parametrize("d,V", [(256, 5120), (320, 33001)])
def test_replayed_from_a_graph(d, V, n_top):
    T, M = 900, 700
    hidden, w, idx, targets = problem(T, d, V, M, 31)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    outs = [torch.zeros(M, device=DEV) for _ in range(3)]
    top_id = torch.zeros((M, n_top), dtype=torch.int32, device=DEV) if n_top else None
    top_lp = torch.zeros((M, n_top), device=DEV) if n_top else None
    ws = torch.empty(b.mosaic_masked_logprobs_workspace_bytes(T, M, d, V, n_top, ld_h=hidden.stride(0)), dtype=torch.uint8, device=DEV)
    everything = [t for t in (*outs, top_id, top_lp) if t is not None]

    def step():
        b.mosaic_masked_logprobs(hidden, w, idx, count, M, targets, *outs, ws, top_id=top_id, top_logprob=top_lp)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    gen = torch.Generator().manual_seed(6)
    for n in (700, 90, 300, 0, 20, 513):
        hidden.copy_(grid((T, d), gen, 1 / 8))
        count.fill_(n)
        for t in everything:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in everything]
        for t in everything:
            t.fill_(-7)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, everything))
        named = dict(zip(("logprob", "entropy", "lse", "top_id", "top_logprob"), got))
        check(named, hidden[idx[:n].long()], w, targets[:n], n_top)
