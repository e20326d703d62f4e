"""Calls of the token operators that are allowed and rare: two at once, graphs that share a workspace, few steps of K, vocabularies near
the largest."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_tokens_logprobs import check, grid, problem, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.mark.parametrize("T,d,V,M", [(70, 64, 256, 70), (300, 64, 1024, 256), (70, 128, 768, 70), (600, 192, 2560, 600), (9, 320, 300, 9),
                                     (1300, 64, 5120, 1281), (40, 704, 50257, 33)])
@pytest.mark.parametrize("n_top", [0, 2, 16])
def test_few_steps_of_k(T, d, V, M, n_top):
    hidden, w, idx, targets = problem(T, d, V, M, T + d + V + n_top)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    check(run(hidden, w, idx, count, M, targets, n_top), ref.logits(hidden[idx.long()], w), targets, n_top, d, 0.0, M, exact_logits=True)


def everything(hidden, w, idx, count, M, targets, ws, stream=None):
    """Forward and backward into new tensors; (the outputs)."""
    V, d = w.shape
    own, entropy, lse = (torch.zeros(M, device=DEV) for _ in range(3))
    ids, best = torch.zeros((M, 3), dtype=torch.int32, device=DEV), torch.zeros((M, 3), device=DEV)
    dx, dw, dh = torch.zeros((M, d), dtype=BF16, device=DEV), torch.zeros((V, d), device=DEV), torch.zeros((hidden.shape[0], d), device=DEV)
    g = torch.full((M,), 0.5, device=DEV)

    def go():
        b.mosaic_masked_logprobs(hidden, w, idx, count, M, targets, own, entropy, lse, ws, top_id=ids, top_logprob=best, stream=stream)
        b.mosaic_masked_logprobs_backward(hidden, w, idx, count, M, targets, own, entropy, lse, g, g, dx, dw, ws, stream=stream)
        b.mosaic_embedding_backward(dx, idx, dh, ws, count=count, stream=stream)
    return go, [own, entropy, lse, ids, best, dx, dw, dh]


def space(T, M, d, V):
    return torch.zeros(max(b.mosaic_masked_logprobs_workspace_bytes(T, M, d, V, 3, ld_h=d + 8),
                           b.mosaic_masked_logprobs_backward_workspace_bytes(M, d, V),
                           b.mosaic_embedding_backward_workspace_bytes(M, d, T)), dtype=torch.uint8, device=DEV)


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own: the same bits as one after the other."""
    sizes = [(700, 256, 5000, 500), (90, 512, 8192, 40)]
    calls = []
    for n, (T, d, V, M) in enumerate(sizes):
        hidden, w, idx, targets = problem(T, d, V, M, 50 + n)
        count = torch.tensor([M], dtype=torch.int32, device=DEV)
        calls.append([everything(hidden, w, idx, count, M, targets, space(T, M, d, V), s)
                      for s in (None, torch.cuda.Stream())])
    for (alone, _), _ in calls:
        alone()
    torch.cuda.synchronize()
    for _ in range(5):
        for _, (beside, _) in calls:
            beside()
    torch.cuda.synchronize()
    for (_, want), (_, got) in calls:
        assert all(torch.equal(a, c) for a, c in zip(want, got))


def test_graphs_that_share_a_workspace():
    sizes = [(700, 256, 5000, 500), (90, 512, 8192, 40)]
    ws = space(700, 500, 512, 8192)
    graphs, outs, eager = [], [], []
    for n, (T, d, V, M) in enumerate(sizes):
        hidden, w, idx, targets = problem(T, d, V, M, 60 + n)
        count = torch.tensor([M], dtype=torch.int32, device=DEV)
        go, want = everything(hidden, w, idx, count, M, targets, space(T, M, d, V))
        go()
        eager.append((go, want))
        go, out = everything(hidden, w, idx, count, M, targets, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        graphs.append((graph, go))          # (what a graph reads has to live as long as it)
        outs.append(out)
    for order in ((0, 1), (1, 0), (1, 1), (0, 0)):
        for n in order:
            for t in outs[n]:
                t.zero_()
            graphs[n][0].replay()
            eager[n][0]()
        torch.cuda.synchronize()
        for n in order:
            assert all(torch.equal(a, c) for a, c in zip(eager[n][1], outs[n])), order


def test_a_workspace_for_more_rows_serves_fewer():
    hidden, w, idx, targets = problem(600, 512, 32000, 519, 70)
    ws = torch.full((b.mosaic_masked_logprobs_workspace_bytes(600, 519, 512, 32000, 3),), 0xFF, dtype=torch.uint8, device=DEV)
    for M in (1, 37, 256, 257, 482, 519):
        count = torch.tensor([M], dtype=torch.int32, device=DEV)
        own, entropy, lse = (torch.zeros(M, device=DEV) for _ in range(3))
        ids, best = torch.zeros((M, 3), dtype=torch.int32, device=DEV), torch.zeros((M, 3), device=DEV)
        b.mosaic_masked_logprobs(hidden, w, idx, count, M, targets, own, entropy, lse, ws, top_id=ids, top_logprob=best)
        torch.cuda.synchronize()
        got = dict(logprob=own.cpu(), entropy=entropy.cpu(), lse=lse.cpu(), top_id=ids.cpu(), top_logprob=best.cpu())
        check(got, ref.logits(hidden[idx[:M].long()], w), targets[:M], 3, 512, 0.0, M, exact_logits=True)


def test_the_largest_vocabulary():
    """2^31 - 257 ids: all logits zero but a few.  Sums of up to 2^23 equal terms a part are exact in 32 bits."""
    V, d = 2 ** 31 - 257, 8
    w = torch.zeros((V, d), dtype=BF16, device=DEV)
    planted = {0: 12.0, 5: -3.0, 2 ** 30: 20.0, V - 2: 25.0, V - 1: 24.0}
    for at, value in planted.items():
        w[at, 0] = value
    hidden = torch.zeros((2, d), dtype=BF16, device=DEV)
    hidden[0, 0] = 1.0                                              # the second row is uniform
    targets = torch.tensor([V - 1, 2 ** 31 - 300], dtype=torch.int32, device=DEV)
    got = run(hidden, w, None, None, 2, targets, 4)
    x = torch.tensor(list(planted.values()), dtype=torch.float64)
    rest = float(V - len(planted))
    lse = torch.log(x.exp().sum() + rest)
    p = (x - lse).exp()
    entropy = -(p * (x - lse)).sum() + rest * (-lse).exp() * lse
    uniform = torch.log(torch.tensor(float(V), dtype=torch.float64))
    # exponentials and their sums: 2^-20 each, of which up to 2^8 tiles' worth is added a part; of values up to 25 then 2^-18
    for name, first, second in (("lse", lse, uniform), ("logprob", 24.0 - lse, -uniform), ("entropy", entropy, uniform)):
        assert abs(got[name][0].item() - float(first)) <= 2.0 ** -12 and abs(got[name][1].item() - float(second)) <= 2.0 ** -12, name
    assert got["top_id"][0].tolist() == [V - 2, V - 1, 2 ** 30, 0]
    assert got["top_id"][1].tolist() == [0, 1, 2, 3]
