"""The token operators together, as the examples use them: a training step of a masked-diffusion model around one layer against
64-bit automatic differentiation, rows that a gather list names twice, a captured step, and the commands."""
import pytest
import torch

import layer_reference
import token_reference as ref
from paper_2601_06562_amd import binding as b
from paper_2601_06562_amd import example, example_tokens

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF16 = torch.bfloat16


def a_model(T, d, d_ff, V, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    model = example_tokens.MaskedDiffusion(T, d, d_ff, V, gen, DEV)
    tokens = torch.randint(0, V, (T,), generator=gen, device=DEV).to(torch.int32)
    mask = (torch.rand(T, generator=gen, device=DEV) < 0.6).to(torch.uint8)
    return model, tokens, mask


def as_stored(value, stored):
    """What the kernels kept, with the gradient of `value`."""
    return value + (stored.detach().cpu().double() - value).detach()


# Roundings to 16 bits that a gradient has passed on its way: of the logits' gradient and the rows' (2), of the final norm's (3),
# the dropout's (4), the block's inner gradient (5), its projections' (6) and the input's (7), the layer's sum (8), the first
# dropout (9); a weight's gradient has its own beside those of what it is made from.  A rounding moves a gradient by at most 2^-8
# of its 2-norm (half a step everywhere); what follows is linear and takes such a difference, which has no direction, no further than
# the gradient itself.
ROUNDINGS = dict(head=2, final=2, down=6, gate=7, up=7, gamma=7, places=9, table=9)


def test_training_step():
    T, d, d_ff, V, seed = 260, 192, 384, 1003, 5
    model, tokens, mask = a_model(T, d, d_ff, V, 21)
    masked = int(mask.sum().item())
    loss, grads, kept = model.train_step(tokens, mask, masked, seed)
    torch.cuda.synchronize()
    layer = model.layer
    given = dict(head=model.head, final=model.gamma, down=layer.w_down, gate=layer.w_gate, up=layer.w_up, gamma=layer.gamma,
                 places=model.places, table=model.table)
    leaf = {k: v.cpu().double().requires_grad_(True) for k, v in given.items()}
    shown = torch.where(mask.bool(), V, tokens).cpu().long()
    (keep0, grow), (keep1, _) = (ref.kept(T, d, model.p, seed, site) for site in (0, 1))
    total = leaf["table"][shown] * model.scale * keep0 * grow + leaf["places"]
    total = as_stored(total, layer_reference.restored(model.kept[0].values.cpu(), model.kept[0].scales.cpu(), 128))
    y = layer_reference.norm(total, leaf["gamma"], example_tokens.EPS)
    y = as_stored(y, layer_reference.restored(model.kept[1].values.cpu(), model.kept[1].scales.cpu(), 128))
    out = layer_reference.ffn(y, leaf["gate"], leaf["up"], "silu") @ leaf["down"].t()
    stream = as_stored(total + out * keep1 * grow, kept["stream"])
    at = mask.cpu().nonzero()[:, 0]
    hidden = as_stored(layer_reference.norm(stream, leaf["final"], example_tokens.EPS)[at], kept["hidden"][at.to(DEV)])
    own = ref.logprobs(hidden @ leaf["head"].t(), tokens.cpu()[at])[0]
    want = -own.sum() / masked
    want.backward()
    assert torch.equal(kept["targets"].cpu(), tokens.cpu()[at])
    assert abs(loss.item() - want.item()) <= 2.0 ** -12 * abs(want.item())
    assert set(grads) == set(leaf)
    off = {k: ref.relative(grads[k], leaf[k].grad) * 2.0 ** 8 for k in grads}
    print(off)
    for k in grads:
        assert off[k] <= ROUNDINGS[k], (k, off)
    unnamed = torch.ones(V + 1, dtype=torch.bool)
    unnamed[shown] = False
    assert bool((grads["table"].cpu()[unnamed] == 0).all())


def test_steps_repeat():
    """The same bits for the same seed, others for another one."""
    model, tokens, mask = a_model(130, 128, 256, 777, 3)
    masked = int(mask.sum().item())
    first = model.train_step(tokens, mask, masked, 9)[1]
    again = model.train_step(tokens, mask, masked, 9)[1]
    other = model.train_step(tokens, mask, masked, 10)[1]
    assert all(torch.equal(first[k], again[k]) for k in ("head", "table", "places", "final"))
    assert not torch.equal(first["table"], other["table"])


@pytest.mark.parametrize("T,d,V", [(300, 64, 500), (2100, 200, 40)])
def test_rows_listed_twice(T, d, V):
    """Shifted lists name a row twice where a sequence begins with two masked positions; both gradients arrive there."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T)
    hidden, w = (torch.randn(shape, generator=gen, device=DEV).to(BF16) for shape in ((T, d), (V, d)))
    w = (w.float() * d ** -0.5).to(BF16)
    mask = (torch.rand(T, generator=gen, device=DEV) < 0.4).to(torch.uint8)
    starts = [0, T // 3, T // 2, T]
    for s in starts[:-1]:
        mask[s:s + 2] = 1
    idx, gather = (torch.zeros(T, dtype=torch.int32, device=DEV) for _ in range(2))
    count = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.mosaic_mask_compact(mask, idx, count, torch.empty(b.mosaic_compact_scratch_bytes(T) + 16, dtype=torch.uint8, device=DEV))
    b.mosaic_shift_indices(idx, count, T, torch.tensor(starts, dtype=torch.int32, device=DEV), gather)
    M = int(count.item())
    rows = gather[:M].cpu().long()
    assert rows.unique().numel() == M - 3
    targets = torch.randint(-1, V, (T,), generator=gen, device=DEV).to(torch.int32)
    g = torch.randn(T, generator=gen, device=DEV)
    own, entropy, lse = (torch.zeros(T, device=DEV) for _ in range(3))
    need = max(b.mosaic_masked_logprobs_workspace_bytes(T, T, d, V), b.mosaic_masked_logprobs_backward_workspace_bytes(T, d, V),
               b.mosaic_embedding_backward_workspace_bytes(T, d, T))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    drows, dhidden = (torch.empty((T, d), dtype=BF16, device=DEV) for _ in range(2))
    b.mosaic_masked_logprobs(hidden, w, gather, count, T, targets, own, entropy, lse, ws)
    b.mosaic_masked_logprobs_backward(hidden, w, gather, count, T, targets, own, entropy, lse, g, None, drows, None, ws)
    b.mosaic_embedding_backward(drows, gather, dhidden, ws, count=count)
    want, _ = ref.logprob_gradients(hidden[rows.to(DEV)], w, targets[:M], g[:M])
    want = torch.zeros((T, d), dtype=torch.float64).index_add(0, rows, want)
    assert ref.relative(dhidden, want) <= 3 * 2.0 ** -8 + 2.0 ** -14      # terms, rows, and sums of rows
    exact = torch.zeros((T, d), dtype=torch.float64).index_add(0, rows, drows[:M].cpu().double())
    assert ((dhidden.cpu().double() - exact).abs() <= (2.0 ** -8 + 2.0 ** -20) * exact.abs() + 1e-30).all()


def test_a_captured_step():
    """Lookup, dropout, log probabilities, their gradients and the table's in one graph: every replay gives what eager calls give,
    with other tokens, masks and counts, and eager work between the replays."""
    T, d, V, n = 150, 128, 700, 3
    gen = torch.Generator(device=DEV)
    gen.manual_seed(8)
    table = (torch.randn((V, d), generator=gen, device=DEV) * d ** -0.5).to(BF16)
    tokens, targets = (torch.zeros(T, dtype=torch.int32, device=DEV) for _ in range(2))
    mask = torch.zeros(T, dtype=torch.uint8, device=DEV)
    scratch = torch.empty(b.mosaic_compact_scratch_bytes(T) + 16, dtype=torch.uint8, device=DEV)
    need = max(b.mosaic_masked_logprobs_workspace_bytes(T, T, d, V, n), b.mosaic_masked_logprobs_backward_workspace_bytes(T, d, V),
               b.mosaic_embedding_backward_workspace_bytes(T, d, V))

    def buffers():
        f = [torch.zeros(T, device=DEV) for _ in range(3)]
        return dict(x=torch.zeros((T, d), dtype=BF16, device=DEV), idx=torch.zeros(T, dtype=torch.int32, device=DEV),
                    count=torch.zeros(1, dtype=torch.int32, device=DEV), own=f[0], entropy=f[1], lse=f[2],
                    ids=torch.zeros((T, n), dtype=torch.int32, device=DEV), best=torch.zeros((T, n), device=DEV),
                    drows=torch.zeros((T, d), dtype=BF16, device=DEV), dhead=torch.zeros((V, d), device=DEV),
                    dx=torch.zeros((T, d), dtype=BF16, device=DEV), dtable=torch.zeros((V, d), device=DEV),
                    ws=torch.zeros(need, dtype=torch.uint8, device=DEV))
    ones = torch.full((T,), -1.0, device=DEV)

    def step(o):
        b.mosaic_embedding_forward(tokens, table, o["x"], scale=d ** 0.5)
        b.mosaic_dropout_forward(o["x"], None, o["x"], 0.2, 77, site=3)
        b.mosaic_mask_compact(mask, o["idx"], o["count"], scratch)
        b.mosaic_masked_logprobs(o["x"], table, o["idx"], o["count"], T, targets, o["own"], o["entropy"], o["lse"], o["ws"],
                                 top_id=o["ids"], top_logprob=o["best"])
        b.mosaic_masked_logprobs_backward(o["x"], table, o["idx"], o["count"], T, targets, o["own"], o["entropy"], o["lse"], ones, ones,
                                          o["drows"], o["dhead"], o["ws"])
        b.mosaic_embedding_backward(o["drows"], o["idx"], o["dx"], o["ws"], count=o["count"])
        b.mosaic_dropout_backward(o["dx"], o["dx"], 0.2, 77, site=3)
        b.mosaic_embedding_backward(o["dx"], tokens, o["dtable"], o["ws"], scale=d ** 0.5)
    eager, captured = buffers(), buffers()
    mask.fill_(1)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for share in (0.5, 0.0, 1.0, 0.1):
        tokens.copy_(torch.randint(-1, V, (T,), generator=gen, device=DEV))
        targets.copy_(torch.randint(-1, V, (T,), generator=gen, device=DEV))
        mask.copy_(torch.rand(T, generator=gen, device=DEV) < share)
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        M = int(captured["count"].item())
        assert M == int(mask.sum().item())
        for k in eager:
            if k == "ws":
                continue
            cut = M if k in ("idx", "own", "entropy", "lse", "ids", "best", "drows") else None
            assert torch.equal(eager[k][:cut], captured[k][:cut]), (k, share)
        assert bool(captured["dtable"].isfinite().all()) and bool(captured["dhead"].isfinite().all())


def test_scoring_unmasks_by_margin():
    model, tokens, mask = a_model(200, 128, 256, 600, 4)
    masked = int(mask.sum().item())
    starts = torch.tensor([0, 90, 200], dtype=torch.int32, device=DEV)
    before, left = tokens.clone(), mask.clone()
    own, margin = model.score_step(before, left, starts, torch.tensor([3, 5], dtype=torch.int32, device=DEV), masked)
    torch.cuda.synchronize()
    at = mask.cpu().nonzero()[:, 0]
    hidden = model.forward(tokens, mask)[2]
    x = ref.logits(hidden[at.to(DEV)], model.head)
    want, _, _, ids, best = ref.logprobs(x, tokens.cpu()[at], 2)
    # a logit is off by at most d products' roundings: 2^-13 at these sizes, and a log probability by twice that
    assert (own.cpu().double() - want).abs().max() <= 2.0 ** -12
    assert (margin.cpu().double() - (best[:, 0].exp() - best[:, 1].exp())).abs().max() <= 2.0 ** -12
    taken = (mask != left).cpu().nonzero()[:, 0]
    assert taken.numel() == 8 and int((taken < 90).sum()) == 3
    for lo, hi, n in ((0, 90, 3), (90, 200, 5)):
        here = (at >= lo) & (at < hi)
        order = torch.sort(margin.cpu()[here], descending=True, stable=True).indices[:n]
        assert sorted(at[here][order].tolist()) == [t for t in taken.tolist() if lo <= t < hi]


def test_the_commands_run():
    example_tokens.main(["--rows", "300", "--d", "256", "--d-ff", "512", "--vocab", "2048"])
    for by in ("margin", "entropy", "probability"):
        example.main(["--seq-len", "256", "--block", "64", "--steps", "3", "--d", "128", "--vocab", "1000", "--by", by])
