"""Lookup, its gradient and the gradients of the log probabilities at 2^31 - 257 ids: four digits to sort by, clearing in several launches,
thousands of parts of the vocabulary."""
import pytest
import torch

from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
V, D = 2 ** 31 - 257, 8


@pytest.mark.parametrize("T", [1, 5000, 20011])
def test_lookup_and_its_gradient(T):
    gen = torch.Generator(device=DEV).manual_seed(T)
    tokens = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    tokens[T // 2:] = tokens[:T - T // 2].clone()                   # half of them a second time
    tokens[0], tokens[T - 1] = V - 1, 0 if T > 1 else V - 1
    dout = torch.randint(-3, 4, (T, D), generator=gen, device=DEV).to(BF16)
    dtable = torch.full((V, D), 7.0, dtype=BF16, device=DEV)
    ws = torch.empty(b.mosaic_embedding_backward_workspace_bytes(T, D, V), dtype=torch.uint8, device=DEV)
    print("gradient", T, flush=True)
    b.mosaic_embedding_backward(dout, tokens, dtable, ws)
    named, where = torch.unique(tokens.long(), return_inverse=True)
    want = torch.zeros((named.numel(), D), device=DEV).index_add_(0, where, dout.float())
    assert torch.equal(dtable[named].float(), want)
    assert int((dtable != 0).any(dim=1).sum()) == int((want != 0).any(dim=1).sum())      # and zeros everywhere else
    out = torch.full((T, D), 777.0, device=DEV)
    b.mosaic_embedding_forward(tokens, dtable, out, scale=0.5)
    assert torch.equal(out, want[where] * 0.5)


def test_gradients_of_log_probabilities():
    """All logits zero but a few, of one row; another row of zeros takes no part in dw."""
    planted = {0: 12.0, 5: -3.0, 2 ** 30: 20.0, V - 2: 25.0, V - 1: 24.0}
    w = torch.zeros((V, D), dtype=BF16, device=DEV)
    for at, value in planted.items():
        w[at, 0] = value
    hidden = torch.zeros((2, D), dtype=BF16, device=DEV)
    hidden[0, 0] = 1.0
    targets = torch.tensor([V - 1, 77], dtype=torch.int32, device=DEV)
    x = torch.tensor(list(planted.values()), dtype=torch.float64)
    lse = torch.log(x.exp().sum() + float(V - len(planted)))
    own = torch.tensor([24.0 - float(lse), -float(torch.log(torch.tensor(float(V), dtype=torch.float64)))], device=DEV).float()
    forward = [own, torch.zeros(2, device=DEV), torch.tensor([float(lse), -float(own[1])], device=DEV).float()]
    g = torch.full((2,), -0.5, device=DEV)
    dx, dw = torch.full((2, D), 777.0, dtype=BF16, device=DEV), torch.full((V, D), 777.0, dtype=BF16, device=DEV)
    ws = torch.full((b.mosaic_masked_logprobs_backward_workspace_bytes(2, D, V),), 0xFF, dtype=torch.uint8, device=DEV)
    print("logprobs backward", flush=True)
    b.mosaic_masked_logprobs_backward(hidden, w, None, None, 2, targets, forward[0], None, forward[2], g, None, dx, dw, ws)
    torch.cuda.synchronize()
    p = (x - lse).exp()
    dl = 0.5 * p
    dl[-1] -= 0.5
    # a result's rounding, 2^-8, and p, off by 2^-14 as its exponent is by 2^-15: the logits are up to 25, the log-sum-exp rounded to 32 bits
    close = 2.0 ** -8 + 2.0 ** -13
    got = dw[torch.tensor(list(planted), device=DEV), 0].cpu().double()
    assert ((got - dl).abs() <= close * dl.abs()).all()
    rest = 0.5 * float((-lse).exp())
    for r in range(0, V, 1 << 28):
        part = dw[r:r + (1 << 28), 0].float()
        off = (part - rest).abs() > close * rest
        assert set((off.nonzero()[:, 0] + r).tolist()) <= set(planted)
    assert not bool(dw[:, 1:].any())
    want = (dl * x).sum()
    assert abs(dx[0, 0].item() - float(want)) <= close * float((dl * x).abs().sum()) and not bool(dx[:, 1:].any())
    assert abs(dx[1, 0].item() - 0.5 * float(x.sum()) / V) <= close * float(x.abs().sum()) / V
