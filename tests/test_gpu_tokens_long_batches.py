"""The lookup's gradient for more tokens than a sorting wave holds in registers (from 524289 on), over one, two and three digits.  The
gradients are small whole numbers, whose sums are exact in 32 bits in any order."""
import pytest
import torch

from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T", [524287, 524288, 524289, 540673, 1000003])
@pytest.mark.parametrize("V", [1, 300, 126464, (1 << 21) + 5])
@pytest.mark.parametrize("same", [0.0, 0.5])
def test_more_tokens_than_waves_hold(T, V, same):
    d = 8
    gen = torch.Generator(device=DEV).manual_seed(T + V)
    tokens = torch.randint(-V // 100 - 1, V + V // 100 + 1, (T,), generator=gen, device=DEV, dtype=torch.int32)
    tokens[torch.rand(T, generator=gen, device=DEV) < same] = V - 1
    dout = torch.randint(-3, 4, (T, d), generator=gen, device=DEV).to(BF16)
    found = T - 1234
    count = torch.tensor([found], dtype=torch.int32, device=DEV)
    need = b.mosaic_embedding_backward_workspace_bytes(T, d, V)
    ws = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device=DEV)
    print("gradient", T, V, same, flush=True)
    for n, at in ((T, None), (found, count)):
        t = tokens[:n].long()
        there = (t >= 0) & (t < V)
        want = torch.zeros((V, d), device=DEV).index_add_(0, t[there], dout[:n][there].float())
        dtable = torch.full((V, d), 7.0, device=DEV)
        b.mosaic_embedding_backward(dout, tokens, dtable, ws[:need], count=at)
        assert torch.equal(dtable, want)
        b.mosaic_embedding_backward(dout, tokens, dtable, ws[:need], count=at, accumulate=True)
        assert torch.equal(dtable, 2 * want)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xAB).all())
