"""Log probabilities of few rows found of a large bound, of hidden states past 2 GiB, whose listed rows are gathered beforehand: what the
call takes and writes follows from the rows found."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_tokens_logprobs import BF16, DEV, check, grid

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("found", [0, 1, 10, 1000])
@pytest.mark.parametrize("d,V", [(64, 512), (72, 300)])
def test_rows_past_the_last_found_are_not_written(found, d, V):
    T, most = 520, 1000
    hidden = torch.zeros((T, 1 << 21), dtype=BF16, device=DEV)[:, :d]
    gen = torch.Generator().manual_seed(found + d)
    hidden.copy_(grid((T, d), gen, 1 / 8))
    w = grid((V, d), gen, 2.0 ** -8).to(DEV)
    idx = torch.randint(0, T, (most,), generator=gen).to(torch.int32).to(DEV)
    idx[found:] = 10 ** 9
    count = torch.tensor([found], dtype=torch.int32, device=DEV)
    targets = torch.randint(0, V, (most,), generator=gen).to(torch.int32).to(DEV)
    out = {k: torch.full((most,), -7.0, device=DEV) for k in ("logprob", "entropy", "lse")}
    near = b.mosaic_masked_logprobs_workspace_bytes(T, most, d, V)
    need = b.mosaic_masked_logprobs_workspace_bytes(T, most, d, V, ld_h=hidden.stride(0))
    assert need == near + 2 * most * d                       # the gathered rows come last
    ws = torch.full((need,), 0xAB, dtype=torch.uint8, device=DEV)
    b.mosaic_masked_logprobs(hidden, w, idx, count, most, targets, out["logprob"], out["entropy"], out["lse"], ws)
    torch.cuda.synchronize()
    assert bool((ws[near + 2 * found * d:] == 0xAB).all())
    got = {k: v.cpu() for k, v in out.items()}
    if found:
        check(got, ref.logits(hidden[idx[:found].long()], w), targets[:found], 0, d, 0.0, found, exact_logits=True)
    else:
        assert all(bool((v == -7).all()) for v in got.values())
