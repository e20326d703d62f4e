"""A list with entries outside the rows: clamped in both directions of the log probabilities, left out where gradients are brought back
to their rows, unless the caller has clamped them."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b
from test_gpu_tokens_logprobs import problem
from test_gpu_tokens_logprobs_backward import BF16, DEV, F32, check, run, upstream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V,M", [(50, 64, 400, 20), (300, 128, 1024, 200), (90, 320, 2560, 80)])
@pytest.mark.parametrize("dw_type", [BF16, F32])
def test_gradients_of_clamped_entries(T, d, V, M, dw_type):
    hidden, w, idx, targets = problem(T, d, V, M, T + M, kind="any")
    idx[3], idx[5], idx[M - 1], idx[7] = -9, 10 ** 6, T, -2 ** 31
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    dl, de = upstream(M, M)
    dx, dw = run(hidden, w, idx, count, M, targets, dl, de, dw_type)
    clamped = idx.clamp(0, T - 1)
    check(dx, dw, hidden, w, clamped, targets, dl, de, M)
    same = run(hidden, w, clamped, count, M, targets, dl, de, dw_type)
    assert torch.equal(same[0], dx) and torch.equal(same[1], dw)
    # brought back to their rows: with the list as it is, without them; with the clamped one, all
    rows = dx[:M].contiguous()
    ws = torch.empty(b.mosaic_embedding_backward_workspace_bytes(M, d, T), dtype=torch.uint8, device=DEV)
    back = torch.full((T, d), 7.0, device=DEV)
    for tokens in (idx, clamped):
        b.mosaic_embedding_backward(rows, tokens, back, ws, count=count)
        want, size, n = ref.embedding_gradient(rows, tokens, T, 1.0)
        assert ((back.cpu().double() - want).abs() <= (n[:, None] + 1) * ref.U[F32] * size).all()
        there = (tokens >= 0) & (tokens < T)
        assert int(there.sum()) == (M if tokens is clamped else M - 4)
