"""Gradients of the log probabilities in the workspace that their query gives, where it is smallest: 33 to 63 rows, few ids, or a budget
that leaves room for one tile of ids."""
import pytest
import torch

from test_gpu_tokens_logprobs import problem
from test_gpu_tokens_logprobs_backward import BF16, DEV, F32, check, run, upstream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,budget", [(5, 0), (256, 0), (5000, 1), (8191, 1)])
@pytest.mark.parametrize("M", [1, 32, 33, 40, 63, 64, 65])
def test_the_smallest(M, V, budget):
    hidden, w, idx, targets = problem(M + 7, 128, V, M, M + V, kind="any")
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    dl, de = upstream(M, M + 1)
    for dw_type in (BF16, F32):
        dx, dw = run(hidden, w, idx, count, M, targets, dl, de, dw_type, budget=budget)
        check(dx, dw, hidden, w, idx, targets, dl, de, M)
