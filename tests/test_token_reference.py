"""What the token operators' tests compare with, pinned: the generator by its published known-answer vectors, gradients by
differences."""
import os

import numpy as np
import torch

import token_reference as ref

ROOT = os.path.dirname(os.path.abspath(__file__))


def test_generator_gives_the_published_words():
    seen = 0
    for line in open(os.path.join(ROOT, "golden", "closed_forms.txt")):
        if not line.startswith("philox"):
            continue
        words = [int(x, 16) for x in line.split()[1:]]
        got = ref.philox([np.array([c], dtype=np.uint64) for c in words[:4]], words[4:6])
        assert [int(g[0]) for g in got] == words[6:]
        seen += 1
    assert seen == 3


def test_mask_drops_the_share_and_keeps_the_mean():
    for p in (0.0, 0.1, 0.5, 0.9):
        mask, grow = ref.kept(200, 512, p, seed=12345678901234567890, site=2, first_row=(1 << 32) - 100)
        share = 1 - mask.double().mean().item()
        assert abs(share - p) <= 5 * (p * (1 - p) / mask.numel()) ** 0.5 + 2.0 ** -17
        assert abs(grow * (1 - round(p * 65536) / 65536) - 1) < 1e-12
    a, b = ref.kept(4, 64, 0.5, 7, first_row=10)[0], ref.kept(2, 64, 0.5, 7, first_row=12)[0]
    assert torch.equal(a[2:], b)
    assert not torch.equal(ref.kept(4, 64, 0.5, 7, site=1)[0], ref.kept(4, 64, 0.5, 7, site=0)[0])


def test_gradients_by_differences():
    gen = torch.Generator().manual_seed(3)
    rows, w = torch.randn((3, 8), generator=gen, dtype=torch.float64), torch.randn((11, 8), generator=gen, dtype=torch.float64)
    targets = torch.tensor([4, -1, 10])
    dl, de = torch.tensor([-0.5, 2.0, 0.25]), torch.tensor([0.3, -0.7, 0.0])

    def loss(r, m):
        logprob, entropy, _, _, _ = ref.logprobs(r @ m.t(), targets)
        return ((logprob * dl.double()) + entropy * de.double()).sum().item()
    dr, dw = ref.logprob_gradients(rows, w, targets, dl, de)
    h = 1e-6
    for t, g, at in ((rows, dr, (0, 3)), (rows, dr, (1, 5)), (w, dw, (4, 0)), (w, dw, (10, 7)), (w, dw, (2, 2))):
        up, down = t.clone(), t.clone()
        up[at] += h
        down[at] -= h
        d = (loss(up, w) - loss(down, w)) if t is rows else (loss(rows, up) - loss(rows, down))
        assert abs(d / (2 * h) - g[at].item()) < 1e-7


def test_logprobs_by_hand():
    x = torch.tensor([[0.0, 1.0, 1.0, -2.0]], dtype=torch.float64)
    logprob, entropy, lse, ids, tops = ref.logprobs(x, torch.tensor([3]), 6)
    z = 1 + 2 * np.e + np.exp(-2.0)
    assert abs(lse.item() - np.log(z)) < 1e-12 and abs(logprob.item() - (-2 - np.log(z))) < 1e-12
    p = np.array([1, np.e, np.e, np.exp(-2.0)]) / z
    assert abs(entropy.item() + (p * np.log(p)).sum()) < 1e-12
    assert ids.tolist() == [[1, 2, 0, 3, -1, -1]] and tops[0, 4] == -float("inf")
