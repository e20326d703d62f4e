"""Which kernels and tiles the log probabilities and their gradients take, on the CPU: whatever the heads of the measured cases take, at any
number of rows up to a batch's, is run by test_gpu_tokens_widths.py and test_gpu_tokens_gradient_tiles.py."""
import math
import os
import random

import pytest

import test_gpu_tokens_gradient_tiles as gradients
import test_gpu_tokens_widths as forward
import token_choice as tc

HEADS = [(512, 8192), (1024, 32000), (1032, 32003), (704, 50257), (2048, 65536), (4096, 126464), (3584, 152064), (64, 256), (128, 5000)]
pytestmark = pytest.mark.skipif(not os.path.exists(tc.HIPCC), reason="no hipcc")


@pytest.fixture(scope="module")
def choice(tmp_path_factory):
    return tc.Choice(str(tmp_path_factory.mktemp("choice")))


def sweep(n, most, seed):
    rng = random.Random(seed)
    return [(int(math.exp(rng.uniform(0, math.log(most)))), *rng.choice(HEADS), rng.random() < 0.5) for _ in range(n)]


def missing(taken, sizes, tested):
    first = {}
    for size, ways in zip(sizes, taken):
        for w in ways:
            first.setdefault(w, size)
    return {w: s for w, s in first.items() if w not in tested}


def test_the_forward_sizes_run_all_that_heads_take(choice):
    tested = set(tc.forward_ways(choice, [(*s, n) for s in forward.SIZES for n in forward.TOPS]))
    sizes = sweep(6000, 9000, 1)
    assert not missing([{w} for w in tc.forward_ways(choice, sizes)], sizes, tested)
    for name in ("statistics 4", "alternatives 4"):
        for streamed in (False, True):
            assert {w[1] for w in tested if w[0] == name and w[2] and w[3] is streamed} == set(range(1, 9)), (name, streamed)
        assert {w[1] for w in tested if w[0] == name and not w[2]} == set(range(1, 9)), name
        assert any(w[0] == name and w[4] for w in tested)
    assert {w[1:3] for w in tested if w[0] == "statistics 8"} == {(t, s) for t in (64, 128, 256) for s in (False, True)}
    assert {w[1:3] for w in tested if w[0] == "alternatives 8"} == {(t, s) for t in (64, 128) for s in (False, True)}


def test_the_gradients_sizes_run_all_that_heads_take(choice):
    tested = set().union(*tc.gradient_ways(choice, gradients.SIZES + [(2048, 192, 140003, wide) for wide in (False, True)]))
    sizes = sweep(6000, 6000, 2)
    assert not missing(tc.gradient_ways(choice, sizes), sizes, tested)
    for low in (False, True):
        for several in (False, True):
            assert {w[2] for w in tested if w[0] == "logits 4" and w[1] is low and w[3] is several} >= set(range(2, 9)), (low, several)
    assert {w[1] for w in tested if w[0] == "dx"} == set(range(7))
    assert all(("parts of " + of, several) in tested for of in ("dx", "the vocabulary") for several in (False, True))
