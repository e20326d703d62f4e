"""The few rows whose dg and du have low halves, on the CPU: their workspace, and the tiles that write and read them."""
import random

from paper_2601_06562_amd import binding as b
from test_ffn_choice_host import choose  # noqa: F401


def test_the_tiles_of_few_rows_write_low_halves(choose):  # noqa: F811
    """Those of 64 rows do, so every call of up to 64 rows takes one; twice 32 rows are one tile of rows for dx."""
    rng = random.Random(4)
    sizes = [(rng.randint(1, 64), 8 * rng.randint(1, 1024), 8 * rng.choice([rng.randint(1, 64), rng.randint(1, 3584)]))
             for _ in range(20000)]
    for (T, d, F), c in zip(sizes, choose(sizes)):
        assert c["recompute"][2] == 64 and c["forward"][2] == 64
    twice = choose([(2 * T, d, F) for T, d, F in sizes if T <= 32])
    for (T, d, F), c in zip([s for s in sizes if s[0] <= 32], twice):
        assert c["dx"][3] % -(-d // c["dx"][1]) == 0 and c["dw"][0] in range(7)


def test_the_workspace_holds_both_halves(choose):  # noqa: F811
    """dg | du twice, and sums of dx for the halves of every part of K."""
    rng = random.Random(5)
    sizes = [(T, 8 * rng.randint(1, 1024), 8 * rng.randint(1, 3584)) for T in range(1, 33) for _ in range(40)]
    for (T, d, F), c in zip(sizes, choose(sizes)):
        for eight in (False, True):
            need = b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, eight)
            assert need >= 8 * T * F + (2 * T * d if eight else 0) + 4 * 2 * T * c["parts"] * d


def test_more_rows_need_no_less():
    for d, F in ((8, 8), (136, 264), (4096, 12288), (16384, 8)):
        for eight in (False, True):
            need = [b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, eight) for T in range(0, 600)]
            assert need == sorted(need)
