"""Log probabilities of given tokens at listed rows, with entropy and alternatives, against plain 64-bit statements of the same."""
import pytest
import torch

import token_reference as ref
from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def grid(shape, gen, step, spread=16):
    """Multiples of `step`, small enough that every sum of products here is exact in 32 bits, in any order."""
    return ((torch.randn(shape, generator=gen) * spread).round().clamp(-127, 127) * step).to(BF16)


def strided(t, pad):
    full = torch.full((t.shape[0], t.shape[1] + pad), 777.0, dtype=t.dtype)
    full[:, :t.shape[1]] = t
    return full.to(DEV)[:, :t.shape[1]]


def run(hidden, w, idx, count, max_rows, targets, n_top, want=("logprob", "entropy", "lse")):
    """Outputs over poisoned buffers with room behind max_rows, which has to stay."""
    rows = max_rows + 3
    out = {k: torch.full((rows,), -7.0, device=DEV) if k in want else None for k in ("logprob", "entropy", "lse")}
    top_id = torch.full((rows, n_top), -7, dtype=torch.int32, device=DEV) if n_top else None
    top_lp = torch.full((rows, n_top), -7.0, device=DEV) if n_top else None
    T, d = hidden.shape
    ld_h = hidden.stride(0) if T > 1 else d
    need = b.mosaic_masked_logprobs_workspace_bytes(T, max_rows, d, w.shape[0], n_top, ld_h=ld_h)
    ws = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device=DEV)
    print("logprobs", tuple(hidden.shape), tuple(w.shape), max_rows, n_top, flush=True)
    b.mosaic_masked_logprobs(hidden, w, idx, count, max_rows, targets, out["logprob"], out["entropy"], out["lse"], ws[:need],
                             top_id=top_id, top_logprob=top_lp)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xAB).all())
    out = {k: v.cpu() for k, v in out.items() if v is not None}
    if n_top:
        out["top_id"], out["top_logprob"] = top_id.cpu(), top_lp.cpu()
    return out


def bounds(x, d, size):
    """How far statistics may be off, for logits x off by `off`.  A sum of d exact products in 32 bits: d units of the sum of
    magnitudes `size`, twice that for a matrix core's own order and truncation.  Exponentials are good to 2^-20 relative (the
    argument's rounding, |x - m| log2 e < 128 units, and the instruction's), their sum of V terms, added by tiles of 256 and
    in parts, to a few hundred units."""
    off = 2 * d * ref.U[F32] * size
    lse = off + 2.0 ** -15 + 2 * ref.U[F32] * x.abs().amax(dim=1)
    return off, lse


def check(got, x, targets, n_top, d, size, rows, exact_logits=False):
    logprob, entropy, lse, ids, tops = ref.logprobs(x, targets, n_top)
    off, off_lse = bounds(x, d, size)
    if exact_logits:
        off, off_lse = 0 * off, off_lse - off
    spread = (x.amax(dim=1) - x.amin(dim=1)) + 1
    assert ((got["lse"][:rows].double() - lse).abs() <= off_lse).all()
    assert ((got["logprob"][:rows].double() - logprob).abs() <= off + off_lse + 2.0 ** -20 * logprob.abs()).all()
    assert ((got["entropy"][:rows].double() - entropy).abs() <= 2 * (off + off_lse) * spread).all()
    if n_top:
        assert ((got["top_logprob"][:rows].double() - tops).abs()[tops > -float("inf")] <=
                ((off + off_lse)[:, None] + 2.0 ** -20 * tops.abs())[tops > -float("inf")]).all()
        assert torch.equal(got["top_logprob"][:rows] == -float("inf"), tops == -float("inf"))
        if exact_logits:
            assert torch.equal(got["top_id"][:rows].long(), ids)
    for k, v in got.items():
        assert bool((v[rows:] == -7).all()), k


def problem(T, d, V, M, seed, kind="grid", pad=8):
    """hidden, w, idx, targets (CPU) with M listed rows in any order, some listed twice, a few without a target."""
    gen = torch.Generator().manual_seed(seed)
    if kind == "grid":
        hidden, w = grid((T, d), gen, 1 / 8), grid((V, d), gen, 2.0 ** -(4 + (d.bit_length() + 1) // 2))
    else:
        hidden, w = torch.randn((T, d), generator=gen).to(BF16), (torch.randn((V, d), generator=gen) * 2 * d ** -0.5).to(BF16)
    idx = torch.randint(0, T, (M,), generator=gen).to(torch.int32)
    targets = torch.randint(0, V, (M,), generator=gen).to(torch.int32)
    if M > 4:
        targets[1], targets[2], targets[3], idx[4] = -1, V, 2 ** 31 - 1, idx[0]
        targets[4] = V - 1
    return strided(hidden, pad), strided(w, 8 if seed % 2 else 0), idx.to(DEV), targets.to(DEV)


SIZES = [  # T, d, V, M
    (1, 8, 1, 1), (1, 64, 5, 1), (3, 72, 255, 3), (5, 128, 256, 5), (9, 136, 257, 9), (64, 64, 300, 64), (65, 512, 1000, 65),
    (40, 1032, 8192, 37), (200, 256, 3001, 128), (129, 200, 2056, 129), (300, 64, 513, 256), (257, 320, 4096, 257),
    (700, 128, 32003, 500), (1100, 96, 1500, 1024), (5000, 64, 700, 3000), (30, 4096, 2000, 2), (16, 2048, 65536, 16),
]


@pytest.mark.parametrize("T,d,V,M", SIZES)
@pytest.mark.parametrize("n_top", [0, 1, 3, 8, 16])
def test_exact_logits(T, d, V, M, n_top):
    hidden, w, idx, targets = problem(T, d, V, M, T + d + V + n_top)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    got = run(hidden, w, idx, count, M, targets, n_top)
    rows = hidden[idx.long()]
    check(got, ref.logits(rows, w), targets, n_top, d, 0.0, M, exact_logits=True)


@pytest.mark.parametrize("T,d,V,M", SIZES)
def test_any_logits(T, d, V, M):
    hidden, w, idx, targets = problem(T, d, V, M, T + d + V, kind="any", pad=0)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    got = run(hidden, w, idx, count, M, targets, 4)
    rows = hidden[idx.long()]
    size = (rows.cpu().double().abs() @ w.cpu().double().abs().t()).amax(dim=1)
    check(got, ref.logits(rows, w), targets, 4, d, size, M)
    again = run(hidden, w, idx, count, M, targets, 4)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("M,count", [(200, 0), (200, 1), (200, 63), (200, 200), (200, 1000), (200, -4), (3000, 5), (3000, 70)])
def test_count_below_the_bound(M, count):
    hidden, w, idx, targets = problem(500, 128, 3000, M, M + count)
    n = torch.tensor([count], dtype=torch.int32, device=DEV)
    have = max(0, min(M, count))
    got = run(hidden, w, idx, n, M, targets, 5)
    rows = hidden[idx[:have].long()]
    if have:
        check(got, ref.logits(rows, w), targets[:have], 5, 128, 0.0, have, exact_logits=True)
    else:
        assert all(bool((v == -7).all()) for v in got.values())


def test_all_rows_without_a_list():
    hidden, w, _, _ = problem(333, 192, 2000, 5, 3)
    targets = torch.randint(0, 2000, (333,)).to(torch.int32).to(DEV)
    got = run(hidden, w, None, None, 333, targets, 2)
    check(got, ref.logits(hidden, w), targets, 2, 192, 0.0, 333, exact_logits=True)


def test_entries_outside_are_clamped():
    hidden, w, idx, targets = problem(50, 64, 400, 20, 8)
    idx[3], idx[5] = -9, 10 ** 6
    count = torch.tensor([20], dtype=torch.int32, device=DEV)
    got = run(hidden, w, idx, count, 20, targets, 1)
    rows = hidden[idx.long().clamp(0, 49)]
    check(got, ref.logits(rows, w), targets, 1, 64, 0.0, 20, exact_logits=True)


@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "zero rows"])
@pytest.mark.parametrize("n_top", [1, 5, 16])
def test_orders_that_candidates_have_it_hard_with(kind, n_top):
    """All logits equal, every id better than all before it, the reverse, and two values in turn: the lower id comes first."""
    d, V, T = 64, 20000, 70
    w = torch.zeros((V, d))
    v = torch.arange(V)
    w[:, 0] = {"equal": torch.ones(V), "rising": (v // 128).float(), "falling": -(v // 128).float(), "two": (v % 2).float(),
               "zero rows": (v // 128).float()}[kind]
    w[:, 1] = (v % 128).float() / 128 * (0 if kind in ("equal", "two") else 1)
    hidden = torch.zeros((T, d))
    hidden[:, 0] = hidden[:, 1] = 0.0 if kind == "zero rows" else 0.25
    hidden, w = hidden.to(BF16).to(DEV), w.to(BF16).to(DEV)
    targets = torch.randint(0, V, (T,)).to(torch.int32).to(DEV)
    got = run(hidden, w, None, None, T, targets, n_top)
    check(got, ref.logits(hidden, w), targets, n_top, d, 0.0, T, exact_logits=True)


def test_certain_and_shifted_rows():
    """One id far above the others, and logits far from zero."""
    d, V, T = 64, 3000, 40
    gen = torch.Generator().manual_seed(5)
    hidden, w = grid((T, d), gen, 1 / 8), grid((V, d), gen, 2.0 ** -7)
    w[:, 0] = 0
    w[77, 0] = 4.0
    hidden[:20, 0] = 16.0
    w[:, 1] = 8.0
    hidden[10:30, 1] = torch.tensor(-100.0)
    hidden, w = hidden.to(DEV), w.to(DEV)
    targets = torch.full((T,), 77, dtype=torch.int32, device=DEV)
    targets[5:15] = 99
    got = run(hidden, w, None, None, T, targets, 3)
    check(got, ref.logits(hidden, w), targets, 3, d, 0.0, T, exact_logits=True)
    assert bool((got["entropy"][:T] >= 0).all()) and bool((got["logprob"][:T] <= 0).all())


def test_not_a_number_stays_in_its_row():
    hidden, w, idx, targets = problem(150, 64, 5000, 130, 12)
    count = torch.tensor([130], dtype=torch.int32, device=DEV)
    want = run(hidden, w, idx, count, 130, targets, 4)
    idx[7], idx[100] = 149, 148
    idx[(idx >= 148) & (torch.arange(130, device=DEV) != 7) & (torch.arange(130, device=DEV) != 100)] = 0
    clean = run(hidden, w, idx, count, 130, targets, 4)
    hidden[149, 3], hidden[148, 5] = float("nan"), float("inf")
    got = run(hidden, w, idx, count, 130, targets, 4)
    other = torch.ones(133, dtype=torch.bool)
    other[7] = other[100] = False
    for k in got:
        assert torch.equal(got[k][other], clean[k][other])
    for row in (7, 100):
        assert got["lse"][row].isnan() and got["entropy"][row].isnan()
        assert bool(((got["top_id"][row] >= -1) & (got["top_id"][row] < 5000)).all())
    assert want["lse"][:130].isfinite().all()


@pytest.mark.parametrize("want", [("logprob",), ("entropy",), ("lse",), ()])
def test_each_output_alone(want):
    hidden, w, idx, targets = problem(90, 128, 1000, 80, 20)
    count = torch.tensor([80], dtype=torch.int32, device=DEV)
    whole = run(hidden, w, idx, count, 80, targets, 3)
    got = run(hidden, w, idx, count, 80, targets if "logprob" in want else None, 0 if want else 3, want)
    assert set(got) == set(want) or not want
    assert all(torch.equal(got[k], whole[k]) for k in got)


def test_hidden_states_past_two_gib():
    """Beyond 32-bit offsets the listed rows are gathered beforehand."""
    T, d = 600000, 2048
    hidden = torch.zeros((T, d), dtype=BF16, device=DEV)
    gen = torch.Generator().manual_seed(2)
    idx = torch.tensor([0, T - 1, 524288, 262143, 5, T - 1], dtype=torch.int32)
    rows = grid((6, d), gen, 1 / 8)
    rows[5] = rows[1]
    hidden[idx.long().to(DEV)] = rows.to(DEV)
    w = grid((700, d), gen, 2.0 ** -10).to(DEV)
    targets = torch.tensor([1, 2, 3, 4, 5, 699], dtype=torch.int32, device=DEV)
    count = torch.tensor([6], dtype=torch.int32, device=DEV)
    got = run(hidden, w, idx.to(DEV), count, 6, targets, 2)
    check(got, ref.logits(rows, w), targets, 2, d, 0.0, 6, exact_logits=True)


def test_a_vocabulary_past_four_gib():
    V, d, T = 300000, 8192, 3
    gen = torch.Generator(device=DEV).manual_seed(4)
    w = torch.zeros((V, d), dtype=BF16, device=DEV)
    ids = torch.tensor([0, 131071, 131072, 262144, V - 1], device=DEV)
    w[ids, 0] = torch.tensor([1.0, 5.0, 2.0, 4.0, 3.0], device=DEV).to(BF16)
    hidden = torch.zeros((T, d), dtype=BF16, device=DEV)
    hidden[:, 0] = torch.tensor([1.0, 2.0, -4.0], device=DEV).to(BF16)
    targets = ids[[4, 1, 0]].to(torch.int32)
    got = run(hidden, w, None, None, T, targets, 5)
    assert got["top_id"][0].tolist() == [131071, 262144, V - 1, 131072, 0]
    assert got["top_id"][2].tolist() == [1, 2, 3, 4, 5]
    x = (hidden[:, :1].double() @ w[:, :1].double().t()).cpu()
    check(got, x, targets, 5, d, 0.0, T, exact_logits=True)


def test_replayed_from_a_graph():
    hidden, w, idx, targets = problem(900, 256, 5000, 700, 31)
    count = torch.tensor([700], dtype=torch.int32, device=DEV)
    outs = [torch.zeros(700, device=DEV) for _ in range(3)]
    top_id, top_lp = torch.zeros((700, 4), dtype=torch.int32, device=DEV), torch.zeros((700, 4), device=DEV)
    ws = torch.empty(b.mosaic_masked_logprobs_workspace_bytes(900, 700, 256, 5000, 4, ld_h=hidden.stride(0)), dtype=torch.uint8, device=DEV)

    def step():
        b.mosaic_masked_logprobs(hidden, w, idx, count, 700, targets, *outs, ws, top_id=top_id, top_logprob=top_lp)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    gen = torch.Generator().manual_seed(6)
    for n in (700, 90, 300, 20):
        hidden.copy_(grid((900, 256), gen, 1 / 8))
        count.fill_(n)
        for t in (*outs, top_id, top_lp):
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        got = {"logprob": outs[0].cpu(), "entropy": outs[1].cpu(), "lse": outs[2].cpu(), "top_id": top_id.cpu(), "top_logprob": top_lp.cpu()}
        check(got, ref.logits(hidden[idx[:n].long()], w), targets[:n], 4, 256, 0.0, n, exact_logits=True)
        for t in (*outs, top_id, top_lp):
            t.fill_(-7)
        step()
        torch.cuda.synchronize()
        assert torch.equal(outs[0].cpu(), got["logprob"]) and torch.equal(top_id.cpu(), got["top_id"])
