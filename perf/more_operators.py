"""Measured cases of the operators at both ends of a masked-diffusion model: tokens into rows (embedding lookup with scaling,
dropout from a counter-based generator) and rows back onto given tokens (log probabilities at the listed rows, with entropy and
the most probable alternatives), each with its backward pass.

Fields of a case:

  op         "embedding", "embedding_backward", "dropout", "dropout_backward", "logprobs", "logprobs_backward"
  rows       positions
  d, vocab   hidden size, vocabulary size (0 where there is none)
  stream     "bf16" or "f32": type of the residual stream (the embedding's output, what dropout is added to, its gradient) or,
             for embedding_backward, of the table's gradient
  masked     logprobs: how many of the rows are listed; embedding: how many tokens are [MASK], one and the same id
  top        logprobs: alternatives a row
  entropy    logprobs_backward: whether the entropy has a gradient, too
  p          dropout: share of elements that is dropped
  pad        columns between the end of a row and the next row, in every activation
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
SITE = 3            # which of a model's dropouts the cases are


def _case(name=None, *, op, rows, d, vocab=0, stream="bf16", masked=0, top=0, entropy=False, p=0.0, pad=0):
    c = {} if name is None else {"name": name}
    c.update(op=op, rows=rows, d=d, vocab=vocab, stream=stream, masked=masked, top=top, entropy=entropy, p=p, pad=pad)
    return c


def listed():
    return [
        # A block of positions under generation: a step's input rows, where only latency counts.
        _case("embedding_block", op="embedding", rows=37, d=3584, vocab=152064, masked=20),
        # A batch of noised training sequences into a 32-bit residual stream.
        _case("embedding_batch", op="embedding", rows=32768, d=4096, vocab=126464, stream="f32", masked=16384),
        # The table's gradient in 32 bits, a small model and a ragged batch, few positions noised.
        _case("embedding_backward_small", op="embedding_backward", rows=1003, d=1024, vocab=32000, stream="f32", masked=150),
        # The table's gradient of a batch half of whose tokens are [MASK]: one row gets half of all sums.
        _case("embedding_backward_batch", op="embedding_backward", rows=32768, d=4096, vocab=126464, masked=16384),
        # Dropout of a sublayer's output, added to a 32-bit residual stream, over a batch.
        _case("dropout_batch", op="dropout", rows=32768, d=4096, stream="f32", p=0.1),
        # Its gradient for a small ragged batch with strided rows.
        _case("dropout_backward_small", op="dropout_backward", rows=1237, d=1024, p=0.2, pad=64),
        # One position scored, with the alternatives an interface shows: the LM head is read for a single row.
        _case("logprobs_token", op="logprobs", rows=1, d=4096, vocab=126464, masked=1, top=5),
        # A block of positions, by margin (best and second) and entropy.
        _case("logprobs_block", op="logprobs", rows=64, d=3584, vocab=152064, masked=37, top=2),
        # The likelihood of a small batch under a small model, without alternatives.
        _case("logprobs_small", op="logprobs", rows=2000, d=1024, vocab=32000, masked=900),
        # The masked half of a context, scored with alternatives.
        _case("logprobs_batch", op="logprobs", rows=8192, d=4096, vocab=126464, masked=4105, top=8),
        # The training loss's gradient for a small model, with an entropy term.
        _case("logprobs_backward_small", op="logprobs_backward", rows=1237, d=512, vocab=8192, masked=500, entropy=True),
        # The same for a full LM head, tokens weighted by 1 / t as a masked-diffusion loss weights them.
        _case("logprobs_backward_batch", op="logprobs_backward", rows=4096, d=4096, vocab=126464, masked=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(512, 8192), (1024, 32000), (1032, 32003), (704, 50257), (2048, 65536), (4096, 126464), (3584, 152064)]


def draw(rng):
    op = rng.choice(["embedding", "embedding_backward", "dropout", "dropout_backward", "logprobs", "logprobs", "logprobs",
                     "logprobs_backward", "logprobs_backward"])
    d, vocab = rng.choice(HEADS)
    stream, pad = rng.choice(["bf16", "f32"]), rng.choice([0, 0, 8, 64])
    if op.startswith("dropout"):
        return _case(op=op, rows=_log_int(rng, 1, 30000), d=d, stream=stream, p=rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]), pad=pad)
    if op.startswith("embedding"):
        rows = _log_int(rng, 1, 30000)
        return _case(op=op, rows=rows, d=d, vocab=vocab, stream=stream, masked=int(rows * rng.choice([0.0, 0.15, 0.5, 0.9])), pad=pad)
    masked = _log_int(rng, 1, 3400 if op == "logprobs" else 1700)
    rows = max(masked, int(masked / rng.choice([0.05, 0.3, 0.8, 1.0])))
    return _case(op=op, rows=rows, d=d, vocab=vocab, masked=masked, pad=pad,
                 top=rng.choice([0, 1, 2, 3, 5, 8, 16]) if op == "logprobs" else 0,
                 entropy=op == "logprobs_backward" and rng.random() < 0.4)


class _State:
    pass


def _log2_side(d):
    return math.ceil(math.log2(d) / 2)


def _head(vocab, d, gen):
    """LM-head weights of about N(0, 1/d) on a grid, as 8-bit weights restored with one scale lie on one."""
    w = torch.empty((vocab, d), dtype=torch.bfloat16, device=DEVICE)
    for r in range(0, vocab, 16384):
        n = min(vocab, r + 16384) - r
        w[r:r + n] = (torch.randn((n, d), generator=gen, device=DEVICE) * 16).round().clamp(-127, 127) * 2.0 ** -(4 + _log2_side(d))
    return w


def prepare(case, seed):
    """Inputs on the GPU.

    Tokens: ranks by a law that a text's words follow (the logarithm of an id is uniform), shuffled ids, one in a hundred
    none at all (-1, a padding position), and `masked` times the last id, which stands for [MASK].

    Hidden rows of the log probabilities: noise plus a multiple of some id's weights, between none and enough to make that
    id certain; for half of the rows it is the target.  They and the weights lie on grids, as 8-bit ones restored with one
    scale do: every product and every sum is then exact in 32 bits, so which ids come first does not hang on the order of
    a sum, and where two logits are equal the lower id comes first.  One row in fifty has no target (-1)."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = _State()
    s.case, s.op, s.workspace = case, case["op"], None
    T, d, V, pad = case["rows"], case["d"], case["vocab"], case["pad"]
    stream = torch.float32 if case["stream"] == "f32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=DEVICE)

    def blank(rows, cols, dtype=torch.bfloat16):
        return torch.zeros((rows, cols + pad), dtype=dtype, device=DEVICE)[:, :cols]

    def matrix(rows, cols, dtype=torch.bfloat16, by=1.0):
        out = blank(rows, cols, dtype)
        for r in range(0, rows, 16384):
            n = min(rows, r + 16384) - r
            out[r:r + n] = normal(n, cols) * by
        return out

    if s.op.startswith("embedding"):
        ids = torch.randperm(V - 1, generator=gen, device=DEVICE)
        rank = torch.exp(uniform(T) * math.log(V - 1)).long() - 1
        s.tokens = ids[rank.clamp(0, V - 2)].to(torch.int32)
        s.tokens[uniform(T) < 0.01] = -1
        s.tokens[torch.randperm(T, generator=gen, device=DEVICE)[:case["masked"]]] = V - 1
        s.scale = math.sqrt(d)
        if s.op == "embedding":
            s.table = torch.empty((V, d), dtype=torch.bfloat16, device=DEVICE)
            for r in range(0, V, 16384):
                n = min(V, r + 16384) - r
                s.table[r:r + n] = normal(n, d) * d ** -0.5
            s.out = blank(T, d, stream)
        else:
            s.dout = matrix(T, d, by=1e-3)
            s.dtable = torch.zeros((V, d), dtype=stream, device=DEVICE)
        return s
    if s.op.startswith("dropout"):
        s.key = (int(seed) * 0x9E3779B97F4A7C15 + 1) % (1 << 64)
        s.first_row = 1 << 20
        if s.op == "dropout":
            s.x, s.residual = matrix(T, d), matrix(T, d, stream)
            s.out = blank(T, d, stream)
        else:
            s.dout, s.dx = matrix(T, d, stream, by=1e-3), blank(T, d)
        return s

    M = case["masked"]
    s.w = _head(V, d, gen)
    s.idx = torch.randperm(T, generator=gen, device=DEVICE)[:M].sort().values.to(torch.int32)
    s.count = torch.tensor([M], dtype=torch.int32, device=DEVICE)
    s.targets = torch.randint(0, V, (M,), generator=gen, device=DEVICE, dtype=torch.int32)
    toward = torch.where(uniform(M) < 0.5, s.targets, torch.randint(0, V, (M,), generator=gen, device=DEVICE, dtype=torch.int32))
    s.targets[torch.arange(M, device=DEVICE) % 50 == 49] = -1
    s.hidden = blank(T, d)
    for r in range(0, T, 16384):
        n = min(T, r + 16384) - r
        s.hidden[r:r + n] = (normal(n, d) * 24).round().clamp(-127, 127) / 16
    size = 2.0 ** _log2_side(d)
    lean = uniform(M, 1) * (16.0 / math.sqrt(d)) * size
    rows = s.hidden[s.idx.long()].float() + lean * s.w[toward.long()].float()
    s.hidden[s.idx.long()] = ((rows * 16).round().clamp(-127, 127) / 16).to(torch.bfloat16)
    if s.op == "logprobs":
        s.logprob, s.entropy, s.lse = (torch.zeros(M, device=DEVICE) for _ in range(3))
        s.top_id = s.top_logprob = None
        if case["top"]:
            s.top_id = torch.zeros((M, case["top"]), dtype=torch.int32, device=DEVICE)
            s.top_logprob = torch.zeros((M, case["top"]), device=DEVICE)
        return s
    # what the forward pass kept, and the loss's gradient: the mean over the rows of log p / t, t in (0.05, 1]
    s.dlogprob = -1.0 / M / (0.05 + 0.95 * uniform(M))
    s.dentropy = -0.01 / M * torch.ones(M, device=DEVICE) if case["entropy"] else None
    s.logprob, s.entropy, s.lse = (torch.zeros(M, device=DEVICE) for _ in range(3))
    for r in range(0, M, 2048):
        x = s.hidden[s.idx[r:r + 2048].long()].float() @ s.w.float().t()
        t = s.targets[r:r + 2048].long()
        s.lse[r:r + 2048] = torch.logsumexp(x, dim=1)
        x -= s.lse[r:r + 2048, None]
        s.logprob[r:r + 2048] = torch.where(t >= 0, x.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0)
        s.entropy[r:r + 2048] = -(x.exp() * x).sum(dim=1)
    s.dx = blank(M, d)
    s.dw = torch.zeros_like(s.w)
    return s


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end

def _embedding_plain(s):
    t = s.tokens.long()
    there = (t >= 0) & (t < s.case["vocab"])
    rows = s.table[t.clamp(0, s.case["vocab"] - 1)].float() * s.scale
    s.out.copy_(torch.where(there[:, None], rows, 0.0))
    return {"out": s.out}


def _embedding_backward_plain(s):
    t = s.tokens.long()
    there = (t >= 0) & (t < s.case["vocab"])
    total = torch.zeros((s.case["vocab"], s.case["d"]), device=DEVICE)
    total.index_add_(0, t[there], s.dout[there].float())
    s.dtable.copy_(total * s.scale)
    return {"dtable": s.dtable}


def _kept_plain(s, rows, d):
    """(which elements are kept, by how much they grow).  Eight columns of a row share one block of Philox4x32-10 with the
    key s.key and the counter (column / 8, low and high half of the row's number, SITE + 1); column c has the low (c even) or
    high 16 bits of word c / 2 % 4 and is dropped where they are below p 2^16, rounded."""
    low = 0xFFFFFFFF
    groups = -(-d // 8)
    row = torch.arange(rows, device=DEVICE)[:, None] + s.first_row
    c0 = torch.arange(groups, device=DEVICE).expand(rows, groups)
    c1, c2 = (row & low).expand(rows, groups), (row >> 32).expand(rows, groups)
    c3 = torch.full_like(c0, SITE + 1)
    k0, k1 = s.key & low, s.key >> 32

    def product(m, x):   # high and low 32 bits, in numbers that stay below 2^63
        upper = m * (x >> 16) + ((m * (x & 0xFFFF)) >> 16)
        return upper >> 16, ((upper & 0xFFFF) << 16) | ((m * (x & 0xFFFF)) & 0xFFFF)

    for _ in range(10):
        hi0, lo0 = product(0xD2511F53, c0)
        hi1, lo1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = hi1 ^ c1 ^ k0, lo1, hi0 ^ c3 ^ k1, lo0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], dim=2)
    border = round(s.case["p"] * 65536)
    return words.view(rows, groups * 8)[:, :d] >= border, 65536.0 / (65536 - border)


def _dropout_plain(s):
    kept, grow = _kept_plain(s, s.case["rows"], s.case["d"])
    s.out.copy_(torch.where(kept, s.x.float() * grow, 0.0) + s.residual.float())
    return {"out": s.out}


def _dropout_backward_plain(s):
    kept, grow = _kept_plain(s, s.case["rows"], s.case["d"])
    s.dx.copy_(torch.where(kept, s.dout.float() * grow, 0.0))
    return {"dx": s.dx}


def _logprobs_plain(s):
    x = s.hidden[s.idx.long()].float() @ s.w.float().t()
    lse = torch.logsumexp(x, dim=1)
    p = x - lse[:, None]
    t = s.targets.long()
    out = {"logprob": torch.where(t >= 0, p.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0),
           "entropy": -(p.exp() * p).sum(dim=1), "lse": lse}
    if s.case["top"]:
        # by logit, then by id: 32-bit numbers in the order of integers, the id counted down in the low half
        del p
        bits = x.view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -0x80000000 - bits)
        del bits
        order = (order << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=DEVICE))
        best = order.topk(s.case["top"], dim=1).values
        ids = 0xFFFFFFFF - (best & 0xFFFFFFFF)
        out["top_id"] = ids.to(torch.int32)
        out["top_logprob"] = x.gather(1, ids) - lse[:, None]
    return out


def _logprobs_backward_plain(s):
    rows = s.hidden[s.idx.long()].float()
    w = s.w.float()
    logp = rows @ w.t() - s.lse[:, None]
    t = s.targets.long()
    g = torch.where(t >= 0, s.dlogprob, 0.0)
    if s.dentropy is None:
        dl = logp.exp() * -g[:, None]
    else:
        dl = logp.exp() * -(g[:, None] + s.dentropy[:, None] * (logp + s.entropy[:, None]))
    del logp
    dl.scatter_add_(1, t.clamp_min(0)[:, None], g[:, None])
    s.dx.copy_(dl @ w)
    s.dw.copy_(dl.t() @ rows)
    return {"dx": s.dx, "dw": s.dw}


# ---- the framework's operators, as a user calls them

def _workspace(s, need):
    if s.workspace is None:
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE)
    return s.workspace


def _run_own(s):
    from paper_2601_06562_amd import binding as b
    c = s.case
    if s.op == "embedding":
        b.mosaic_embedding_forward(s.tokens, s.table, s.out, scale=s.scale)
        return {"out": s.out}
    if s.op == "embedding_backward":
        if s.workspace is None:
            _workspace(s, b.mosaic_embedding_backward_workspace_bytes(c["rows"], c["d"], c["vocab"]))
        b.mosaic_embedding_backward(s.dout, s.tokens, s.dtable, s.workspace, scale=s.scale)
        return {"dtable": s.dtable}
    if s.op == "dropout":
        b.mosaic_dropout_forward(s.x, s.residual, s.out, c["p"], s.key, site=SITE, first_row=s.first_row)
        return {"out": s.out}
    if s.op == "dropout_backward":
        b.mosaic_dropout_backward(s.dout, s.dx, c["p"], s.key, site=SITE, first_row=s.first_row)
        return {"dx": s.dx}
    if s.op == "logprobs":
        if s.workspace is None:
            _workspace(s, b.mosaic_masked_logprobs_workspace_bytes(c["rows"], c["masked"], c["d"], c["vocab"], c["top"],
                                                                   ld_h=c["d"] + c["pad"]))
        b.mosaic_masked_logprobs(s.hidden, s.w, s.idx, s.count, c["masked"], s.targets, s.logprob, s.entropy, s.lse,
                                 s.workspace, top_id=s.top_id, top_logprob=s.top_logprob)
        out = {"logprob": s.logprob, "entropy": s.entropy, "lse": s.lse}
        if c["top"]:
            out.update(top_id=s.top_id, top_logprob=s.top_logprob)
        return out
    if s.workspace is None:
        _workspace(s, b.mosaic_masked_logprobs_backward_workspace_bytes(c["masked"], c["d"], c["vocab"]))
    b.mosaic_masked_logprobs_backward(s.hidden, s.w, s.idx, s.count, c["masked"], s.targets, s.logprob, s.entropy, s.lse,
                                      s.dlogprob, s.dentropy, s.dx, s.dw, s.workspace)
    return {"dx": s.dx, "dw": s.dw}


def run(s):
    if own:
        return _run_own(s)
    if s.op == "embedding":
        return _embedding_plain(s)
    if s.op == "embedding_backward":
        return _embedding_backward_plain(s)
    if s.op == "dropout":
        return _dropout_plain(s)
    if s.op == "dropout_backward":
        return _dropout_backward_plain(s)
    return _logprobs_plain(s) if s.op == "logprobs" else _logprobs_backward_plain(s)


def work(case):
    """Each input read once, each output written once (of a table only the rows that tokens name, each once a position)."""
    T, d, V, M = case["rows"], case["d"], case["vocab"], case["masked"]
    st = 4 if case["stream"] == "f32" else 2
    if case["op"] == "embedding":
        distinct = min(T, T - M + 1)      # [MASK]'s row once
        return {"bytes": 4.0 * T + 2.0 * distinct * d + st * T * d, "flops": 1.0 * T * d}
    if case["op"] == "embedding_backward":
        return {"bytes": 4.0 * T + 2.0 * T * d + st * V * d, "flops": 2.0 * T * d}
    if case["op"] == "dropout":
        return {"bytes": T * d * (2.0 + st + st), "flops": 3.0 * T * d}
    if case["op"] == "dropout_backward":
        return {"bytes": T * d * (2.0 + st), "flops": 2.0 * T * d}
    if case["op"] == "logprobs":
        return {"bytes": 2.0 * (V + M) * d + M * (20.0 + 8.0 * case["top"]), "flops": 2.0 * M * V * d}
    return {"bytes": 2.0 * (2 * V + 2 * M) * d + 28.0 * M, "flops": 6.0 * M * V * d}


# ---- the definitions in 64 bits, for the comparison alone

def _exact_kept(s, rows, d):
    """As _kept_plain, in unsigned 64-bit numbers on the host."""
    u = np.uint64
    low = u(0xFFFFFFFF)
    n = (d + 7) // 8
    c = [np.tile(np.arange(n, dtype=u), rows), np.repeat((np.arange(rows, dtype=u) + u(s.first_row)) & low, n),
         np.repeat((np.arange(rows, dtype=u) + u(s.first_row)) >> u(32), n), np.full(rows * n, SITE + 1, dtype=u)]
    for r in range(10):
        key = [u(((s.key & 0xFFFFFFFF) + r * 0x9E3779B9) % (1 << 32)), u(((s.key >> 32) + r * 0xBB67AE85) % (1 << 32))]
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ key[0], b & low, (a >> u(32)) ^ c[3] ^ key[1], a & low]
    border = int(math.floor(s.case["p"] * 65536 + 0.5))
    kept = np.empty((rows * n, 8), dtype=bool)
    for k in range(4):
        kept[:, 2 * k] = (c[k] & u(0xFFFF)) >= u(border)
        kept[:, 2 * k + 1] = (c[k] >> u(16)) >= u(border)
    kept = torch.from_numpy(kept.reshape(rows, n * 8)[:, :d].copy()).to(DEVICE)
    return kept.double() * (65536 / (65536 - border))


def exact(case, seed):
    s = prepare(case, seed)
    T, d, V = case["rows"], case["d"], case["vocab"]
    if s.op == "embedding":
        t = s.tokens.long()
        out = torch.zeros((T, d), dtype=torch.float64, device=DEVICE)
        at = ((t >= 0) & (t < V)).nonzero()[:, 0]
        out[at] = s.table.index_select(0, t[at]).double() * s.scale
        return {"out": out}
    if s.op == "embedding_backward":
        t = s.tokens.long()
        at = ((t >= 0) & (t < V)).nonzero()[:, 0]
        return {"dtable": torch.zeros((V, d), dtype=torch.float64, device=DEVICE).index_add(0, t[at], s.dout[at].double() * s.scale)}
    if s.op == "dropout":
        return {"out": s.residual.double() + s.x.double() * _exact_kept(s, T, d)}
    if s.op == "dropout_backward":
        return {"dx": s.dout.double() * _exact_kept(s, T, d)}
    rows = s.hidden.index_select(0, s.idx.long()).double()
    w = s.w.double()
    x = torch.mm(rows, w.t().contiguous())
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    has = s.targets >= 0
    at = s.targets.long() * has
    own_logit = (rows * w.index_select(0, at)).sum(dim=1)
    if s.op == "logprobs":
        gap = (top - x).mul_(e)
        out = {"logprob": (own_logit - lse) * has, "entropy": (torch.log(total) + gap.sum(dim=1, keepdim=True) / total)[:, 0],
               "lse": lse}
        if case["top"]:
            out["top_id"] = None
            out["top_logprob"] = torch.sort(x.topk(case["top"], dim=1).values, dim=1, descending=True).values - lse[:, None]
        return out
    g = s.dlogprob.double() * has
    p = e.div_(total)
    if s.dentropy is None:
        dl = p * -g[:, None]
    else:
        logp = x - lse[:, None]
        entropy = -(p * logp).sum(dim=1, keepdim=True)
        dl = -p * (g[:, None] + s.dentropy.double()[:, None] * (logp + entropy))
    del x, p, e
    dl[torch.arange(dl.shape[0], device=DEVICE), at] += g
    return {"dx": torch.mm(dl, w), "dw": torch.mm(dl.t().contiguous(), rows)}
