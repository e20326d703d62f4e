"""Plain 64-bit statements of the token operators (embedding lookup, dropout, log probabilities of given tokens), on the CPU,
and the units that the tests' bounds count.  Nothing here uses the library."""
import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # relative error of one rounding


def embedding(tokens, table, scale, count=None, before=None):
    """Rows of the table; `before`: what the output held, which stays from `count` on."""
    V = table.shape[0]
    t = tokens.cpu().long()
    there = (t >= 0) & (t < V)
    out = torch.zeros((t.numel(), table.shape[1]), dtype=torch.float64)
    out[there] = table.cpu().double()[t[there]] * scale
    if count is not None:
        out[count:] = before.cpu().double()[count:]
    return out


def embedding_gradient(dout, tokens, V, scale, count=None):
    """(the gradient, the sum of magnitudes, how many rows each token has)."""
    t = tokens.cpu().long()
    there = (t >= 0) & (t < V)
    if count is not None:
        there[count:] = False
    g = dout.cpu().double()[there] * scale
    zero = torch.zeros((V, dout.shape[1]), dtype=torch.float64)
    return (zero.index_add(0, t[there], g), zero.index_add(0, t[there], g.abs()), torch.bincount(t[there], minlength=V))


def philox(counter, key):
    """Philox4x32-10 on arrays of four counter words (uint64 holding 32 bits) and two key words."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=u) for x in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    return c


def kept(T, d, p, seed, site=0, first_row=0):
    """(mask of kept elements [T, d], factor)."""
    groups = (d + 7) // 8
    row = np.repeat(np.array([first_row + t for t in range(T)], dtype=np.uint64), groups)
    words = philox([np.tile(np.arange(groups, dtype=np.uint64), T), row & np.uint64(0xFFFFFFFF), row >> np.uint64(32),
                    np.full(T * groups, site + 1, dtype=np.uint64)], (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.empty((T * groups, 8), dtype=np.int64)
    for w in range(4):
        bits[:, 2 * w] = (words[w] & np.uint64(0xFFFF)).astype(np.int64)
        bits[:, 2 * w + 1] = (words[w] >> np.uint64(16)).astype(np.int64)
    border = int(np.rint(np.float64(np.float32(p)) * 65536))
    return torch.from_numpy(bits.reshape(T, groups * 8)[:, :d] >= border), 65536.0 / (65536 - border)


def logits(rows, w):
    return rows.cpu().double() @ w.cpu().double().t()


def logprobs(x, targets, n_top=0):
    """(logprob of the targets, 0 where there is none; entropy; log-sum-exp; ids and log probabilities of the n_top largest,
    the lower id first among equals, -1 and -inf past the vocabulary) of logits x in 64 bits."""
    lse = torch.logsumexp(x, dim=1)
    logp = x - lse[:, None]
    t = targets.cpu().long()
    has = (t >= 0) & (t < x.shape[1])
    own = logp.gather(1, torch.where(has, t, 0)[:, None])[:, 0]
    entropy = -torch.where(logp.exp() > 0, logp.exp() * logp, 0.0).sum(dim=1)
    n = min(n_top, x.shape[1])
    order = torch.sort(-x, dim=1, stable=True).indices[:, :n]
    ids = torch.full((x.shape[0], n_top), -1, dtype=torch.int64)
    tops = torch.full((x.shape[0], n_top), -float("inf"), dtype=torch.float64)
    ids[:, :n], tops[:, :n] = order, logp.gather(1, order)
    return torch.where(has, own, 0.0), entropy, lse, ids, tops


def logprob_gradients(rows, w, targets, dlogprob, dentropy=None):
    """(gradient at the rows, at w) by automatic differentiation of `logprobs`."""
    rows, w = (t.cpu().double().clone().requires_grad_(True) for t in (rows, w))
    logprob, entropy, _, _, _ = logprobs(rows @ w.t(), targets)
    loss = (logprob * dlogprob.cpu().double()).sum()
    if dentropy is not None:
        loss = loss + (entropy * dentropy.cpu().double()).sum()
    loss.backward()
    return rows.grad, w.grad


def relative(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    norm = want.norm().item()
    return (got - want).norm().item() / norm if norm else (got - want).norm().item()
