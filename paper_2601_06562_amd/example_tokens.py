"""Both ends of a masked-diffusion model around one layer, for training and for scoring:

    python -m paper_2601_06562_amd.example_tokens [--rows 4096] [--share 0.5]

Training: a share of the tokens is replaced by [MASK]; tokens and positions are looked up, the embeddings and the feed-forward
block's output pass through dropout onto the residual stream, the final norm sees the masked positions alone, and the loss is
made of the log probabilities of the tokens that were there.  The backward pass gives every parameter's gradient, with the dropout
masks made again from the seed.  No logits are written in either direction.  Scoring: the same pass tells how probable given tokens
are, and the two best tokens of each masked position, whose margin decides which are taken first.
Weights and tokens are random; there is no attention.  Needs an MI355X and the built library; nothing here falls back to the CPU.
"""
import argparse
import time

import torch

from . import binding, workloads
from .example_layer import EPS, FeedForward

BF16 = torch.bfloat16


class MaskedDiffusion:
    """Embeddings, one layer, the final norm and the LM head, with what a program keeps between steps."""

    def __init__(self, T, d, d_ff, V, gen, device, p=0.1):
        self.T, self.V, self.p, self.device = T, V, p, device
        self.layer = FeedForward(d, d_ff, gen, device)
        self.scale = d ** 0.5
        self.table = workloads._normal_bf16(V + 1, d, d ** -0.5, gen, device)      # the last row is [MASK]'s
        self.places = workloads._normal_bf16(T, d, 0.1, gen, device)
        self.gamma = torch.ones(d, device=device)
        self.head = workloads._normal_bf16(V, d, d ** -0.5, gen, device)
        self.rows = torch.arange(T, dtype=torch.int32, device=device)
        self.idx = torch.empty(T, dtype=torch.int32, device=device)
        self.count = torch.zeros(1, dtype=torch.int32, device=device)
        self.kept = [binding.Q8Rows.empty(T, d, torch.int8, 128, device) for _ in range(2)]
        need = max(binding.mosaic_masked_logprobs_workspace_bytes(T, T, d, V, 2),
                   binding.mosaic_masked_logprobs_backward_workspace_bytes(T, d, V),
                   binding.mosaic_embedding_backward_workspace_bytes(T, d, V + 1),
                   binding.mosaic_rmsnorm_backward_workspace_bytes(T, d), binding.mosaic_compact_scratch_bytes(T), 16)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def forward(self, tokens, mask, seed=None):
        """The final hidden states, of which only masked rows hold something; seed: of the dropouts (None: no dropout)."""
        like = dict(dtype=BF16, device=self.device)
        d, p = self.layer.d, self.p if seed is not None else 0.0
        x, stream = torch.empty((self.T, d), **like), torch.empty((self.T, d), **like)
        shown = torch.where(mask.bool(), torch.full_like(tokens, self.V), tokens)
        binding.mosaic_embedding_forward(shown, self.table, x, scale=self.scale)
        binding.mosaic_embedding_forward(self.rows, self.places, stream)
        binding.mosaic_dropout_forward(x, None, x, p, seed or 0, site=0)
        out = self.layer.forward(x, stream, keep=self.kept)
        binding.mosaic_dropout_forward(out, stream, stream, p, seed or 0, site=1)
        binding.mosaic_mask_compact(mask, self.idx, self.count, self.workspace)
        hidden = torch.zeros((self.T, d), **like)
        binding.mosaic_rmsnorm_forward(None, stream, self.gamma, EPS, hidden, idx=self.idx, count=self.count, max_rows=self.T)
        return shown, stream, hidden

    def logprobs(self, hidden, max_rows, targets, n_top=0):
        """(log probability of each listed row's target, entropy, log-sum-exp, and the n_top best ids with theirs)."""
        new = dict(device=self.device)
        own, entropy, lse = (torch.zeros(max_rows, **new) for _ in range(3))
        ids = torch.empty((max_rows, n_top), dtype=torch.int32, **new) if n_top else None
        best = torch.empty((max_rows, n_top), **new) if n_top else None
        binding.mosaic_masked_logprobs(hidden, self.head, self.idx, self.count, max_rows, targets, own, entropy, lse, self.workspace,
                                       top_id=ids, top_logprob=best)
        return own, entropy, lse, ids, best

    def train_step(self, tokens, mask, max_rows, seed):
        """(loss, gradients of every parameter, what the pass kept).  max_rows: how many masked positions there are, at most."""
        shown, stream, hidden = self.forward(tokens, mask, seed)
        targets = tokens[self.idx.long().clamp(0, self.T - 1)][:max_rows].contiguous()
        own, entropy, lse, _, _ = self.logprobs(hidden, max_rows, targets)
        dlogprob = torch.full_like(own, -1.0 / max_rows)
        like = dict(dtype=BF16, device=self.device)
        drows = torch.empty((max_rows, self.layer.d), **like)
        grads = dict(head=torch.empty_like(self.head), table=torch.empty(self.table.shape, device=self.device),
                     places=torch.empty(self.places.shape, device=self.device), final=torch.empty_like(self.gamma))
        binding.mosaic_masked_logprobs_backward(hidden, self.head, self.idx, self.count, max_rows, targets, own, None, lse, dlogprob,
                                                None, drows, grads["head"], self.workspace)
        dhidden, dstream, dout = (torch.empty((self.T, self.layer.d), **like) for _ in range(3))
        binding.mosaic_embedding_backward(drows, self.idx[:max_rows], dhidden, self.workspace, count=self.count)   # rows back to their places
        binding.mosaic_rmsnorm_backward(dhidden, stream, self.gamma, EPS, dstream, grads["final"], self.workspace)
        binding.mosaic_dropout_backward(dstream, dout, self.p, seed, site=1)
        dsum, of_layer = self.layer.backward(dout, dstream, self.kept)
        grads.update(of_layer)
        dx = torch.empty_like(dsum)
        binding.mosaic_dropout_backward(dsum, dx, self.p, seed, site=0)
        binding.mosaic_embedding_backward(dx, shown, grads["table"], self.workspace, scale=self.scale)
        binding.mosaic_embedding_backward(dsum, self.rows, grads["places"], self.workspace)
        return -own.sum() / max_rows, grads, dict(stream=stream, hidden=hidden, targets=targets, drows=drows, dsum=dsum, dx=dx)

    def score_step(self, tokens, mask, seq_starts, per_step, max_rows):
        """Unmasks the positions of each sequence whose two best tokens are furthest apart; (its log probabilities of the tokens
        given in their place, margins)."""
        _, _, hidden = self.forward(tokens, mask)
        given = tokens[self.idx.long().clamp(0, self.T - 1)][:max_rows].contiguous()
        own, _, _, ids, best = self.logprobs(hidden, max_rows, given, n_top=2)
        margin = best[:, 0].exp() - best[:, 1].exp()
        binding.mosaic_unmask_topn(margin, ids[:, 0].contiguous(), self.idx, self.count, max_rows, seq_starts, per_step, tokens, mask)
        return own, margin


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--share", type=float, default=0.5, help="of the positions that are masked")
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--d-ff", type=int, default=12288)
    ap.add_argument("--vocab", type=int, default=126464)
    args = ap.parse_args(argv)
    if not torch.cuda.is_available():
        raise SystemExit("this example needs the GPU")
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    T = args.rows
    model = MaskedDiffusion(T, args.d, args.d_ff, args.vocab, gen, dev)
    tokens = torch.randint(0, args.vocab, (T,), generator=gen, device=dev).to(torch.int32)
    mask = (torch.rand(T, generator=gen, device=dev) < args.share).to(torch.uint8)
    mask[0] = 1
    masked = int(mask.sum().item())
    for seed in range(2):                      # the first pass loads kernels
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        loss, grads, _ = model.train_step(tokens, mask, masked, seed)
        torch.cuda.synchronize()
        spent = time.perf_counter() - t0
    assert all(bool(g.isfinite().all()) for g in grads.values())
    print(f"training: {T} rows, {masked} of them masked: loss {loss.item():.3f}, forward and backward {spent * 1e3:.2f} ms")
    starts = torch.tensor([0, T // 2, T], dtype=torch.int32, device=dev)
    per_step = torch.full((2,), max(1, T // 16), dtype=torch.int32, device=dev)
    guess, left = tokens.clone(), mask.clone()
    t0 = time.perf_counter()
    own, margin = model.score_step(guess, left, starts, per_step, masked)
    torch.cuda.synchronize()
    spent = time.perf_counter() - t0
    assert bool(own.isfinite().all()) and bool((margin >= 0).all())
    print(f"scoring: mean log probability {own.mean().item():.3f}, {masked - int(left.sum().item())} positions unmasked by margin, "
          f"{spent * 1e3:.2f} ms")


if __name__ == "__main__":
    main()
