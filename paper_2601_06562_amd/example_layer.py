"""The last layer of a denoising step and the mask-only logits behind it, then the layer's backward pass:

    python -m paper_2601_06562_amd.example_layer [--rows 4096] [--chunks 4] [--train-rows 4096]

Serving: the attention's output is added to the residual stream and normed, the feed-forward block runs over all positions in
chunks of rows (so that its activations never exceed a chunk), and the final norm and the LM head see the masked positions
alone, by the list that compaction makes.  Training: the forward pass keeps the layer's sum and the block's input in 8 bits;
the backward pass computes both projections again from there.  Weights and inputs are random; the down projection is a
plain library product.  Needs an MI355X and the built library; nothing here falls back to the CPU.
"""
import argparse
import time

import torch

from . import binding, workloads

EPS = 1e-5


class FeedForward:
    """One layer's norm and gated feed-forward block, with the workspaces a program keeps."""

    def __init__(self, d, d_ff, gen, device):
        def weight(rows, cols):
            return workloads._normal_bf16(rows, cols, cols ** -0.5, gen, device)
        self.d, self.d_ff, self.device = d, d_ff, device
        self.gamma = torch.ones(d, device=device)
        self.w_gate, self.w_up, self.w_down = weight(d_ff, d), weight(d_ff, d), weight(d, d_ff)

    def forward(self, x, stream, chunks=1, keep=None):
        """x + stream into `stream`, then the block's output; `keep`: two Q8Rows for the sum and the block's input."""
        T = x.shape[0]
        y = torch.empty_like(x)
        binding.mosaic_rmsnorm_forward(x, stream, self.gamma, EPS, y, sum=stream, q8=keep[1] if keep else None)
        if keep:
            binding.mosaic_checkpoint_store(stream, keep[0])
        out = torch.empty_like(x)
        rows = -(-T // chunks)
        act = torch.empty((min(rows, T), self.d_ff), dtype=torch.bfloat16, device=self.device)
        for t in range(0, T, rows):
            n = min(rows, T - t)
            binding.mosaic_gated_ffn_forward(y[t:t + n], self.w_gate, self.w_up, act[:n])
            torch.matmul(act[:n], self.w_down.t(), out=out[t:t + n])
        return out

    def backward(self, dout, dstream, kept):
        """Gradients from those of the block's output and of the residual stream behind it: (dstream at the layer's
        input, a dict of the weights')."""
        T = dout.shape[0]
        dact = torch.matmul(dout, self.w_down)
        act, dy = torch.empty_like(dact), torch.empty_like(dout)
        dw = torch.empty((2 * self.d_ff, self.d), dtype=torch.bfloat16, device=self.device)
        need = max(binding.mosaic_gated_ffn_backward_workspace_bytes(T, self.d, self.d_ff, q8_input=True),
                   binding.mosaic_rmsnorm_backward_workspace_bytes(T, self.d), 16)
        workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        binding.mosaic_gated_ffn_backward(dact, kept[1], self.w_gate, self.w_up, dy, dw[:self.d_ff], dw[self.d_ff:],
                                          workspace, out=act)
        dgamma = torch.empty_like(self.gamma)
        dsum = torch.empty_like(dstream)
        binding.mosaic_rmsnorm_backward(dy, kept[0], self.gamma, EPS, dsum, dgamma, workspace, dsum_in=dstream)
        return dsum, dict(gate=dw[:self.d_ff], up=dw[self.d_ff:], down=torch.matmul(dout.t(), act), gamma=dgamma)


def serve(layer, args, gen):
    T, dev = args.rows, layer.device
    head = workloads._normal_bf16(args.vocab, layer.d, layer.d ** -0.5, gen, dev)
    x, stream = (workloads._normal_bf16(T, layer.d, 1.0, gen, dev) for _ in range(2))
    mask = torch.zeros(T, dtype=torch.uint8, device=dev)
    mask[T - max(1, T // 8):] = 1
    op = binding.MaskOnlyLogits(T, layer.d, args.vocab, max_rows=max(1, T // 8), device=dev)
    hidden = torch.zeros_like(x)
    gamma = torch.ones(layer.d, device=dev)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    out = layer.forward(x, stream, args.chunks)
    binding.mosaic_mask_compact(mask, op.idx, op.count, op.scratch)
    binding.mosaic_rmsnorm_forward(out, stream, gamma, EPS, hidden, idx=op.idx, count=op.count, max_rows=op.max_rows)
    binding.mosaic_masked_logits_reduce(hidden, head, op.idx, op.count, op.max_rows, op.token, op.conf, op.lse, op.plan,
                                        op.workspace)
    torch.cuda.synchronize()
    print(f"serving: {T} rows, {op.max_rows} of them masked, in {args.chunks} chunks: {(time.perf_counter() - t0) * 1e3:.2f} ms; "
          f"activations of a chunk {2 * -(-T // args.chunks) * layer.d_ff / 1e6:.1f} MB (both projections of all rows "
          f"would be {4 * T * layer.d_ff / 1e6:.1f} MB)")
    return hidden, op


def train(layer, args, gen):
    T, dev = args.train_rows, layer.device
    x, stream, dout, dstream = (workloads._normal_bf16(T, layer.d, s, gen, dev) for s in (1.0, 1.0, 1e-3, 1e-3))
    kept = [binding.Q8Rows.empty(T, layer.d, torch.int8, 128, dev) for _ in range(2)]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    layer.forward(x, stream, 1, keep=kept)
    dsum, grads = layer.backward(dout, dstream, kept)
    torch.cuda.synchronize()
    eight = sum(k.values.numel() + 4 * k.scales.numel() for k in kept)
    print(f"training: {T} rows forward and backward: {(time.perf_counter() - t0) * 1e3:.2f} ms; kept between them "
          f"{eight / 1e6:.1f} MB (sum, input, both projections and their product in 16 bits: "
          f"{2 * T * (2 * layer.d + 3 * layer.d_ff) / 1e6:.1f} MB)")
    return dsum, grads


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--chunks", type=int, default=4, help="chunks of rows the feed-forward block runs in")
    ap.add_argument("--train-rows", type=int, default=4096)
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--d-ff", type=int, default=12288)
    ap.add_argument("--vocab", type=int, default=126464)
    args = ap.parse_args(argv)
    if not torch.cuda.is_available():
        raise SystemExit("this example needs the GPU")
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    layer = FeedForward(args.d, args.d_ff, gen, dev)
    for _ in range(2):                      # the first pass loads kernels
        hidden, op = serve(layer, args, gen)
        dsum, grads = train(layer, args, gen)
    assert bool(op.lse[:int(op.count.item())].isfinite().all()) and bool(dsum.isfinite().all())
    assert all(bool(g.isfinite().all()) for g in grads.values())


if __name__ == "__main__":
    main()
