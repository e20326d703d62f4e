"""The layer operators together, as the example uses them: a layer, the final norm of the masked rows and mask-only logits in
chunks against the same in one piece, and the layer's backward pass from 8 bits against 64-bit automatic differentiation."""
import types

import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding, example_layer

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def a_layer(d, d_ff, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return example_layer.FeedForward(d, d_ff, gen, DEV), gen


def test_chunks_change_nothing():
    """Rows are independent, so any number of chunks gives the same block output bit for bit, tokens included."""
    layer, gen = a_layer(256, 512, 3)
    x, stream = (torch.randn((300, 256), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    whole = layer.forward(x, stream.clone(), 1)
    for chunks in (2, 7, 300):
        assert ref.relative(layer.forward(x, stream.clone(), chunks), whole) <= 2e-2   # the library's down projection
    y = torch.empty_like(x)
    binding.mosaic_rmsnorm_forward(x, stream, layer.gamma, example_layer.EPS, y)
    act = torch.empty((300, 512), dtype=torch.bfloat16, device=DEV)
    binding.mosaic_gated_ffn_forward(y, layer.w_gate, layer.w_up, act)
    parts = torch.empty_like(act)
    for lo, hi in ((0, 17), (17, 130), (130, 300)):
        binding.mosaic_gated_ffn_forward(y[lo:hi], layer.w_gate, layer.w_up, parts[lo:hi])
    assert torch.equal(parts[17:], act[17:]) and ref.relative(parts[:17], act[:17]) <= ref.U_BF16


def test_serving_norms_the_masked_rows_alone():
    layer, gen = a_layer(256, 512, 5)
    args = types.SimpleNamespace(rows=512, chunks=3, vocab=1024)
    hidden, op = example_layer.serve(layer, args, gen)
    torch.cuda.synchronize()
    M = int(op.count.item())
    assert M == 64 and torch.equal(op.idx[:M].cpu(), torch.arange(448, 512, dtype=torch.int32))
    assert (hidden[:448] == 0).all() and (hidden[448:] != 0).any(dim=1).all()
    rms = hidden[448:].float().square().mean(dim=1).sqrt()
    assert (rms - 1).abs().max() <= 2 * ref.U_BF16                             # the gains are one
    assert op.lse[:M].isfinite().all() and (op.token[:M] >= 0).all()


def test_training_from_eight_bits():
    """Against automatic differentiation in 64 bits at the values that the checkpoints stand for.  The block's input is
    restored from its own checkpoint and so a constant there; each gradient passes at most three roundings to bf16 of
    2^-8 / sqrt 3 and the library's products (one more), which bounds it in the 2-norm."""
    d, d_ff, T = 192, 384, 260
    layer, gen = a_layer(d, d_ff, 7)
    x, stream, dout, dstream = (torch.randn((T, d), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(4))
    kept = [binding.Q8Rows.empty(T, d, torch.int8, 32, DEV) for _ in range(2)]
    layer.forward(x, stream, 1, keep=kept)
    dsum, grads = layer.backward(dout, dstream, kept)
    h, y = (ref.restored(k.values.cpu(), k.scales.cpu(), 32) for k in kept)
    do, wd = dout.cpu().double(), layer.w_down.cpu().double()
    dact = do @ wd
    dy, dgate, dup = ref.ffn_gradients(dact, y, layer.w_gate.cpu(), layer.w_up.cpu(), "silu")
    want, dgamma = ref.norm_gradients(dy, h, layer.gamma.cpu(), example_layer.EPS, dstream.cpu())
    act = ref.ffn(y, layer.w_gate.cpu(), layer.w_up.cpu(), "silu")
    bound = 2 * ref.U_BF16
    assert ref.relative(grads["gate"], dgate) <= bound and ref.relative(grads["up"], dup) <= bound
    assert ref.relative(grads["down"], do.t() @ act) <= bound
    assert ref.relative(dsum, want) <= bound and ref.relative(grads["gamma"], dgamma) <= bound


def test_the_command_runs():
    example_layer.main(["--rows", "300", "--train-rows", "200", "--d", "256", "--d-ff", "512", "--vocab", "2048", "--chunks", "2"])
