"""A batch of rows taken in chunks: every chunk's rows are within the elementwise bound of the 64-bit statement, whichever kernel
its number of rows leads to.  The block's last bits may differ with the number of rows; the norm's and the checkpoints' do not."""
import pytest
import torch

import layer_reference as ref
from paper_2601_06562_amd import binding as b, example_layer
from test_gpu_layer_ffn import ACT, DEV, generator, inputs, matrix

pytestmark = pytest.mark.gpu
CUTS = {   # of 300 rows: the kernel for few rows (1 to 64 rows), one tile of rows, several
    "few": [1, 16, 17, 33, 64, 97, 130, 161, 194, 210, 240, 257, 299],
    "one_tile": [65, 131, 200, 265],
    "halves": [150],
    "uneven": [3, 203],
}


def pieces(name):
    ends = [0] + CUTS[name] + [300]
    return list(zip(ends[:-1], ends[1:]))


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("d,F,act", [(256, 512, "silu"), (200, 1288, "gelu"), (136, 18952, "silu")])
def test_the_block(cut, d, F, act):
    gen, x, wg, wu = inputs(300, d, F, d + F, 8)
    out, full = matrix(300, F, gen, 8)
    for lo, hi in pieces(cut):
        b.mosaic_gated_ffn_forward(x[lo:hi], wg, wu, out[lo:hi], activation=ACT[act])
    exact, bound = ref.ffn_bound(x, wg, wu, act)
    assert ((out.double() - exact).abs() <= bound).all() and (full[:, F:] == 777.0).all()
    again = torch.empty_like(out)
    for lo, hi in pieces(cut):
        b.mosaic_gated_ffn_forward(x[lo:hi], wg, wu, again[lo:hi], activation=ACT[act])
    assert torch.equal(again, out)                                             # the same chunks, the same bits


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("d", [256, 1032])
def test_norms_and_checkpoints_have_the_bits_of_the_whole(cut, d):
    gen = generator(d)
    x, r, dy = (matrix(300, d, gen, 8)[0] for _ in range(3))
    gamma = torch.rand(d, generator=gen).to(DEV)

    def run(spans):
        y, total, dsum = (torch.empty((300, d), dtype=torch.bfloat16, device=DEV) for _ in range(3))
        kept = [b.Q8Rows.empty(300, d, torch.int8, 64, DEV) for _ in range(2)]
        work = torch.empty(b.mosaic_rmsnorm_backward_workspace_bytes(300, d), dtype=torch.uint8, device=DEV)
        for lo, hi in spans:
            one, two = (b.Q8Rows(k.values[lo:hi], k.scales[lo:hi], 64) for k in kept)
            b.mosaic_rmsnorm_forward(x[lo:hi], r[lo:hi], gamma, 1e-5, y[lo:hi], sum=total[lo:hi], q8=one)
            b.mosaic_checkpoint_store(total[lo:hi], two)
            b.mosaic_rmsnorm_backward(dy[lo:hi], total[lo:hi], gamma, 1e-5, dsum[lo:hi], None, work)
        return [y, total, dsum] + [t for k in kept for t in (k.values, k.scales)]

    for got, want in zip(run(pieces(cut)), run([(0, 300)])):
        assert torch.equal(got, want)


def test_the_example_in_chunks():
    """The example's layer: the block within its bound of the normed rows it is given, the down projection a library product,
    whose sums of F products of bf16 numbers are held in 32 bits and rounded once."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    layer = example_layer.FeedForward(256, 512, gen, torch.device(DEV))
    x, stream = (torch.randn((300, 256), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    y = torch.empty_like(x)
    b.mosaic_rmsnorm_forward(x, stream, layer.gamma, example_layer.EPS, y)
    exact, bound = ref.ffn_bound(y, layer.w_gate, layer.w_up, "silu")
    down = layer.w_down.double()
    want = exact @ down.t()
    off = bound @ down.abs().t() + 2 * 512 * ref.U_F32 * ((exact.abs() + bound) @ down.abs().t())
    for chunks in (1, 2, 3, 7, 30, 300):
        out = layer.forward(x, stream.clone(), chunks)
        assert ((out.double() - want).abs() <= off + ref.U_BF16 * (want.abs() + off) + 1e-38).all()
