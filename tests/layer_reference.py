"""Plain 64-bit statements of the layer operators (norm, 8-bit rows, gated feed-forward block), on the CPU, and the bounds
that the tests hold the kernels to.  Nothing here uses the library."""
import math

import torch

U_BF16 = 2.0 ** -8      # relative error of one rounding to bf16 (8 significant bits)
U_F32 = 2.0 ** -24
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def norm(h, gamma, eps):
    h, gamma = h.double(), gamma.double()
    return h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps) * gamma


def norm_gradients(dy, h, gamma, eps, dsum_in=None):
    """(dsum, dgamma) by automatic differentiation of `norm`."""
    h = h.double().clone().requires_grad_(True)
    gamma = gamma.double().clone().requires_grad_(True)
    norm(h, gamma, eps).backward(dy.double())
    return h.grad if dsum_in is None else h.grad + dsum_in.double(), gamma.grad


def group_scales(v, dtype, group):
    T, d = v.shape
    n = -(-d // group)
    wide = torch.zeros((T, n * group), dtype=torch.float64)
    wide[:, :d] = v.double()
    return wide.view(T, n, group).abs().amax(dim=2) / TOP[dtype]


def widen(scales, group, d):
    return scales.double().repeat_interleave(group, dim=1)[:, :d]


def restored(values, scales, group):
    """The bf16 numbers that 8-bit values stand for: one product in 32 bits, rounded."""
    return (values.float() * widen(scales.float(), group, values.shape[1]).float()).to(torch.bfloat16)


def activation(g, kind):
    if kind == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))


def ffn(x, w_gate, w_up, kind):
    x, wg, wu = x.double(), w_gate.double(), w_up.double()
    return activation(x @ wg.t(), kind) * (x @ wu.t())


def ffn_gradients(dout, x, w_gate, w_up, kind):
    """(dx, dw_gate, dw_up) by automatic differentiation of `ffn`."""
    x, wg, wu = (t.double().clone().requires_grad_(True) for t in (x, w_gate, w_up))
    ffn(x, wg, wu, kind).backward(dout.double())
    return x.grad, wg.grad, wu.grad


def ffn_bound(x, w_gate, w_up, kind):
    """Elementwise bound on the block's output error: each projection's 32-bit sum of d exact products is off by at most
    d units of the sum of magnitudes (twice that, for a matrix core's own order and truncation); the activation's slope
    is below 1.13; exponential and reciprocal are good to 2^-20; one rounding to bf16."""
    x, wg, wu = x.double(), w_gate.double(), w_up.double()
    d = x.shape[1]
    off_g = 2 * d * U_F32 * (x.abs() @ wg.abs().t())
    off_u = 2 * d * U_F32 * (x.abs() @ wu.abs().t())
    g, u = x @ wg.t(), x @ wu.t()
    a = activation(g, kind)
    exact = a * u
    before = 1.13 * off_g * (u.abs() + off_u) + a.abs() * off_u + 2.0 ** -20 * (g.abs() * u.abs())
    return exact, U_BF16 * (exact.abs() + before) + before + 1e-38


def relative(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    norm_ = want.norm().item()
    return (got - want).norm().item() / norm_ if norm_ else (got - want).norm().item()
