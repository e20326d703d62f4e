"""Measured cases of the operators around the mask-only pass: the root-mean-square norm with the residual's addition and
an 8-bit output, activation checkpoints in 8 bits, and the gated feed-forward block, each with its backward pass.

Fields of a case:

  op          "norm", "norm_backward", "checkpoint", "ffn", "ffn_backward"
  rows, d, f  positions, hidden size, feed-forward size (0 where there is none)
  stream      type of the residual stream: "bf16" or "f32"
  masked      norm: how many of the rows are listed (0: all of them, without a list)
  q8          "": none; "int8", "e4m3": norm: an 8-bit output beside the bf16 one, restored as a backward pass does;
              checkpoint: the format; norm_backward and ffn_backward: what the forward pass kept is a checkpoint
  group       columns that share a scale
  act         "silu" or "gelu" (tanh form)
  pad         columns between the end of a row and the next row, in every activation
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5
Q_MAX = {"int8": 127.0, "e4m3": 448.0}


def _case(name=None, *, op, rows, d, f=0, stream="bf16", masked=0, q8="", group=128, act="silu", pad=0):
    c = {} if name is None else {"name": name}
    c.update(op=op, rows=rows, d=d, f=f, stream=stream, masked=masked, q8=q8, group=group, act=act, pad=pad)
    return c


def listed():
    return [
        # One new token through a layer's norm, with the 8-bit copy: only latency counts.
        _case("norm_token", op="norm", rows=1, d=4096, q8="int8"),
        # The final norm ahead of mask-only logits: the masked half of the last 8192 positions of a long context.
        _case("norm_masked", op="norm", rows=32768, d=4096, masked=4105),
        # A layer's norm over a batch of long sequences on a 32-bit residual stream, with an e4m3 copy.
        _case("norm_batch", op="norm", rows=32768, d=4096, stream="f32", q8="e4m3"),
        # The norm's backward pass over a short ragged batch, from the 8-bit checkpoint of the residual sum.
        _case("norm_backward_q8", op="norm_backward", rows=1003, d=3584, q8="int8", group=64),
        # The same over a batch of long sequences, from the sum itself.
        _case("norm_backward_batch", op="norm_backward", rows=16384, d=4096),
        # What a training step keeps of one small layer's activations, stored and restored.
        _case("checkpoint_small", op="checkpoint", rows=512, d=512, q8="e4m3", group=32),
        # The same for a batch of long sequences.
        _case("checkpoint_batch", op="checkpoint", rows=65535, d=3584, q8="int8"),
        # The feed-forward block for one new token: the weights are read once for a single row.
        _case("ffn_token", op="ffn", rows=1, d=4096, f=12288),
        # For a block of positions under generation.
        _case("ffn_block", op="ffn", rows=37, d=3584, f=18944),
        # For every position of a batch of prompts.
        _case("ffn_batch", op="ffn", rows=16384, d=4096, f=12288),
        # Training, a small layer and a ragged batch.
        _case("ffn_backward_small", op="ffn_backward", rows=1237, d=1024, f=4096, act="gelu", pad=64),
        # Training, a full layer from the 8-bit checkpoint of its input.
        _case("ffn_backward_q8", op="ffn_backward", rows=4096, d=4096, f=12288, q8="int8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_backward", "checkpoint", "ffn", "ffn", "ffn_backward", "ffn_backward"])
    if op == "ffn":
        d, f = rng.choice([(512, 2048), (1024, 4096), (1032, 2744), (2048, 8192), (3584, 18944), (4096, 12288)])
        rows = _log_int(rng, 1, 12000)
    elif op == "ffn_backward":
        d, f = rng.choice([(512, 2048), (1024, 4096), (1032, 2744), (2048, 8192), (3584, 18944), (4096, 12288)])
        rows = _log_int(rng, 1, 2700)
    else:
        d, f = rng.choice([512, 1000, 1024, 2048, 3584, 4096, 8192]), 0
        rows = _log_int(rng, 1, 12000 if op == "norm" else 16000)
    q8 = rng.choice(["", "int8", "e4m3"])
    if op == "ffn":
        q8 = ""
    if op == "checkpoint":
        q8 = rng.choice(["int8", "e4m3"])
    masked = max(1, int(rows * rng.choice([0.05, 0.3, 0.8]))) if op == "norm" and not q8 and rng.random() < 0.5 else 0
    return _case(op=op, rows=rows, d=d, f=f, stream=rng.choice(["bf16", "bf16", "f32"]), masked=masked, q8=q8,
                 group=rng.choice([32, 64, 128, 128]), act=rng.choice(["silu", "silu", "gelu"]),
                 pad=rng.choice([0, 0, 8, 64]))


class _State:
    pass


def _groups(case):
    return -(-case["d"] // case["group"])


def prepare(case, seed):
    """Inputs on the GPU.  Activations are N(0, 1) with a few columns ten times as large, as residual streams have
    them; weights N(0, 1/d); gains around one; gradients N(0, 1) scaled as a mean over the rows leaves them."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = _State()
    s.case, s.op = case, case["op"]
    T, d, f, pad = case["rows"], case["d"], case["f"], case["pad"]
    stream = torch.float32 if case["stream"] == "f32" else torch.bfloat16
    scale = torch.ones(d, device=DEVICE)
    scale[torch.randint(0, d, (max(1, d // 256),), generator=gen, device=DEVICE)] = 10.0

    def rows(cols, dtype=torch.bfloat16, by=1.0, wide=None):
        out = torch.empty((T, cols + pad), dtype=dtype, device=DEVICE)[:, :cols]
        for r in range(0, T, 16384):
            n = min(T, r + 16384) - r
            z = torch.randn((n, cols), generator=gen, device=DEVICE) * by
            out[r:r + n] = z if wide is None else z * wide
        return out

    def blank(cols, dtype=torch.bfloat16):
        return torch.zeros((T, cols + pad), dtype=dtype, device=DEVICE)[:, :cols]

    def weight(r, c):
        return (torch.randn((r, c), generator=gen, device=DEVICE) * c ** -0.5).to(torch.bfloat16)

    def eight_bit(v):
        """What a forward pass kept: the values and scales of `v` in 8 bits."""
        s.values, s.scales = _quantise(v.float(), case)

    s.workspace = None
    if s.op in ("norm", "norm_backward"):
        s.gamma = 1.0 + 0.1 * torch.randn(d, generator=gen, device=DEVICE)
    if s.op == "norm":
        s.x, s.residual = rows(d), rows(d, stream, wide=scale)
        s.sum, s.y = blank(d, stream), blank(d)
        s.idx = s.count = None
        if case["masked"]:
            s.idx = torch.randperm(T, generator=gen, device=DEVICE)[:case["masked"]].sort().values.to(torch.int32)
            s.count = torch.tensor([case["masked"]], dtype=torch.int32, device=DEVICE)
    elif s.op == "norm_backward":
        s.h = rows(d, stream, wide=scale)
        s.dy, s.dsum_in = rows(d, by=1e-3), rows(d, stream, by=1e-3)
        s.dsum, s.dgamma = blank(d, stream), torch.zeros(d, device=DEVICE)
        if case["q8"]:
            eight_bit(s.h)
            s.h = None
    elif s.op == "checkpoint":
        s.x = rows(d, wide=scale)
    else:
        s.x = rows(d, wide=scale)
        s.w_gate, s.w_up = weight(f, d), weight(f, d)
        s.out = blank(f)
        if s.op == "ffn_backward":
            s.dout = rows(f, by=1e-3)
            s.dx = blank(d)
            s.dw_gate, s.dw_up = torch.zeros_like(s.w_gate), torch.zeros_like(s.w_up)
            if case["q8"]:
                eight_bit(s.x)
                s.x = None
    if case["q8"] and s.op in ("norm", "checkpoint"):
        kind = torch.int8 if case["q8"] == "int8" else torch.float8_e4m3fn
        s.values = torch.zeros((T, d), dtype=kind, device=DEVICE)
        s.scales = torch.zeros((T, _groups(case)), device=DEVICE)
        s.restored = blank(d)
    s.q8 = None
    return s


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end

def _by_group(v, case):
    """`v` as [rows, groups, group], the last group filled up with zeros."""
    fill = _groups(case) * case["group"] - v.shape[1]
    return torch.nn.functional.pad(v, (0, fill)).view(v.shape[0], -1, case["group"])


def _quantise(v, case):
    """(values, scales) of the rows of `v`: each group's largest magnitude becomes the format's largest number."""
    top = Q_MAX[case["q8"]]
    g = _by_group(v, case)
    most = g.abs().amax(dim=2, keepdim=True)
    q = g * (top / most.clamp_min(1e-30))
    q = q.round().to(torch.int8) if case["q8"] == "int8" else q.to(torch.float8_e4m3fn)
    return q.view(v.shape[0], -1)[:, :v.shape[1]].contiguous(), (most / top).squeeze(2)


def _restore(values, scales, case):
    """The bf16 numbers that 8-bit values stand for."""
    g = _by_group(values.float(), case) * scales[:, :, None]
    return g.view(values.shape[0], -1)[:, :values.shape[1]].to(torch.bfloat16)


def _norm_plain(s):
    case = s.case
    at = slice(None) if s.idx is None else s.idx.long()
    h = s.x[at].float() + s.residual[at].float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS) * s.gamma
    s.sum[at] = h.to(s.sum.dtype)
    s.y[at] = y.to(torch.bfloat16)
    out = {"sum": s.sum, "y": s.y}
    if case["q8"]:
        values, scales = _quantise(y, case)
        out.update(restored=_restore(values, scales, case), scales=scales)
    return out


def _norm_backward_plain(s):
    h = s.h.float() if s.h is not None else _restore(s.values, s.scales, s.case).float()
    dy = s.dy.float()
    rstd = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    xh, c = h * rstd, dy * s.gamma
    dh = rstd * (c - xh * (c * xh).mean(dim=1, keepdim=True)) + s.dsum_in.float()
    return {"dsum": dh.to(s.dsum.dtype), "dgamma": (dy * xh).sum(dim=0)}


def _act_plain(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    k, c = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(k * (g + c * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3.0 * c * g * g)


def _ffn_plain(s):
    x = s.x.float()
    a, _ = _act_plain(x @ s.w_gate.float().t(), s.case["act"])
    return {"out": (a * (x @ s.w_up.float().t())).to(torch.bfloat16)}


def _ffn_backward_plain(s):
    x = s.x.float() if s.x is not None else _restore(s.values, s.scales, s.case).float()
    wg, wu, do = s.w_gate.float(), s.w_up.float(), s.dout.float()
    u = x @ wu.t()
    a, slope = _act_plain(x @ wg.t(), s.case["act"])
    dg, du = do * u * slope, do * a
    return {"out": (a * u).to(torch.bfloat16), "dx": (dg @ wg + du @ wu).to(torch.bfloat16),
            "dw_gate": (dg.t() @ x).to(torch.bfloat16), "dw_up": (du.t() @ x).to(torch.bfloat16)}


# ---- the framework's operators, as a user calls them

def _kept(s):
    """The checkpoint's handle over the state's values and scales."""
    from paper_2601_06562_amd import binding
    if s.q8 is None:
        s.q8 = binding.Q8Rows(s.values, s.scales, s.case["group"])
    return s.q8


def _run_own(s):
    from paper_2601_06562_amd import binding as b
    case = s.case
    if s.op == "norm":
        q8 = _kept(s) if case["q8"] else None
        b.mosaic_rmsnorm_forward(s.x, s.residual, s.gamma, EPS, s.y, sum=s.sum, q8=q8, idx=s.idx, count=s.count)
        out = {"sum": s.sum, "y": s.y}
        if q8 is not None:
            b.mosaic_checkpoint_load(q8, s.restored)
            out.update(restored=s.restored, scales=s.scales)
        return out
    if s.op == "checkpoint":
        b.mosaic_checkpoint_store(s.x, _kept(s))
        b.mosaic_checkpoint_load(_kept(s), s.restored)
        return {"restored": s.restored, "scales": s.scales}
    if s.op == "norm_backward":
        if s.workspace is None:
            need = b.mosaic_rmsnorm_backward_workspace_bytes(case["rows"], case["d"])
            s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE)
        b.mosaic_rmsnorm_backward(s.dy, s.h if s.h is not None else _kept(s), s.gamma, EPS, s.dsum, s.dgamma, s.workspace,
                                  dsum_in=s.dsum_in)
        return {"dsum": s.dsum, "dgamma": s.dgamma}
    act = b.ACT_SILU if case["act"] == "silu" else b.ACT_GELU_TANH
    if s.op == "ffn":
        b.mosaic_gated_ffn_forward(s.x, s.w_gate, s.w_up, s.out, activation=act)
        return {"out": s.out}
    if s.workspace is None:
        need = b.mosaic_gated_ffn_backward_workspace_bytes(case["rows"], case["d"], case["f"], q8_input=bool(case["q8"]))
        s.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE)
    b.mosaic_gated_ffn_backward(s.dout, s.x if s.x is not None else _kept(s), s.w_gate, s.w_up, s.dx, s.dw_gate, s.dw_up,
                                s.workspace, activation=act, out=s.out)
    return {"out": s.out, "dx": s.dx, "dw_gate": s.dw_gate, "dw_up": s.dw_up}


def run(s):
    if own:
        return _run_own(s)
    if s.op == "norm":
        return _norm_plain(s)
    if s.op == "norm_backward":
        return _norm_backward_plain(s)
    if s.op == "checkpoint":
        values, scales = _quantise(s.x.float(), s.case)
        return {"restored": _restore(values, scales, s.case), "scales": scales}
    return _ffn_plain(s) if s.op == "ffn" else _ffn_backward_plain(s)


def work(case):
    """Each input read once, each output written once; an 8-bit copy that is restored is written and read."""
    T, d, f = case["rows"], case["d"], case["f"]
    st = 4 if case["stream"] == "f32" else 2
    eight = T * d + 4.0 * T * _groups(case)
    if case["op"] == "norm":
        n = case["masked"] or T
        total = n * d * (2.0 + st + st + 2.0) + 4.0 * d + (4.0 * n if case["masked"] else 0.0)
        if case["q8"]:
            total += 2 * eight + 2.0 * T * d
        return {"bytes": total, "flops": 8.0 * n * d}
    if case["op"] == "norm_backward":
        kept = eight if case["q8"] else st * T * d
        return {"bytes": kept + T * d * (2.0 + 2 * st) + 8.0 * d, "flops": 14.0 * T * d}
    if case["op"] == "checkpoint":
        return {"bytes": 2 * eight + 4.0 * T * d, "flops": 4.0 * T * d}
    if case["op"] == "ffn":
        return {"bytes": 2.0 * (T * d + 2 * f * d + T * f), "flops": 4.0 * T * d * f}
    kept = eight if case["q8"] else 2.0 * T * d
    return {"bytes": kept + 2.0 * (T * d + 2 * T * f + 4 * f * d), "flops": 12.0 * T * d * f}


# ---- the definitions in 64 bits, for the comparison alone

def _round_e4m3(v):
    """Nearest number of 4 exponent and 3 fraction bits (smallest step 2^-9), ties to even; |v| <= 448."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 4, min=-9))
    return torch.round(v / step) * step


def _exact_eight(v, case):
    """What the rows of `v` become in 8 bits, and the scales."""
    of = torch.arange(v.shape[1], device=v.device) // case["group"]      # each column's group
    most = v.new_zeros((v.shape[0], _groups(case))).scatter_reduce_(1, of.expand_as(v), v.abs(), "amax")
    scales = most / Q_MAX[case["q8"]]
    wide = scales.index_select(1, of)
    q = v / wide.clamp_min(1e-300)
    return (torch.round(q) if case["q8"] == "int8" else _round_e4m3(q)) * wide, scales


def _exact_kept(s, whole):
    """The layer's input in 64 bits: as it was kept, whole or in 8 bits (where it stands for a bf16 number)."""
    if whole is not None:
        return whole.double()
    v = s.values.double() * s.scales.double().repeat_interleave(s.case["group"], dim=1)[:, :s.values.shape[1]]
    return v.to(torch.bfloat16).double()


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "checkpoint":
        restored, scales = _exact_eight(s.x.double(), case)
        return {"restored": restored, "scales": scales}
    if s.op == "norm":
        total, y_all = s.sum.double(), s.y.double()
        at = torch.arange(case["rows"], device=DEVICE) if s.idx is None else s.idx.long()
        h = s.x.double().index_select(0, at) + s.residual.double().index_select(0, at)
        y = h / torch.sqrt((h * h).sum(dim=1, keepdim=True) / case["d"] + EPS) * s.gamma.double()
        out = {"sum": total.index_copy(0, at, h), "y": y_all.index_copy(0, at, y)}
        if case["q8"]:
            out["restored"], out["scales"] = _exact_eight(y, case)
        return out
    if s.op == "norm_backward":
        h, dy, gamma = _exact_kept(s, s.h), s.dy.double(), s.gamma.double()
        root = torch.sqrt((h * h).sum(dim=1, keepdim=True) / case["d"] + EPS)
        along = (dy * gamma * h).sum(dim=1, keepdim=True) / case["d"]
        return {"dsum": s.dsum_in.double() + dy * gamma / root - h * along / root ** 3, "dgamma": (dy * h / root).sum(dim=0)}
    x = _exact_kept(s, s.x)
    wg, wu = s.w_gate.double(), s.w_up.double()
    g, u = torch.mm(x, wg.t().contiguous()), torch.mm(x, wu.t().contiguous())
    if case["act"] == "silu":
        a = g * torch.sigmoid(g)
        slope = torch.sigmoid(g) + a * torch.sigmoid(-g)
    else:
        z = math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
        a = g * torch.sigmoid(2.0 * z)                               # (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        slope = torch.sigmoid(2.0 * z) * (1.0 + 2.0 * g * torch.sigmoid(-2.0 * z) * math.sqrt(2.0 / math.pi)
                                          * (1.0 + 3.0 * 0.044715 * g * g))
    if s.op == "ffn":
        return {"out": a * u}
    do = s.dout.double()
    du, dg = do * a, do * slope * u
    return {"out": a * u, "dx": torch.mm(dg, wg) + torch.mm(du, wu), "dw_gate": torch.mm(dg.t().contiguous(), x),
            "dw_up": torch.mm(du.t().contiguous(), x)}
