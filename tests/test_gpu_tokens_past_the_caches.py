"""Lookups and dropouts whose outputs, from 128 MiB on, are written past the caches, with an odd last row: lookups against plain ones,
dropouts against the same taken in parts that are below that size (which test_gpu_tokens_dropout.py holds to the definition)."""
import pytest
import torch

from paper_2601_06562_amd import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
PAST = 128 << 20
SEED = 0x0123456789ABCDEF


def blank(T, d, dtype, pad, rows=1):
    full = torch.full((T + rows, d + pad), 777.0, dtype=dtype, device=DEV)
    return full[:T, :d], full


def untouched(full, T, d):
    return bool((full[:, d:] == 777.0).all()) and bool((full[T:] == 777.0).all())


def rows_for(d, dtype):
    """The fewest rows of an output of at least 128 MiB, made odd."""
    return -(-PAST // (d * dtype.itemsize)) | 1


@pytest.mark.parametrize("d,pad", [(1024, 0), (1032, 8), (4096, 8), (2056, 16)])
@pytest.mark.parametrize("table_type", [BF16, F32])
@pytest.mark.parametrize("out_type", [BF16, F32])
def test_lookup(d, pad, table_type, out_type):
    T, V = rows_for(d, out_type), 5003
    assert T * d * out_type.itemsize >= PAST and T % 2 == 1
    gen = torch.Generator(device=DEV).manual_seed(d)
    table = torch.randn((V, d), generator=gen, device=DEV).to(table_type)
    tokens = torch.randint(-20, V + 20, (T,), generator=gen, device=DEV, dtype=torch.int32)
    tokens[T - 1], tokens[T - 2] = V - 1, -1
    there = ((tokens >= 0) & (tokens < V))[:, None]
    # scaled by a power of two, so that a result is rounded by its type alone
    want = torch.where(there, table[tokens.long().clamp(0, V - 1)].float() * 0.125, 0.0).to(out_type)
    for count in (None, T - 1, T - 2, 3):
        out, full = blank(T, d, out_type, pad)
        n = T if count is None else count
        print("lookup", T, d, table_type, out_type, count, flush=True)
        b.mosaic_embedding_forward(tokens, table, out, scale=0.125,
                                   count=None if count is None else torch.tensor([count], dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        assert torch.equal(out[:n], want[:n]) and bool((out[n:] == 777.0).all()) and untouched(full, T, d)


@pytest.mark.parametrize("d,pad", [(1024, 0), (1032, 8), (2056, 16)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("stream_type", [BF16, F32])
def test_dropout(d, pad, add, stream_type):
    T = rows_for(d, stream_type)
    gen = torch.Generator(device=DEV).manual_seed(d + add)
    x, r = (torch.randn((T, d), generator=gen, device=DEV).to(t) for t in (BF16, stream_type))
    x[T - 1, :8] = float("nan")
    (out, full), (parts, _) = blank(T, d, stream_type, pad), blank(T, d, stream_type, pad)
    print("dropout", T, d, add, stream_type, flush=True)
    b.mosaic_dropout_forward(x, r if add else None, out, 0.5, SEED, site=2, first_row=5)
    each = T // 3 + 1
    for t in range(0, T, each):
        b.mosaic_dropout_forward(x[t:t + each], r[t:t + each] if add else None, parts[t:t + each], 0.5, SEED, site=2, first_row=5 + t)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16 if stream_type is BF16 else torch.int32), parts.view(torch.int16 if stream_type is BF16 else torch.int32))
    assert untouched(full, T, d)
    kept = (out.float() - (r.float() if add else 0.0)) != 0
    assert abs(kept.double().mean().item() - 0.5) < 1e-3
    if stream_type is BF16:      # into its own input, and into the residual's memory
        mine = x.clone()
        b.mosaic_dropout_forward(mine, r if add else None, mine, 0.5, SEED, site=2, first_row=5)
        assert torch.equal(mine.view(torch.int16), parts.contiguous().view(torch.int16))
    if add:
        b.mosaic_dropout_forward(x, r, r, 0.5, SEED, site=2, first_row=5)
        assert torch.equal(r.nan_to_num(7.0), parts.nan_to_num(7.0))


@pytest.mark.parametrize("d,pad", [(1024, 0), (1032, 8), (2056, 16)])
@pytest.mark.parametrize("stream_type", [BF16, F32])
def test_dropout_backward(d, pad, stream_type):
    T = rows_for(d, BF16)
    gen = torch.Generator(device=DEV).manual_seed(d)
    g = torch.randn((T, d), generator=gen, device=DEV).to(stream_type)
    (dx, full), (parts, _) = blank(T, d, BF16, pad), blank(T, d, BF16, pad)
    print("dropout backward", T, d, stream_type, flush=True)
    b.mosaic_dropout_backward(g, dx, 0.3, SEED, first_row=1 << 33)
    each = T // 3 + 1
    for t in range(0, T, each):
        b.mosaic_dropout_backward(g[t:t + each], parts[t:t + each], 0.3, SEED, first_row=(1 << 33) + t)
    torch.cuda.synchronize()
    assert torch.equal(dx, parts) and untouched(full, T, d)
    if stream_type is BF16:
        b.mosaic_dropout_backward(g, g, 0.3, SEED, first_row=1 << 33)
        assert torch.equal(g, parts)
