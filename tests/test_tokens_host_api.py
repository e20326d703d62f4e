"""The token operators' boundary without a GPU: the header's functions are exported and bound, it compiles as C99, and
every bad argument is refused before anything is enqueued (the pointers here are never followed)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2601_06562_amd as package
from paper_2601_06562_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, SMALL = 0, b.MOSAIC_ERR_INVALID_ARG, b.MOSAIC_ERR_UNSUPPORTED_SHAPE, b.MOSAIC_ERR_WORKSPACE_TOO_SMALL
P = 0x10000            # an aligned address that no call here gets to
NAN, INF = float("nan"), float("inf")
MOST_V = (1 << 31) - 257


def header():
    return open(os.path.join(ROOT, "include", "mosaic_tokens.h")).read()


def test_the_header_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", header(), flags=re.S)
    names = re.findall(r"\b(mosaic_\w+)\s*\(", text)
    assert sorted(names) == sorted(b.TOKEN_EXPORTS)
    for n in names:
        assert getattr(b._tokens(), n).argtypes
        assert getattr(package, n) is getattr(b, n)
    assert f"#define MOSAIC_MAX_TOP {b.MAX_TOP}" in header()


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no gcc")
def test_the_header_is_c99(tmp_path):
    src = tmp_path / "tokens.c"
    refs = ", ".join(f"(void (*)(void))&{n}" for n in b.TOKEN_EXPORTS)
    src.write_text('#include <stdio.h>\n#include "mosaic_tokens.h"\ntypedef void (*fn)(void);\n'
                   f"static fn all[] = {{{refs}}};\n"
                   'int main(void) { size_t i, n = 0; for (i = 0; i < sizeof all / sizeof all[0]; ++i) n += all[i] != 0;\n'
                   'printf("%zu %d %d %lld\\n", n, MOSAIC_MAX_TOP, mosaic_dropout_forward(0, 8, 0, 0, 0, 4, 8, 0.5f, 1u, 0, 0, 0, 8, 0),\n'
                   '(long long)mosaic_embedding_backward_workspace_bytes(4096, 512, 32000)); return 0; }\n')
    exe, libdir = str(tmp_path / "tokens"), os.path.dirname(b.LIB_PATH)
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-o", exe, str(src), "-L" + libdir, "-lmosaic", "-Wl,-rpath," + libdir, "-Wl,-rpath,/opt/rocm/lib"],
                   check=True)
    got = subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert [int(x) for x in got] == [len(b.TOKEN_EXPORTS), b.MAX_TOP, INVALID,
                                     b.mosaic_embedding_backward_workspace_bytes(4096, 512, 32000)]


def call_with(name, defaults):
    def f(**changes):
        assert set(changes) <= set(defaults)
        return getattr(b._tokens(), name)(*[changes.get(k, v) for k, v in defaults.items()])
    return f


embedding = call_with("mosaic_embedding_forward", dict(
    tokens=P, T=4, count=None, table=P, table_type=0, ld_table=512, V=100, d=512, scale=1.0, out=P, out_type=1, ld_out=512,
    stream=None))
embedding_backward = call_with("mosaic_embedding_backward", dict(
    dout=P, dout_type=0, ld_dout=512, tokens=P, T=4, count=None, V=100, d=512, scale=1.0, dtable=P, dtable_type=1, ld_dtable=512,
    accumulate=0, ws=P, bytes=1 << 30, stream=None))
dropout = call_with("mosaic_dropout_forward", dict(
    x=P, ld_x=512, residual=P, type=1, ld_r=512, T=4, d=512, p=0.1, seed=7, site=0, first_row=0, out=P, ld_out=512, stream=None))
dropout_backward = call_with("mosaic_dropout_backward", dict(
    dout=P, type=1, ld_dout=512, T=4, d=512, p=0.1, seed=7, site=0, first_row=0, dx=P, ld_dx=512, stream=None))
logprobs = call_with("mosaic_masked_logprobs", dict(
    hidden=P, ld_h=512, T=4, d=512, w=P, ld_w=512, V=1000, idx=P, count=P, max_rows=4, targets=P, logprob=P, entropy=P, lse=P,
    n_top=2, top_id=P, top_logprob=P, ws=P, bytes=1 << 40, stream=None))
logprobs_backward = call_with("mosaic_masked_logprobs_backward", dict(
    hidden=P, ld_h=512, T=4, d=512, w=P, ld_w=512, V=1000, idx=P, count=P, max_rows=4, targets=P, logprob=P, entropy=P, lse=P,
    dlogprob=P, dentropy=P, dx=P, ld_dx=512, dw=P, dw_type=0, ld_dw=512, accumulate=0, ws=P, bytes=1 << 40, stream=None))

SIZES = [(dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=-8), INVALID), (dict(d=508), SHAPE), (dict(T=1 << 31), SHAPE),
         (dict(d=1 << 18), SHAPE)]
VOCAB = [(dict(V=0), INVALID), (dict(V=-5), INVALID), (dict(V=MOST_V + 1), SHAPE), (dict(V=(1 << 31) - 1), SHAPE)]
MASK = [(dict(p=-0.01), INVALID), (dict(p=1.0), INVALID), (dict(p=NAN), INVALID), (dict(p=INF), INVALID),
        (dict(p=1.0 - 2.0 ** -17), INVALID), (dict(site=-1), INVALID), (dict(site=(1 << 31) - 1), INVALID),
        (dict(first_row=-1), INVALID), (dict(first_row=(1 << 63) - 4), SHAPE), (dict(type=2), INVALID), (dict(type=-1), INVALID)]
SCALE = [(dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(scale=-INF), INVALID)]
LISTED = [(dict(max_rows=-1), INVALID), (dict(max_rows=1 << 31), SHAPE), (dict(idx=0), INVALID), (dict(count=0), INVALID),
          (dict(idx=0, count=0, max_rows=3), INVALID), (dict(idx=P + 2), INVALID), (dict(count=P + 1), INVALID),
          (dict(targets=P + 2), INVALID), (dict(logprob=P + 2), INVALID), (dict(entropy=P + 1), INVALID), (dict(lse=P + 3), INVALID),
          (dict(hidden=0), INVALID), (dict(w=0), INVALID), (dict(hidden=P + 8), INVALID), (dict(w=P + 2), INVALID),
          (dict(ld_h=504), SHAPE), (dict(ld_h=516), SHAPE), (dict(ld_w=504), SHAPE), (dict(ld_w=1 << 22), SHAPE),
          (dict(ld_h=1 << 22), SHAPE), (dict(ws=0), INVALID), (dict(ws=P + 8), INVALID), (dict(targets=0), INVALID)]


@pytest.mark.parametrize("call,bad", [
    (embedding, SIZES + VOCAB + SCALE + [
        (dict(tokens=0), INVALID), (dict(tokens=P + 2), INVALID), (dict(count=P + 2), INVALID), (dict(table=0), INVALID),
        (dict(out=0), INVALID), (dict(table=P + 8), INVALID), (dict(out=P + 4), INVALID), (dict(table_type=2), INVALID),
        (dict(out_type=-1), INVALID), (dict(ld_table=504), SHAPE), (dict(ld_out=515), SHAPE), (dict(ld_out=1 << 22), SHAPE)]),
    (embedding_backward, SIZES + VOCAB + SCALE + [
        (dict(tokens=0), INVALID), (dict(tokens=P + 1), INVALID), (dict(count=P + 2), INVALID), (dict(dout=0), INVALID),
        (dict(dtable=0), INVALID), (dict(dout=P + 8), INVALID), (dict(dtable=P + 4), INVALID), (dict(dout_type=2), INVALID),
        (dict(dtable_type=5), INVALID), (dict(dtable_type=0, accumulate=1), INVALID), (dict(ld_dout=504), SHAPE),
        (dict(ld_dtable=511), SHAPE), (dict(ws=0), INVALID), (dict(ws=P + 4), INVALID), (dict(bytes=0), SMALL),
        (dict(bytes=b.mosaic_embedding_backward_workspace_bytes(4, 512, 100) - 1), SMALL)]),
    (dropout, SIZES + MASK + [
        (dict(x=0), INVALID), (dict(out=0), INVALID), (dict(x=P + 8), INVALID), (dict(residual=P + 8), INVALID),
        (dict(out=P + 2), INVALID), (dict(ld_x=504), SHAPE), (dict(ld_r=516), SHAPE), (dict(ld_out=8), SHAPE)]),
    (dropout_backward, SIZES + MASK + [
        (dict(dout=0), INVALID), (dict(dx=0), INVALID), (dict(dout=P + 8), INVALID), (dict(dx=P + 2), INVALID),
        (dict(ld_dout=504), SHAPE), (dict(ld_dx=1 << 22), SHAPE)]),
    (logprobs, SIZES + VOCAB + LISTED + [
        (dict(n_top=-1), INVALID), (dict(n_top=17), INVALID), (dict(top_id=0), INVALID), (dict(top_logprob=0), INVALID),
        (dict(top_id=P + 2), INVALID), (dict(top_logprob=P + 1), INVALID), (dict(bytes=0), SMALL),
        (dict(logprob=0, entropy=0, lse=0, n_top=0), INVALID),
        (dict(bytes=b.mosaic_masked_logprobs_workspace_bytes(4, 4, 512, 1000, 2) - 1), SMALL)]),
    (logprobs_backward, SIZES + VOCAB + LISTED + [
        (dict(dx=0, dw=0), INVALID), (dict(dlogprob=0, dentropy=0), INVALID), (dict(lse=0), INVALID), (dict(logprob=0), INVALID),
        (dict(entropy=0), INVALID), (dict(dlogprob=P + 2), INVALID), (dict(dentropy=P + 1), INVALID), (dict(dx=P + 8), INVALID),
        (dict(dw=P + 8), INVALID), (dict(dw_type=2), INVALID), (dict(accumulate=1), INVALID), (dict(ld_dx=504), SHAPE),
        (dict(ld_dw=511), SHAPE), (dict(bytes=0), SMALL), (dict(bytes=4 * 512 * 10), SMALL)]),
], ids=["embedding", "embedding_backward", "dropout", "dropout_backward", "logprobs", "logprobs_backward"])
def test_bad_arguments_are_refused(call, bad):
    for changes, want in bad:
        assert call(**changes) == want, changes


def test_calls_that_enqueue_nothing():
    assert embedding(T=0, tokens=0, table=0, out=0) == OK
    assert embedding_backward(T=0, accumulate=1, tokens=0, dout=0, ws=0) == OK
    assert dropout(T=0, x=0, out=0) == OK and dropout_backward(T=0, dout=0, dx=0) == OK
    assert logprobs(max_rows=0, hidden=0, w=0, ws=0) == OK and logprobs(T=0, max_rows=0, idx=0, count=0) == OK
    assert logprobs(T=0, hidden=0, ws=0) == OK                     # a bound on a list of nothing
    assert logprobs_backward(max_rows=0, dw=0, hidden=0, ws=0) == OK and logprobs_backward(T=0, dw=0, w=0) == OK
    assert logprobs_backward(max_rows=0, accumulate=1, dw_type=1, ws=0) == OK


def test_workspaces():
    """Zero for sizes that the calls refuse; what they hold is bounded."""
    assert [b.mosaic_embedding_backward_workspace_bytes(*s) for s in ((4, 100, 5), (-1, 8, 5), (4, 8, 0), (4, 8, MOST_V + 1))] == [0] * 4
    for T, d, V in ((1, 8, 1), (1000, 4096, 50000), (1 << 20, 8192, 126464)):
        n = b.mosaic_embedding_backward_workspace_bytes(T, d, V)
        assert 8 * T <= n <= 4 * d * (T // 4 + 2) + 64 * T + (1 << 22)
    query = b.mosaic_masked_logprobs_workspace_bytes
    assert [query(*s) for s in ((4, 4, 100, 5), (4, -1, 64, 5), (4, 4, 64, 0), (4, 4, 64, 5, 17), (4, 4, 64, 5, -1))] == [0] * 5
    assert query(4, 4, 64, 5, ld_h=56) == 0
    for n_top in (0, 1, 8, 16):      # sums (12 bytes) and candidates (8 a piece) of both halves of the units, and of alternatives the lists
        for rows in (1, 100, 4096, 1 << 20):
            units = max(512, 4 * ((rows + 255) // 256) + 256)
            n = query(rows, rows, 1024, 126464, n_top)
            lists = 64 << 20 if n_top else 0
            assert lists < n <= lists + 2 * 256 * units * (12 + 8 * n_top) + 4 * rows + 2048, (rows, n_top, n)
    query = b.mosaic_masked_logprobs_backward_workspace_bytes
    assert query(0, 64, 5) == 0 and query(4, 60, 5) == 0 and query(4, 64, 0) == 0
    for rows, d, V in ((1, 64, 300), (100, 512, 5000), (4096, 4096, 126464)):
        least, default = query(rows, d, V, 1), query(rows, d, V)
        assert 10 * rows * d < least <= default <= least + (256 << 20) + (1 << 20)
        for budget in (least, least + 1234567, default + (1 << 30)):
            assert least <= query(rows, d, V, budget) <= budget


def test_a_workspace_serves_fewer_rows():
    for d, V in ((64, 300), (512, 32000), (4096, 126464)):
        rows = (*range(1, 3000, 37), 4096, 20000, 131072)
        need = [b.mosaic_embedding_backward_workspace_bytes(T, d, V) for T in rows]
        assert need == sorted(need)
        for n_top in (0, 5):
            need = [b.mosaic_masked_logprobs_workspace_bytes(1 << 20, n, d, V, n_top) for n in rows]
            assert need == sorted(need)
        need = [b.mosaic_masked_logprobs_backward_workspace_bytes(n, d, V, 1) for n in rows]
        assert need == sorted(need)


def test_the_binding_checks_shapes_and_types():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    w = torch.zeros((128, 64), dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    ws = torch.zeros(16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device memory"):
        b.mosaic_embedding_forward(ids, w, x)
    with pytest.raises((ValueError, TypeError)):
        b.mosaic_embedding_forward(ids.long(), w, x)
    with pytest.raises(ValueError, match="device memory"):
        b.mosaic_embedding_backward(x, ids, w, ws)
    with pytest.raises(TypeError, match="residual's type"):
        b.mosaic_dropout_forward(x, x.float(), x, 0.1, 1)
    with pytest.raises(ValueError, match="go together"):
        b.mosaic_masked_logprobs(x, w, ids, None, 4, None, None, None, None, ws)
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(w=w.half())):
        with pytest.raises((ValueError, TypeError)):
            b.mosaic_masked_logprobs(bad.get("x", x), bad.get("w", w), None, None, 4, None, None, None, None, ws)
