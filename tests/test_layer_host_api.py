"""The layer operators' boundary without a GPU: the header's functions are exported and bound, it compiles as C99, and
every bad argument is refused before anything is enqueued (the pointers here are never followed)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2601_06562_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, SMALL = 0, b.MOSAIC_ERR_INVALID_ARG, b.MOSAIC_ERR_UNSUPPORTED_SHAPE, b.MOSAIC_ERR_WORKSPACE_TOO_SMALL
P = 0x10000            # an aligned address that no call here gets to


def header():
    return open(os.path.join(ROOT, "include", "mosaic_layer.h")).read()


def test_the_header_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", header(), flags=re.S)
    names = re.findall(r"\b(mosaic_\w+)\s*\(", text)
    assert sorted(names) == sorted(b.LAYER_EXPORTS)
    for n in names:
        assert getattr(b._layer(), n).argtypes
    assert f"#define MOSAIC_MAX_NORM_ROW {b.MAX_NORM_ROW}" in header() and "#define MOSAIC_MAX_ROW (1 << 17)" in header()
    assert b.MAX_ROW == 1 << 17


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no gcc")
def test_the_header_is_c99(tmp_path):
    src = tmp_path / "layer.c"
    refs = ", ".join(f"(void (*)(void))&{n}" for n in b.LAYER_EXPORTS)
    src.write_text('#include <stdio.h>\n#include "mosaic_layer.h"\ntypedef void (*fn)(void);\n'
                   f"static fn all[] = {{{refs}}};\n"
                   'int main(void) { size_t i, n = 0; for (i = 0; i < sizeof all / sizeof all[0]; ++i) n += all[i] != 0;\n'
                   'printf("%zu %zu %d %lld\\n", n, sizeof(mosaic_q8_rows), mosaic_checkpoint_store(0, 0, 0, -1, 8, 0, 0),\n'
                   '(long long)mosaic_gated_ffn_backward_workspace_bytes(4096, 512, 2048, 1)); return 0; }\n')
    exe, libdir = str(tmp_path / "layer"), os.path.dirname(b.LIB_PATH)
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-o", exe, str(src), "-L" + libdir, "-lmosaic", "-Wl,-rpath," + libdir, "-Wl,-rpath,/opt/rocm/lib"],
                   check=True)
    got = subprocess.run([exe], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert [int(x) for x in got] == [len(b.LAYER_EXPORTS), ctypes.sizeof(b.MosaicQ8Rows), INVALID,
                                     b.mosaic_gated_ffn_backward_workspace_bytes(4096, 512, 2048, True)]


def q8(values=P, scales=P, ld_values=512, ld_scales=4, fmt=0, group=128):
    return ctypes.byref(b.MosaicQ8Rows(values, scales, ld_values, ld_scales, fmt, group))


BAD_Q8 = [(dict(values=0), INVALID), (dict(scales=0), INVALID), (dict(values=P + 4), INVALID), (dict(scales=P + 2), INVALID),
          (dict(fmt=2), INVALID), (dict(group=16), INVALID), (dict(group=96), INVALID), (dict(ld_values=504), SHAPE),
          (dict(ld_values=516), SHAPE), (dict(ld_scales=3), SHAPE)]


def with_defaults(call, defaults):
    def f(**changes):
        assert set(changes) <= set(defaults)
        return call(*[changes.get(k, v) for k, v in defaults.items()])
    return f


def store(**c):
    return with_defaults(b._layer().mosaic_checkpoint_store, dict(x=P, type=0, ld=512, T=4, d=512, q8=q8(), stream=None))(**c)


def load(**c):
    return with_defaults(b._layer().mosaic_checkpoint_load, dict(q8=q8(), T=4, d=512, out=P, type=0, ld=512, stream=None))(**c)


def norm(**c):
    return with_defaults(b._layer().mosaic_rmsnorm_forward, dict(
        x=P, ld_x=512, residual=P, type=0, ld_r=512, gamma=P, gamma_type=1, eps=1e-5, T=4, d=512, idx=None, count=None,
        max_rows=0, sum=P, ld_sum=512, y=P, ld_y=512, q8=None, stream=None))(**c)


def norm_backward(**c):
    return with_defaults(b._layer().mosaic_rmsnorm_backward, dict(
        dy=P, ld_dy=512, h=P, ld_h=512, q8=None, type=0, gamma=P, gamma_type=1, eps=1e-5, T=4, d=512, dsum_in=P,
        ld_in=512, dsum=P, ld_dsum=512, dgamma=P, accumulate=0, ws=P, bytes=1 << 30, stream=None))(**c)


def ffn(**c):
    return with_defaults(b._layer().mosaic_gated_ffn_forward, dict(
        x=P, ld_x=512, wg=P, wu=P, ld_w=512, T=4, d=512, F=1024, act=0, out=P, ld_out=1024, stream=None))(**c)


def ffn_backward(**c):
    return with_defaults(b._layer().mosaic_gated_ffn_backward, dict(
        dout=P, ld_dout=1024, x=P, ld_x=512, q8=None, wg=P, wu=P, ld_w=512, T=4, d=512, F=1024, act=0, out=P, ld_out=1024,
        dx=P, ld_dx=512, dwg=P, dwu=P, dw_type=0, ld_dw=512, accumulate=0, ws=P, bytes=1 << 40, stream=None))(**c)


COMMON = [(dict(T=-1), INVALID), (dict(d=0), INVALID), (dict(d=-8), INVALID), (dict(d=508), SHAPE), (dict(T=1 << 31), SHAPE),
          (dict(d=1 << 18), SHAPE)]


@pytest.mark.parametrize("call,bad", [
    (store, COMMON + [(dict(x=0), INVALID), (dict(x=P + 8), INVALID), (dict(type=2), INVALID), (dict(ld=504), SHAPE),
                      (dict(ld=513), SHAPE), (dict(ld=1 << 22), SHAPE), (dict(q8=None), INVALID), (dict(d=16392), SHAPE)]),
    (load, COMMON + [(dict(out=0), INVALID), (dict(out=P + 2), INVALID), (dict(type=-1), INVALID), (dict(ld=504), SHAPE),
                     (dict(q8=None), INVALID)]),
    (norm, COMMON + [(dict(x=0, residual=0), INVALID), (dict(sum=0, y=0), INVALID), (dict(gamma=0), INVALID),
                     (dict(gamma=P + 4), INVALID), (dict(gamma_type=3), INVALID), (dict(type=7), INVALID),
                     (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
                     (dict(eps=float("inf")), INVALID), (dict(idx=P), INVALID), (dict(count=P), INVALID),
                     (dict(idx=P, count=P, max_rows=5), INVALID), (dict(idx=P, count=P, max_rows=-1), INVALID),
                     (dict(idx=P + 1, count=P, max_rows=1), INVALID), (dict(x=P + 8), INVALID), (dict(ld_x=504), SHAPE),
                     (dict(ld_r=516), SHAPE), (dict(ld_sum=500), SHAPE), (dict(ld_y=8), SHAPE), (dict(d=16392), SHAPE)]),
    (norm_backward, COMMON + [(dict(dy=0), INVALID), (dict(h=0), INVALID), (dict(q8=q8()), INVALID), (dict(gamma=0), INVALID),
                              (dict(dsum=0, dgamma=0), INVALID), (dict(dgamma=P + 4), INVALID), (dict(ws=0), INVALID),
                              (dict(ws=P + 8), INVALID), (dict(bytes=0), SMALL), (dict(eps=0.0), INVALID),
                              (dict(ld_dy=504), SHAPE), (dict(ld_h=4), SHAPE), (dict(ld_in=511), SHAPE),
                              (dict(ld_dsum=511), SHAPE), (dict(type=2), INVALID)]),
    (ffn, COMMON + [(dict(F=0), INVALID), (dict(F=1020), SHAPE), (dict(F=1 << 18), SHAPE), (dict(x=0), INVALID),
                    (dict(wg=0), INVALID), (dict(wu=0), INVALID), (dict(out=0), INVALID), (dict(x=P + 8), INVALID),
                    (dict(wu=P + 2), INVALID), (dict(act=2), INVALID), (dict(ld_x=504), SHAPE), (dict(ld_w=511), SHAPE),
                    (dict(ld_out=1016), SHAPE), (dict(ld_x=1 << 22), SHAPE)]),
    (ffn_backward, COMMON + [(dict(F=0), INVALID), (dict(F=1020), SHAPE), (dict(x=0), INVALID), (dict(q8=q8()), INVALID),
                             (dict(dout=0), INVALID), (dict(wg=0), INVALID), (dict(dwg=0), INVALID), (dict(dwu=0), INVALID),
                             (dict(dx=0, dwg=0, dwu=0, out=0), INVALID), (dict(accumulate=1), INVALID),
                             (dict(dw_type=5), INVALID), (dict(act=-1), INVALID), (dict(ws=0), INVALID),
                             (dict(ws=P + 4), INVALID), (dict(bytes=4 * 4 * 1024 - 1), SMALL), (dict(ld_dw=504), SHAPE),
                             (dict(ld_dx=504), SHAPE), (dict(ld_dout=1016), SHAPE), (dict(ld_out=1000), SHAPE),
                             (dict(dx=P + 8), INVALID)]),
], ids=["store", "load", "norm", "norm_backward", "ffn", "ffn_backward"])
def test_bad_arguments_are_refused(call, bad):
    for changes, want in bad:
        assert call(**changes) == want, changes


def test_bad_eight_bit_rows_are_refused():
    for changes, want in BAD_Q8:
        bad = q8(**changes)
        assert store(q8=bad) == want and load(q8=bad) == want and norm(q8=bad) == want, changes
        assert norm_backward(h=0, q8=bad) == want and ffn_backward(x=0, q8=bad) == want, changes
    assert ffn_backward(x=0, q8=q8(ld_values=1 << 15, ld_scales=1 << 10), d=16392) == SHAPE


def test_calls_that_enqueue_nothing():
    assert store(T=0, x=0) == OK and load(T=0, out=0) == OK and norm(T=0, x=0, residual=0) == OK and ffn(T=0, x=0) == OK
    assert norm(idx=P, count=P, max_rows=0) == OK
    assert norm_backward(T=0, dgamma=0, dy=0, h=0) == OK and norm_backward(T=0, accumulate=1, ws=0) == OK
    assert ffn_backward(T=0, dwg=0, dwu=0, ws=0) == OK and ffn_backward(T=0, dw_type=1, accumulate=1, ws=0) == OK


def test_workspaces():
    """Bounded by what they hold, zero for sizes the calls refuse."""
    for T, d in ((1, 8), (1000, 4096), (1 << 20, 16384)):
        n = b.mosaic_rmsnorm_backward_workspace_bytes(T, d)
        assert 4 * d <= n <= 4 * d * max(8, T) and n <= 4 * d * 1024
    assert b.mosaic_rmsnorm_backward_workspace_bytes(5, 100) == 0 and b.mosaic_rmsnorm_backward_workspace_bytes(-1, 8) == 0
    for T, d, F in ((1, 64, 64), (100, 4096, 12288), (131072, 4096, 12288)):
        n, q = (b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, k) for k in (False, True))
        assert 4 * T * F <= n and n + 2 * T * d <= q <= n + 2 * T * d + 256
    assert b.mosaic_gated_ffn_backward_workspace_bytes(131072, 4096, 12288) == 4 * 131072 * 12288   # no partial sums
    assert b.mosaic_gated_ffn_backward_workspace_bytes(4, 100, 64) == 0


def test_a_workspace_serves_fewer_rows():
    for d, F in ((64, 64), (512, 384), (1024, 4096), (4096, 12288)):
        for q8_input in (False, True):
            need = [b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F, q8_input) for T in (*range(0, 9000, 37), 20000, 131072)]
            assert need == sorted(need)
        need = [b.mosaic_rmsnorm_backward_workspace_bytes(T, d) for T in (*range(0, 9000, 37), 20000, 131072)]
        assert need == sorted(need)


def test_the_binding_checks_shapes_and_types():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    w = torch.zeros((128, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device memory"):
        b.mosaic_gated_ffn_forward(x, w, w, torch.zeros((4, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="disagree"):
        b.mosaic_gated_ffn_forward(x, w[:, :32], w[:, :32], torch.zeros((4, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="needed"):
        b.mosaic_rmsnorm_forward(None, None, torch.ones(64), 1e-5, x)
    with pytest.raises(TypeError, match="residual's type"):
        b.mosaic_rmsnorm_forward(x, x, torch.ones(64), 1e-5, x, sum=x.float())
    with pytest.raises(TypeError, match="values"):
        b.Q8Rows(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 1)))
    with pytest.raises(ValueError, match="device memory"):
        b.Q8Rows(torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2)), group=32)
