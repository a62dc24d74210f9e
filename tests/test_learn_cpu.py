"""Host-side checks of the layers in 8-bit floating point, group norm and the
gradients' norm (no GPU needed): the library exports every symbol hpacmlt.h
declares, the binding's structures match the header's, and bad calls are refused
before any device work."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest

from paper_2407_18352_amd import _abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "hpacmlt.h")
FAKE = 0x10000000   # never dereferenced
L = _abi.lib()
BIG = 1 << 40


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(hpacmlt_[a-z_]+)\s*\(", text))
    assert names == set(_abi.SIGNATURES_T)
    out = subprocess.run(["nm", "-D", "--defined-only", _abi.LIB_PATH], capture_output=True, text=True).stdout
    assert set(re.findall(r"\b(hpacmlt_\w+)\b", out)) == names


def test_header_compiles_as_c_and_structures_agree(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hpacmlt.h"\nint main(void) { printf("%zu %zu %zu %zu %d %d %d %d", '
                   "sizeof(hpacmlt_matrix), offsetof(hpacmlt_matrix, width), sizeof(hpacmlt_gradient), "
                   "offsetof(hpacmlt_gradient, to_dtype), HPACMLT_BLOCK, HPACMLT_MAX_CHANNELS, HPACMLT_ACT_SILU, HPACMLT_NORM_MAX); return 0; }")
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(_abi.Matrix), _abi.Matrix.width.offset, C.sizeof(_abi.Gradient), _abi.Gradient.to_dtype.offset, _abi.BLOCKF8,
                   _abi.MAX_CHANNELS, _abi.ACT_SILU, _abi.NORM_MAX]


@pytest.mark.parametrize("rows, width, codes, scales", [(0, 0, 0, 0), (1, 1, 4096, 128), (32, 128, 4096, 128), (33, 129, 16384, 256),
                                                       (129, 128, 5 * 4096, 256), (0, 700, 0, 0), (700, 0, 0, 0)])
def test_matrix_bytes(rows, width, codes, scales):
    c, s = C.c_size_t(), C.c_size_t()
    assert L.hpacmlt_matrix_bytes(rows, width, c, s) == _abi.OK and (c.value, s.value) == (codes, scales)


def test_matrix_descriptions():
    c, s = C.c_size_t(), C.c_size_t()
    assert L.hpacmlt_matrix_bytes(-1, 5, c, s) == _abi.E_INVAL and L.hpacmlt_matrix_bytes(5, -1, c, s) == _abi.E_INVAL
    assert L.hpacmlt_matrix_bytes(BIG, 5, c, s) == _abi.E_UNSUPPORTED and L.hpacmlt_matrix_bytes(5, BIG, c, s) == _abi.E_UNSUPPORTED
    assert L.hpacmlt_matrix_bytes(5, 5, None, s) == _abi.E_INVAL


@pytest.mark.parametrize("rows, width, status", [(1 << 31, 1, _abi.E_UNSUPPORTED), ((1 << 31) - 1, 1, _abi.E_UNSUPPORTED), ((1 << 31) - 128, 128, _abi.OK),
                                                 ((1 << 30) + 1, 129, _abi.E_UNSUPPORTED), (1 << 24, 1 << 14, _abi.E_UNSUPPORTED), (1 << 24, (1 << 14) - 128, _abi.OK)])
def test_fewer_blocks_than_a_launch_has(rows, width, status):
    c, s = C.c_size_t(), C.c_size_t()
    assert L.hpacmlt_matrix_bytes(rows, width, c, s) == status and L.hpacmlt_matrix_bytes(width, rows, c, s) == status
    assert L.hpacmlt_backward_scratch(rows, 5, width, 0, 1, 0, c) == status
    assert L.hpacmlt_linear_scratch(matrix(9, width), rows, c) == status
    if status != _abi.OK:
        assert L.hpacmlt_quantize(FAKE, _abi.F32, width, rows, width, matrix(rows, width), None, 0, None) == status
        assert L.hpacmlt_load(matrix(rows, width), FAKE, _abi.F32, width, None) == status


def matrix(rows, width):
    return _abi.Matrix(FAKE, FAKE + (1 << 20), rows, width)


@pytest.mark.parametrize("more, status", [
    (dict(dtype=2), _abi.E_INVAL), (dict(rows=-1), _abi.E_INVAL), (dict(ldx=19), _abi.E_INVAL), (dict(by_row=None, by_column=None), _abi.E_INVAL),
    (dict(rows=BIG), _abi.E_UNSUPPORTED), (dict(by_row=matrix(10, 21)), _abi.E_SHAPE), (dict(by_row=matrix(20, 10)), _abi.E_SHAPE),
    (dict(by_column=matrix(10, 20)), _abi.E_SHAPE), (dict(by_row=matrix(-1, 20)), _abi.E_INVAL),
    (dict(rows=0, by_row=matrix(0, 20), by_column=None), _abi.OK)])
def test_quantize_refusals(more, status):
    a = dict(dtype=_abi.F32, ldx=20, rows=10, width=20, by_row=matrix(10, 20), by_column=matrix(20, 10)) | more
    assert L.hpacmlt_quantize(FAKE, a["dtype"], a["ldx"], a["rows"], a["width"], a["by_row"], a["by_column"], 0, None) == status


@pytest.mark.parametrize("more, status", [
    (dict(dtype=5), _abi.E_INVAL), (dict(act=2), _abi.E_INVAL), (dict(ldy=8), _abi.E_INVAL), (dict(q=matrix(9, 301)), _abi.E_SHAPE),
    (dict(accumulate=1, dtype=_abi.BF16), _abi.E_INVAL), (dict(accumulate=1, b=FAKE), _abi.E_INVAL), (dict(accumulate=1, act=_abi.ACT_RELU), _abi.E_INVAL),
    (dict(p=matrix(100, 30000), q=matrix(9, 30000)), _abi.E_RANGE), (dict(p=matrix(0, 300)), _abi.OK), (dict(q=matrix(0, 300)), _abi.OK)])
def test_product_refusals(more, status):
    a = dict(p=matrix(10, 300), q=matrix(9, 300), b=None, act=_abi.ACT_IDENTITY, dtype=_abi.F32, ldy=9, accumulate=0) | more
    assert L.hpacmlt_product(a["p"], a["q"], a["b"], a["act"], FAKE, a["dtype"], a["ldy"], a["accumulate"], None, 0, None) == status


@pytest.mark.parametrize("more, status", [
    (dict(xt=3), _abi.E_INVAL), (dict(yt=-1), _abi.E_INVAL), (dict(act=_abi.ACT_SILU), _abi.E_INVAL), (dict(rows=-1), _abi.E_INVAL), (dict(ldx=299), _abi.E_INVAL),
    (dict(ldy=8), _abi.E_INVAL), (dict(W=matrix(0, 300)), _abi.E_INVAL), (dict(rows=BIG), _abi.E_UNSUPPORTED), (dict(keep=matrix(300, 99)), _abi.E_SHAPE),
    (dict(keep=matrix(100, 300)), _abi.E_SHAPE), (dict(bytes=1000), _abi.E_RANGE), (dict(rows=0, keep=matrix(300, 0)), _abi.OK)])
def test_linear_refusals(more, status):
    a = dict(W=matrix(9, 300), xt=_abi.F32, ldx=300, rows=100, yt=_abi.BF16, ldy=9, act=_abi.ACT_RELU, keep=None, bytes=0) | more
    assert L.hpacmlt_linear_run(a["W"], None, FAKE, a["xt"], a["ldx"], a["rows"], FAKE, a["yt"], a["ldy"], a["act"], a["keep"], FAKE, a["bytes"],
                                None) == status
    n = C.c_size_t()
    assert L.hpacmlt_linear_scratch(None, 5, n) == _abi.E_INVAL and L.hpacmlt_linear_scratch(matrix(9, 300), 5, None) == _abi.E_INVAL


@pytest.mark.parametrize("more, status", [
    (dict(dtype=2), _abi.E_INVAL), (dict(n_out=0), _abi.E_INVAL), (dict(lddy=8), _abi.E_INVAL), (dict(y=FAKE, ldy=8), _abi.E_INVAL),
    (dict(dw=None, db=None, dx=None), _abi.E_INVAL), (dict(lddw=299), _abi.E_INVAL), (dict(lddx=299), _abi.E_INVAL), (dict(Wt=None), _abi.E_INVAL),
    (dict(Wt=matrix(9, 300)), _abi.E_SHAPE), (dict(kept=matrix(0, 100)), _abi.E_INVAL), (dict(bytes=1000), _abi.E_RANGE)])
def test_backward_refusals(more, status):
    a = dict(kept=matrix(300, 100), y=None, dtype=_abi.F32, lddy=9, ldy=9, n_out=9, Wt=matrix(300, 9), dw=FAKE, lddw=300, db=FAKE, dx=FAKE, lddx=300,
             bytes=0) | more
    assert L.hpacmlt_backward(a["kept"], FAKE, a["y"], a["dtype"], a["lddy"], a["ldy"], a["n_out"], a["Wt"], a["dw"], a["lddw"], a["db"], a["dx"], a["lddx"],
                              0, FAKE, a["bytes"], None) == status


NORM = dict(dtype=_abi.F32, ld=24, images=3, points=50, channels=24, groups=4, eps=1e-5, act=_abi.ACT_SILU, mean=FAKE, rstd=FAKE, bytes=1 << 30)


@pytest.mark.parametrize("more, status", [
    (dict(dtype=7), _abi.E_INVAL), (dict(images=-1), _abi.E_INVAL), (dict(points=0), _abi.E_INVAL), (dict(channels=0), _abi.E_INVAL), (dict(groups=0), _abi.E_INVAL),
    (dict(groups=5), _abi.E_INVAL), (dict(ld=23), _abi.E_INVAL), (dict(act=3), _abi.E_INVAL), (dict(eps=0.0), _abi.E_INVAL), (dict(eps=-1.0), _abi.E_INVAL),
    (dict(eps=math.nan), _abi.E_INVAL), (dict(eps=2.0 ** -127), _abi.E_INVAL), (dict(eps=math.inf), _abi.E_INVAL), (dict(mean=None), _abi.E_INVAL),
    (dict(channels=32768, ld=32768), _abi.E_UNSUPPORTED), (dict(images=1 << 20, points=1 << 20), _abi.E_UNSUPPORTED),
    (dict(points=100000, bytes=0), _abi.E_RANGE), (dict(images=0), _abi.OK)])
def test_group_norm_refusals(more, status):
    a = NORM | more
    assert L.hpacmlt_group_norm(FAKE, a["dtype"], a["ld"], a["images"], a["points"], a["channels"], a["groups"], None, None, a["eps"], a["act"], FAKE, a["ld"],
                                a["mean"], a["rstd"], FAKE, a["bytes"], None) == status
    if status != _abi.OK and not {"eps", "mean"} & set(more):
        assert L.hpacmlt_group_norm_backward(FAKE, a["dtype"], a["ld"], a["images"], a["points"], a["channels"], a["groups"], None, None, a["act"], FAKE, FAKE,
                                             FAKE, a["ld"], FAKE, a["ld"], FAKE, FAKE, 0, FAKE, a["bytes"], None) == status


def test_group_norm_backward_wants_something():
    a = NORM
    assert L.hpacmlt_group_norm_backward(FAKE, a["dtype"], a["ld"], a["images"], a["points"], a["channels"], a["groups"], None, None, a["act"], FAKE, FAKE, FAKE,
                                         a["ld"], None, 0, None, None, 0, FAKE, a["bytes"], None) == _abi.E_INVAL


def test_gradient_refusals():
    h, n = C.c_void_p(), C.c_size_t()
    assert L.hpacmlt_gradients_create(None, 3, h) == _abi.E_INVAL and L.hpacmlt_gradients_create(None, -1, h) == _abi.E_INVAL
    assert L.hpacmlt_gradients_create(None, 0, None) == _abi.E_INVAL
    assert L.hpacmlt_gradients_scratch(None, n) == _abi.E_INVAL
    assert L.hpacmlt_gradients_norm(None, 0, FAKE, FAKE, 1 << 20, None) == _abi.E_INVAL
    assert L.hpacmlt_gradients_clip(None, 0, math.nan, FAKE, FAKE, 1 << 20, None) == _abi.E_INVAL
    assert L.hpacmlt_gradients_clip(None, 0, 1.0, FAKE, FAKE, 1 << 20, None) == _abi.E_INVAL
    L.hpacmlt_gradients_destroy(None)
