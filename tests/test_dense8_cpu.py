"""Host-side checks of the 8-bit dense layers (no GPU needed): the library
exports every symbol hpacml8.h declares, the binding's structure matches the
header's, and bad descriptions are refused before any device work."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2407_18352_amd import _abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "hpacml8.h")
FAKE = 0x10000000   # never dereferenced


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(hpacml8_[a-z_]+)\s*\(", text))
    assert names == set(_abi.SIGNATURES8)
    out = subprocess.run(["nm", "-D", "--defined-only", _abi.LIB_PATH], capture_output=True, text=True).stdout
    assert set(re.findall(r"\b(hpacml8_\w+)\b", out)) == names


def test_header_compiles_as_c_and_structures_agree(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "hpacml8.h"\nint main(void) { printf("%zu %zu %d %d", sizeof(hpacml8_checkpoint), '
                   "offsetof(hpacml8_checkpoint, act), HPACML8_BLOCK, HPACML8_MAX_WIDTH); return 0; }")
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(_abi.Checkpoint8), _abi.Checkpoint8.act.offset, _abi.BLOCK8, _abi.MAX_WIDTH8]


def _kept(**more):
    c = _abi.Checkpoint8()
    c.codes, c.exps, c.rows, c.ld_codes, c.ld_exps, c.width, c.act = FAKE, FAKE, 10, 64, 2, 40, _abi.ACT_RELU
    for k, v in more.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("more, status", [
    ({}, _abi.OK), (dict(rows=0), _abi.OK), (dict(rows=-1), _abi.E_INVAL), (dict(width=0), _abi.E_INVAL),
    (dict(act=2), _abi.E_INVAL), (dict(ld_codes=63), _abi.E_INVAL), (dict(ld_codes=80), _abi.E_INVAL),
    (dict(ld_codes=32), _abi.E_INVAL), (dict(ld_exps=1), _abi.E_INVAL), (dict(rows=1 << 40), _abi.E_UNSUPPORTED),
    (dict(width=_abi.MAX_WIDTH8 + 1, ld_codes=1 << 16, ld_exps=1 << 16), _abi.E_UNSUPPORTED),
])
def test_checkpoint_descriptions(more, status):
    n = C.c_size_t()
    assert _abi.lib().hpacml8_backward_scratch(_kept(**more), FAKE, _abi.BF16, 8, 8, 1, 1, C.byref(n)) == status


@pytest.mark.parametrize("kind, lddy, n_out, status", [
    (_abi.F32, 8, 8, _abi.OK), (2, 8, 8, _abi.E_INVAL), (_abi.F32, 7, 8, _abi.E_INVAL), (_abi.F32, 8, 0, _abi.E_INVAL),
    (_abi.F32, 1 << 20, 1 << 20, _abi.E_UNSUPPORTED),
])
def test_backward_descriptions(kind, lddy, n_out, status):
    n = C.c_size_t()
    assert _abi.lib().hpacml8_backward_scratch(_kept(), FAKE, kind, lddy, n_out, 1, 1, C.byref(n)) == status


def test_null_arguments():
    L = _abi.lib()
    n, h = C.c_size_t(), C.c_void_p()
    assert L.hpacml8_backward_scratch(None, FAKE, 0, 8, 8, 1, 1, C.byref(n)) == _abi.E_INVAL
    assert L.hpacml8_backward_scratch(_kept(), FAKE, 0, 8, 8, 1, 1, None) == _abi.E_INVAL
    assert L.hpacml8_linear_create(4, 4, None, None, C.byref(h)) == _abi.E_INVAL and not h.value
    assert L.hpacml8_linear_create(0, 4, FAKE, None, C.byref(h)) == _abi.E_INVAL and not h.value
    assert L.hpacml8_linear_create(4, _abi.MAX_WIDTH8 + 1, FAKE, None, C.byref(h)) == _abi.E_UNSUPPORTED and not h.value
    assert L.hpacml8_linear_create(4, 4, FAKE, None, None) == _abi.E_INVAL
    assert L.hpacml8_linear_scratch(None, 4, C.byref(n)) == _abi.E_INVAL
    assert L.hpacml8_linear_run(None, FAKE, 0, 4, 1, FAKE, 0, 4, 0, FAKE, 0, None) == _abi.E_INVAL
    assert L.hpacml8_checkpoint_save(None, FAKE, 0, 40, None, 0, 0, None) == _abi.E_INVAL
    assert L.hpacml8_checkpoint_load(None, FAKE, 0, 40, None) == _abi.E_INVAL
    L.hpacml8_linear_destroy(None)


SPANS = r"""
#include <cstdio>
#include "span.hpp"
using namespace hpacml;
int main() {
    const char *base = (const char *)0x7f0000000000;
    long long at, rows, pitch, width, size, at2;
    while (std::scanf("%lld %lld %lld %lld %lld %lld", &at, &rows, &pitch, &width, &size, &at2) == 6) {
        const Span s{base + at, rows, pitch, width, false};
        const bool in = inside(s, base, (uint64_t)size);
        std::printf("%d %d\n", in, in && disjoint(s, Span{base + at2, rows, pitch, width, true}));
    }
}
"""


def _compiled(tmp_path, source):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2407_18352_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return lambda text: subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout


def test_operands_against_their_allocations(tmp_path):
    """Inside exactly where the last row's end is, in whole numbers of any
    length: rows times pitch passes 64 bits for 2^31 rows of 2^31 fp32 values."""
    big, cases = 2 ** 31 - 1, []
    for size in (0, 1, 64, 1 << 20, 1 << 38, 1 << 47):
        for at in (0, 1, 63, 64, size - 1, size, size + 1):
            for rows in (1, 2, 3, 1000, 1 << 20, big - 1, big):
                for pitch in (1, 16, 64, 1 << 20, big, 2 * big, 4 * big, 4 * big - 3):
                    for width in {1, min(16, pitch), pitch}:
                        if at >= 0:
                            cases.append((at, rows, pitch, width, size, at + width))
    # the end itself, a byte less, a byte more
    for rows, pitch, width in ((7, 100, 30), (big, 64, 64), (big, 4 * big, 16), (3, 4 * big, 4 * big)):
        for more in (-1, 0, 1):
            size = (rows - 1) * pitch + width + more
            if size < 2 ** 62:
                cases.append((0, rows, pitch, width, size, width))
    out = _compiled(tmp_path, SPANS)("".join("%d %d %d %d %d %d\n" % c for c in cases)).split("\n")
    accepted = 0
    for c, line in zip(cases, out):
        at, rows, pitch, width, size, at2 = c
        fits = at + (rows - 1) * pitch + width <= size
        # the second begins `width` after the first: beside it in its rows or past its end
        apart = fits and (rows == 1 or 2 * width <= pitch)
        assert line == "%d %d" % (fits, apart), c
        accepted += fits
    assert len(out) == len(cases) + 1 and accepted > 300


FORMS = r"""
#include <cstdio>
#include "dense8_rules.hpp"
using namespace hpacml;
int main() {
    long rows, n_in, n_out;
    int planes;
    while (std::scanf("%ld %ld %ld %d", &rows, &n_in, &n_out, &planes) == 4) {
        const DwForm f = choose_dw(rows, (int)n_out, (int)n_in, planes);
        const int dx = (int)nt::tile_for(n_in, rows, (2 * n_out + 63) / 64 * (planes * (planes + 1) / 2));
        std::printf("%d %d %d %ld %d\n", few_rows(rows, (int)n_out, (int)n_in), f.tile, f.splits, (long)f.rows_per_split / 32, dx);
    }
    std::printf("%zu\n", sizeof(kDwTiles) / sizeof(kDwTiles[0]));
}
"""


def test_the_exact_tests_reach_every_form(tmp_path):
    """Of dw: each tile of the table with four slabs of rows or more (its rings
    go round), in one type at least each with the rows in one part, in several
    and in many; of dx: each tile, in both types; the one launch for few rows."""
    from test_gpu_dense8_exact import GENERAL, SHAPES
    run = _compiled(tmp_path, FORMS)

    def forms(shapes, planes):
        lines = run("".join("%d %d %d %d\n" % (s + (planes,)) for s in shapes)).split("\n")
        return [tuple(map(int, l.split())) for l in lines[:len(shapes)]], int(lines[len(shapes)])

    parts = lambda splits: 0 if splits == 1 else 1 if splits < 16 else 2
    seen = set()
    for planes in (1, 3):
        got, tiles = forms(SHAPES, planes)
        general = [f for f in got if not f[0]]
        assert len(got) - len(general) >= 3
        long = {t for _, t, _, slabs, _ in general if slabs >= 4}
        # three planes at once are of fp32 alone
        assert long == ({0, 1, 2, 3, 4} if planes == 1 else set(range(tiles))), (planes, long)
        whole = [n_in % 32 == 0 for _, n_in, _ in SHAPES]      # dx in whole cache lines, and not
        for lines in (True, False):
            assert {f[4] for f, w in zip(got, whole) if not f[0] and w == lines} == {0, 1, 2, 3}, (planes, lines)
        seen |= {(t, parts(splits)) for _, t, splits, slabs, _ in general}
        few, t = forms(GENERAL, planes)
        assert not any(f[0] for f in few) and {parts(f[2]) for f in few} == {0, 1, 2}, few
    assert tiles == 7 and {t for t, _ in seen} == set(range(7)) and {p for _, p in seen} == {0, 1, 2}
    # the largest tile, which large batches take, with its parts joined by one thread and by many
    assert {p for t, p in seen if t == 0} == {0, 1, 2}


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_the_exact_tests_tell_a_lost_slab(kind):
    """Any 32 rows that do not take part, or take part twice, change dw."""
    import torch
    from test_gpu_dense8_exact import RELU, results, whole_numbers
    for shape in ((70001, 64, 8), (100003, 35, 5), (3001, 150, 47)):
        codes, exps, dy, W = whole_numbers(*shape, kind, RELU, "cpu")
        a, dw, db, _ = results(codes, exps, dy, W, RELU)
        rows = -(-shape[0] // 32) * 32
        pad = lambda t: torch.nn.functional.pad(t.double(), (0, 0, 0, rows - shape[0])).view(rows // 32, 32, -1)
        slabs = torch.matmul(pad(dy).transpose(1, 2).contiguous(), pad(a))
        assert torch.equal(slabs.sum(0), dw) and (slabs != 0).any(2).any(1).all()
