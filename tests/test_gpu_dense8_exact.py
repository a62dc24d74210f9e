"""The backward pass on whole numbers: every partial sum is exact in fp32, in
whichever order, so the results equal the 64-bit ones bit by bit, and a part of
the rows, a term or a block that is lost, doubled or misplaced shows at any size.
The shapes reach every form that the sizes choose among (checked without a GPU
in test_dense8_cpu.py)."""
import pytest
import torch

from paper_2407_18352_amd import _abi, api
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

RELU, IDENT = _abi.ACT_RELU, _abi.ACT_IDENTITY
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}

# (rows, inputs, outputs)
SHAPES = [
    (200, 50, 70), (1, 1, 1), (1024, 40, 300), (33, 1000, 260),                                     # one launch
    (12042, 1, 1), (100003, 35, 5), (70001, 64, 8), (20000, 256, 128), (1039, 362, 303),            # dw by small tiles
    (38343, 1, 129), (132, 3767, 161), (260, 2716, 201), (1025, 40, 70),
    (3001, 2050, 2047), (3677, 2429, 1035), (146024, 137, 132), (132, 3844, 2054), (11332, 131, 1153),    # 256 x 256
    (1601, 844, 1158), (787, 577, 1603), (2695, 2, 3814), (4096, 1024, 2048),                       # 256 x 128
    (1754, 879, 1156), (864, 1794, 520), (130, 4661, 1568),                                         # 128 x 256
    (2691, 1292, 1807), (150476, 65, 68), (62557, 66, 65), (2046, 2611, 275), (131, 4950, 1550),    # 128 x 128
    (130, 2189, 1359), (300, 2048, 2048),                                                           # the same, three planes at once
    (25100, 1024, 130), (3001, 2048, 100),                                                          # dx in whole cache lines
]
# of the general form, with the rows in many parts, in several and in one
GENERAL = [(20000, 96, 72), (1100, 96, 72), (1039, 362, 303), (132, 3844, 2054)]


def whole_numbers(rows, n_in, n_out, kind, act, device):
    """(codes, exponents, dy, W) whose sums of products stay below 2^24.  In fp32
    some values need two (257) or three (65793) bf16 terms, dy's in the first
    half of the outputs and W's in the second."""
    g = torch.Generator(device=device).manual_seed(rows + 3 * n_in + 5 * n_out)
    ints = lambda lo, hi, shape: torch.randint(lo, hi + 1, shape, generator=g, device=device)
    blocks = -(-n_in // 32)
    codes = ints(0, 3, (rows, blocks * 32)) if act == RELU else ints(-3, 3, (rows, blocks * 32)) + 128
    exps = ints(127, 128, (rows, blocks))
    dy, W = ints(-2, 2, (rows, n_out)).float(), ints(-1, 1, (n_out, n_in)).float()
    if kind == "f32":
        half = n_out - n_out // 2

        def longer(t, chance):
            at = torch.rand(t.shape, generator=g, device=device) < chance
            t[at] = torch.tensor([257.0, -257.0, 65793.0, -65793.0], device=device)[ints(0, 3, (int(at.sum()),))]

        longer(dy[:, :half], min(0.3, 20 / rows))
        longer(W[half:], min(0.3, 20 / n_out))
        dy[:, 0].clamp_(-257, 257)         # 257 x 257: the product of two second terms
        W[0] *= 257
    return codes.to(torch.uint8), exps.to(torch.uint8), dy.to(KINDS[kind]), W.to(KINDS[kind])


def results(codes, exps, dy, W, act):
    """What the codes stand for, dw, db and dx, in 64 bits; every sum of
    magnitudes is checked to be exact in fp32."""
    n_in, c = W.shape[1], codes.double() - (0 if act == RELU else 128)
    a = (c * torch.exp2(exps.double() - 127).repeat_interleave(32, 1))[:, :n_in].contiguous()
    g, w = dy.double(), W.double()
    for left, right in ((g.t().contiguous(), a), (g, w)):
        assert float((left.abs() @ right.abs()).max()) < 2 ** 23      # and twice as much below 2^24
    dx = g @ w
    if act == RELU:
        dx[codes[:, :n_in] == 0] = 0
    return a, g.t().contiguous() @ a, g.sum(0), dx


def _data(shape, kind, act):
    codes, exps, dy, W = whole_numbers(*shape, kind, act, "cuda")
    kept = api.Checkpoint8(shape[0], shape[1], act, codes, exps)
    return (kept, dy, W) + results(codes, exps, dy, W, act)[1:]


def _outputs(shape, kind):
    rows, n_in, n_out = shape
    full = lambda n, m, t: torch.full((n + 2, m + 3), -77.0, dtype=t, device="cuda")
    wide_w, wide_x, wide_b = full(n_out, n_in, torch.float32), full(rows, n_in, KINDS[kind]), full(0, n_out, torch.float32)[0]
    return (wide_w, wide_b, wide_x), (wide_w[1:-1, :n_in], wide_b[:n_out], wide_x[1:-1, :n_in])


def _beside_untouched(wide, shape):
    (w, b, x), (rows, n_in, n_out) = wide, shape
    for t, width in ((w, n_in), (x, n_in)):
        assert (t[0] == -77).all() and (t[-1] == -77).all() and (t[:, width:] == -77).all()
    assert (b[n_out:] == -77).all()


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", [RELU, IDENT])
def test_results_are_exact(shape, kind, act):
    kept, dy, W, dw, db, dx = _data(shape, kind, act)
    wide, (gw, gb, gx) = _outputs(shape, kind)
    api.backward8(kept, dy, gw, gb, W=W, dx=gx)
    assert torch.equal(gw.double(), dw) and torch.equal(gb.double(), db)
    assert torch.equal(gx.double(), dx.float().to(KINDS[kind]).double())
    api.backward8(kept, dy, gw, gb, accumulate=True)
    assert torch.equal(gw.double(), 2 * dw) and torch.equal(gb.double(), 2 * db)
    _beside_untouched(wide, shape)
    # rows after one another: whole cache lines where the width is one of theirs
    gw, gx = torch.empty((shape[2], shape[1]), device="cuda"), torch.empty(shape[:2], dtype=KINDS[kind], device="cuda")
    api.backward8(kept, dy, gw, gb, W=W, dx=gx)
    assert torch.equal(gw.double(), dw) and torch.equal(gx.double(), dx.float().to(KINDS[kind]).double())


@pytest.mark.parametrize("shape", GENERAL, ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("parts", [("dw",), ("db",), ("dx",), ("dw", "db"), ("dw", "dx"), ("db", "dx")])
def test_wanted_parts_of_many_rows(shape, kind, accumulate, parts):
    kept, dy, W, dw, db, dx = _data(shape, kind, RELU)
    wide, out = _outputs(shape, kind)
    given = {n: t if n in parts else None for n, t in zip(("dw", "db", "dx"), out)}
    for t in out[:2]:
        t.fill_(5.0)
    api.backward8(kept, dy, given["dw"], given["db"], W=W, dx=given["dx"], accumulate=accumulate)
    for name, t, want in zip(("dw", "db", "dx"), out, (dw, db, dx.float().to(KINDS[kind]))):
        if name not in parts:
            assert (t == (-77.0 if name == "dx" else 5.0)).all()
        else:
            assert torch.equal(t.double(), want.double() + (5 if accumulate and name != "dx" else 0))
    _beside_untouched(wide, shape)


@pytest.mark.parametrize("rows", [1100, 40000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows_in_accumulated_batches(rows, kind):
    """Batches of the general form and a last one of the other, added up."""
    shape = (rows * 2 + 70, 100, 60)
    kept, dy, W, dw, db, _ = _data(shape, kind, RELU)
    gw, gb = torch.zeros((60, 100), device="cuda"), torch.zeros(60, device="cuda")
    for at in (slice(0, rows), slice(rows, 2 * rows), slice(2 * rows, shape[0])):
        part = api.Checkpoint8(at.stop - at.start, 100, RELU, kept.codes[at], kept.exps[at])
        api.backward8(part, dy[at], gw, gb, accumulate=True)
    assert torch.equal(gw.double(), dw) and torch.equal(gb.double(), db)


# outputs: multiples of 32, of 8 alone, of neither (dy in place for dx and dw, for dw alone, laid out)
@pytest.mark.parametrize("n_out", [64, 72, 61])
@pytest.mark.parametrize("off", [0, 1, 4, 8])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("want_dx", [False, True])
def test_many_rows_at_any_alignment_beside_nan(n_out, off, kind, want_dx):
    """dy and W begin at any element of wider rows, with NaN around them; so do
    dx and dw; the codes' padding is anything."""
    shape = (1300, 70, n_out)
    kept, dy, W, dw, db, dx = _data(shape, kind, RELU)

    def inside(t, more):
        wide = torch.full((t.shape[0] + 2, t.shape[1] + more), float("nan"), dtype=t.dtype, device="cuda")
        wide[1:-1, off:off + t.shape[1]] = t
        return wide[1:-1, off:off + t.shape[1]]

    kept.codes[:, 70:] = torch.randint(0, 256, kept.codes[:, 70:].shape, dtype=torch.uint8, device="cuda")
    for more in (8 + off, 31 + off):
        gw, gx = inside(torch.zeros((n_out, 70), device="cuda"), more), inside(torch.zeros((1300, 70), dtype=KINDS[kind], device="cuda"), more)
        gb = torch.empty(n_out, device="cuda")
        api.backward8(kept, inside(dy, more), gw, gb, W=inside(W, more), dx=gx if want_dx else None)
        assert torch.equal(gw.double(), dw) and torch.equal(gb.double(), db)
        assert torch.equal(gx.double(), dx.float().to(KINDS[kind]).double()) if want_dx else not gx.any()
        around = [t._base.double() for t in (gw, gx)]
        for t, v in zip(around, (gw, gx)):
            assert int(torch.isnan(t).sum()) == t.numel() - v.numel()


@pytest.mark.parametrize("rows, n_in, n_out", [(100, 600, 64), (2048, 1024, 1024), (5000, 600, 1024), (13001, 1040, 1088), (12, 70, 96)])
@pytest.mark.parametrize("x_kind, y_kind", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_linear_into_rows_of_whole_cache_lines(rows, n_in, n_out, x_kind, y_kind):
    """The same bits as into rows that share their cache lines, which are checked
    against the definition."""
    from test_gpu_dense8 import _check_linear, _rand
    x, W, b = _rand(61, (rows, n_in), x_kind), _rand(62, (n_out, n_in)), _rand(63, (1, n_out))[0]
    _check_linear(x, W, b, RELU, y_kind)
    layer = api.Linear8(W, b)
    lines = torch.empty((rows, n_out), dtype=KINDS[y_kind], device="cuda")
    shared = torch.empty((rows, n_out + 1), dtype=KINDS[y_kind], device="cuda")[:, :n_out]
    api.linear8(layer, x, lines, RELU)
    api.linear8(layer, x, shared, RELU)
    assert lines.data_ptr() % 64 == 0 and torch.equal(lines, shared)
