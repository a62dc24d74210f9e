"""Dense layers in 8 bits against plain computations in 64 bits: the integer
product with scales per row and per output, activations kept in 8 bits, and
the backward pass that reads them."""
import numpy as np
import pytest

from paper_2407_18352_amd import _abi, api
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

RELU, IDENT = _abi.ACT_RELU, _abi.ACT_IDENTITY
EPS32, EPSBF = 2.0 ** -24, 2.0 ** -8
EPS_SUM = 2.0 ** -23     # one addition of the matrix instruction, whichever way it rounds


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _torch():
    import torch
    return torch


def _dtype(kind):
    torch = _torch()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[kind]


def _rand(seed, shape, kind="f32", pad=0, scale=1.0):
    """Device matrix of normal values inside rows of width + pad."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.randn((shape[0], shape[1] + pad), generator=g, device="cuda") * scale
    return t.to(_dtype(kind))[:, :shape[1]]


def _guarded(rows, width, kind, pad=5):
    """An output of `rows` rows inside a larger tensor whose other elements
    must stay as they are."""
    torch = _torch()
    whole = torch.full((rows + 2, width + pad), -77.0, dtype=_dtype(kind), device="cuda")
    return whole, whole[1:rows + 1, :width]


def _untouched(whole, rows, width):
    w = whole.float().cpu().numpy()
    assert (w[0] == -77).all() and (w[rows + 1:] == -77).all() and (w[1:rows + 1, width:] == -77).all()


def _np(t):
    return t.detach().to(_torch().float64).cpu().numpy()


# ---- y = act(x W^T + b) -------------------------------------------------------


def _codes(v):
    """Codes and scales of each row: the codes are decisions of fp32
    arithmetic (one division, one product, one rounding), so they are formed
    in it here too; the rest is 64-bit."""
    v = np.asarray(v, np.float32)
    top = np.abs(v).max(axis=1, keepdims=True)
    ok = np.isfinite(top) & (top >= np.float32(2.0 ** -119))
    safe = np.where(ok, top, np.float32(1))
    q = np.rint(np.where(ok, v, np.float32(0)) * (np.float32(127) / safe))
    s = np.where(ok, (safe / np.float32(127)).astype(np.float64), 0.0)
    return q.astype(np.float64), np.where(np.isfinite(top), s, np.nan)


def _linear(x, W, b, act):
    (q, s), (w, t) = _codes(x), _codes(W)
    y = (q @ w.T) * s * t.T
    size = np.abs(y) + (0 if b is None else np.abs(b))
    if b is not None:
        y = y + np.asarray(b, np.float64)
    if act == RELU:
        y = np.where(y < 0, 0, y)
    return y, size


def _check_linear(x, W, b, act, y_kind, what=""):
    torch = _torch()
    rows, n_out = x.shape[0], W.shape[0]
    layer = api.Linear8(W, b)
    whole, y = _guarded(rows, n_out, y_kind)
    api.linear8(layer, x, y, act)
    torch.cuda.synchronize()
    want, size = _linear(x.float().cpu().numpy(), _np(W).astype(np.float32), None if b is None else _np(b), act)
    got = _np(y)
    # the sum is exact; then the sum as fp32, two scales, two products and the
    # bias: six roundings of at most 2^-24, and one to y's type
    tol = 6 * EPS32 * size + (EPSBF if y_kind == "bf16" else 0) * np.abs(want) + 1e-37
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), what
    bad = np.abs(got - want) > tol
    assert not bad[~nan].any(), "%s: %d of %d off, worst %g" % (what, bad.sum(), bad.size, np.nanmax(np.abs(got - want)))
    _untouched(whole, rows, n_out)
    layer.close()


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 16, 17, 33, 63, 64, 65, 130, 257, 1000])
@pytest.mark.parametrize("n_in, n_out", [(1, 1), (5, 3), (64, 64), (127, 129), (128, 256), (200, 50), (513, 70)])
def test_linear_sizes(rows, n_in, n_out):
    W = _rand(2, (n_out, n_in), scale=n_in ** -0.5)
    b = _rand(3, (1, n_out))[0]
    kind = ("f32", "bf16")[(rows + n_in) % 2]
    _check_linear(_rand(1, (rows, n_in), kind, pad=rows % 4), W, b, (RELU, IDENT)[rows % 2], ("bf16", "f32")[n_out % 2])


@pytest.mark.parametrize("rows, n_in, n_out", [(1, 4096, 4096), (7, 4096, 1000), (300, 4096, 512), (1100, 1024, 2048),
                                               (4099, 512, 512), (1, 16384, 33), (3, 33, 16384), (20011, 96, 40)])
@pytest.mark.parametrize("x_kind, y_kind", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_linear_larger(rows, n_in, n_out, x_kind, y_kind):
    _check_linear(_rand(4, (rows, n_in), x_kind), _rand(5, (n_out, n_in), scale=n_in ** -0.5), None, IDENT, y_kind)


@pytest.mark.parametrize("rows, n_in, n_out", [(13001, 1040, 1100), (12950, 1024, 1088), (50011, 70, 1300), (25100, 130, 1024)])
@pytest.mark.parametrize("x_kind, y_kind", [("bf16", "bf16"), ("f32", "f32")])
def test_linear_in_the_largest_tiles(rows, n_in, n_out, x_kind, y_kind):
    """Enough of them for every CU; rows whose ends share cache lines and rows
    whose ends do not."""
    _check_linear(_rand(24, (rows, n_in), x_kind), _rand(25, (n_out, n_in), scale=n_in ** -0.5), None, RELU, y_kind)


@pytest.mark.parametrize("rows, n_in, n_out", [(32768, 5, 16), (32769, 64, 64), (33001, 65, 65), (40000, 201, 50), (32770, 256, 128),
                                               (32768, 257, 130), (33007, 320, 300), (32801, 512, 512), (32768, 511, 1024),
                                               (32790, 512, 1025), (32768, 513, 100), (131073, 40, 33), (131100, 130, 127)])
@pytest.mark.parametrize("x_kind, y_kind", [("bf16", "bf16"), ("f32", "f32")])
def test_linear_many_rows_of_narrow_layers(rows, n_in, n_out, x_kind, y_kind):
    _check_linear(_rand(40, (rows, n_in), x_kind, pad=rows % 5), _rand(41, (n_out, n_in), scale=n_in ** -0.5),
                  _rand(42, (1, n_out))[0], RELU, y_kind)


@pytest.mark.parametrize("x_kind", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1, 4, 8])
def test_linear_alignment(x_kind, pad):
    """Rows that begin at any element of a wider record."""
    for off in (0, 1, 3):
        wide = _rand(6, (77, 65 + pad + off), x_kind)
        _check_linear(wide[:, off:off + 65], _rand(7, (40, 65)), None, RELU, "f32", "pad %d offset %d" % (pad, off))


@pytest.mark.parametrize("rows", [1, 4, 40, 300, 33000])
def test_linear_special_rows(rows):
    """Rows of zeros, of tiny and of huge values, with an infinity or a NaN;
    the same in the weights."""
    torch = _torch()
    x, W = _rand(8, (rows, 70)).clone(), _rand(9, (50, 70)).clone()
    inf, nan = float("inf"), float("nan")
    for i, v in enumerate([None, 0.0, 1e-37, 1e-45, 1e30, inf, -inf, nan]):
        if v is None:
            continue
        if i < rows:
            x[i] = 0 if v == 0.0 else x[i].sign() * v if abs(v) < 1 else x[i]
            if v != v or abs(v) >= 1:
                x[i, 69 - i] = v
    W[3] = 0
    W[17] = W[17].sign() * 1e-40
    W[49, 0] = nan
    for act in (RELU, IDENT):
        _check_linear(x, W, _rand(10, (1, 50))[0], act, "f32")
    y = torch.empty((rows, 50), device="cuda")
    layer = api.Linear8(W)
    api.linear8(layer, x, y, RELU)
    assert torch.isnan(y[:, 49]).all()


def test_linear_codes_hold_the_largest_sum():
    """All codes at +-127 over the widest input: the 32-bit sum is exact."""
    torch = _torch()
    x = torch.full((2, 16384), 3.0, device="cuda")
    x[1] = -x[1]
    W = torch.full((3, 16384), 0.5, device="cuda")
    W[2, 1] = -0.5
    _check_linear(x, W, None, IDENT, "f32")


def test_linear_ties_round_to_even():
    torch = _torch()
    x = torch.zeros((1, 64), device="cuda")
    x[0, :5] = torch.tensor([127.0, 0.5, 1.5, 2.5, -3.5], device="cuda")
    y = torch.empty((1, 64), device="cuda")
    api.linear8(api.Linear8(torch.eye(64)), x, y)
    assert y[0, :5].tolist() == [127.0, 0.0, 2.0, 2.0, -4.0]


def test_linear_weights_from_host_and_device_agree():
    torch = _torch()
    W, b, x = _rand(11, (60, 90)), _rand(12, (1, 60))[0], _rand(13, (50, 90))
    ys = []
    for w, c in ((W, b), (W.cpu(), b.cpu()), (W.cpu().numpy(), b.cpu().numpy())):
        y = torch.empty((50, 60), device="cuda")
        api.linear8(api.Linear8(w, c), x, y, RELU)
        ys.append(y)
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


def test_linear_in_columns_of_one_record():
    """x and y interleaved in the rows of one record."""
    torch = _torch()
    rec = _rand(14, (100, 40)).clone()
    W = _rand(15, (7, 33))
    want = torch.empty((100, 7), device="cuda")
    layer = api.Linear8(W)
    api.linear8(layer, rec[:, :33].clone(), want)
    before = rec.clone()
    api.linear8(layer, rec[:, :33], rec[:, 33:])
    assert torch.equal(rec[:, 33:], want) and torch.equal(rec[:, :33], before[:, :33])


def test_linear_streams_and_repeats():
    """A stream of its own, scratch of its own; equal calls give equal bits."""
    torch = _torch()
    x, W = _rand(16, (5000, 300), "bf16"), _rand(17, (200, 300))
    layer, outs = api.Linear8(W), []
    torch.cuda.synchronize()
    for _ in range(3):
        s = torch.cuda.Stream()
        y = torch.empty((5000, 200), device="cuda")
        scratch = torch.empty(layer.scratch_bytes(5000), dtype=torch.uint8, device="cuda").fill_(0xA5)
        torch.cuda.synchronize()
        api.linear8(layer, x, y, RELU, scratch=scratch, stream=s)
        s.synchronize()
        outs.append(y)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_linear_refusals():
    torch = _torch()
    L = _abi.lib()
    layer = api.Linear8(_rand(18, (8, 16)))
    x, y = _rand(19, (4, 16)), torch.empty((4, 8), device="cuda")
    s = torch.empty(layer.scratch_bytes(4), dtype=torch.uint8, device="cuda")
    h, st = layer.handle, torch.cuda.current_stream().cuda_stream

    def run(x=x.data_ptr(), xt=0, ldx=16, n=4, y=y.data_ptr(), yt=0, ldy=8, act=0, s=s.data_ptr(), sb=s.numel()):
        return L.hpacml8_linear_run(h, x, xt, ldx, n, y, yt, ldy, act, s, sb, st)

    assert run() == _abi.OK
    assert run(n=0) == _abi.OK
    assert run(x=None) == _abi.E_INVAL
    assert run(xt=5) == _abi.E_INVAL and run(act=9) == _abi.E_INVAL
    assert run(ldx=15) == _abi.E_INVAL and run(ldy=7) == _abi.E_INVAL and run(n=-1) == _abi.E_INVAL
    assert run(n=1 << 40) == _abi.E_UNSUPPORTED
    assert run(sb=s.numel() - 1) == _abi.E_RANGE
    assert run(y=x.data_ptr()) == _abi.E_ALIAS
    assert run(x=x.data_ptr() + 2) == _abi.E_INVAL
    host = torch.zeros((4, 16))
    assert run(x=host.data_ptr()) == _abi.E_INVAL
    assert run(ldx=1 << 30) == _abi.E_RANGE      # the last row lies outside the allocation
    with pytest.raises(ValueError):
        api.linear8(layer, x[:, :15], y)
    with pytest.raises(ValueError):
        api.linear8(layer, x.t().contiguous().t(), y)
    with pytest.raises(TypeError):
        api.linear8(layer, x.half(), y)
    with pytest.raises(ValueError):
        api.Linear8(_rand(18, (8, 16)), torch.zeros(7))
    with pytest.raises(_abi.HpacmlError) as e:
        api.Linear8(torch.zeros((1, _abi.MAX_WIDTH8 + 1)))
    assert e.value.status == _abi.E_UNSUPPORTED


# ---- activations kept in 8 bits -----------------------------------------------


def _kept(a, act):
    """Values that the codes of a [rows][width] (after its activation) stand
    for, and the codes, by the definition in 64 bits."""
    a = np.asarray(a, np.float64)
    rows, width = a.shape
    blocks = -(-width // 32)
    p = np.zeros((rows, blocks * 32))
    p[:, :width] = a
    p = p.reshape(rows, blocks, 32)
    bits = 8 if act == RELU else 7
    with np.errstate(invalid="ignore"):
        e = np.frexp(np.where(np.isfinite(p), np.abs(p), 0).max(axis=2))[1] - bits
    e = np.maximum(np.where(p.any(axis=2), e, -126), -126)
    top = 2 ** bits - 1
    step = np.ldexp(1.0, e)[:, :, None]
    with np.errstate(invalid="ignore"):
        c = np.clip(np.rint(p / step), -top, top)
        if act == RELU:
            c = np.where((p > 0) & (c < 1), 1, c)
    return (c * step).reshape(rows, -1)[:, :width], c, e


def _relu(z):
    return np.where(z < 0, 0, z)


@pytest.mark.parametrize("rows, width", [(1, 1), (1, 31), (3, 32), (5, 33), (64, 64), (77, 100), (200, 4096), (33, 513),
                                         (2, 16384), (1000, 35), (513, 8), (100, 256)])
@pytest.mark.parametrize("act", [RELU, IDENT])
@pytest.mark.parametrize("z_kind, a_kind", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_keep_matches_definition(rows, width, act, z_kind, a_kind):
    torch = _torch()
    pad = rows % 3
    z = (_rand(20, (rows, width), pad=pad) * torch.exp2(4 * _rand(21, (rows, width), pad=pad))).to(_dtype(z_kind))
    z[::7] = 0
    wide = torch.empty((rows, width + pad), dtype=z.dtype, device="cuda")
    wide[:, :width] = z
    z = wide[:, :width]
    kept = api.Checkpoint8(rows, width, act)
    whole, a = _guarded(rows, width, a_kind)
    whole_b, back = _guarded(rows, width, a_kind)
    api.checkpoint8_save(kept, z, a)
    api.checkpoint8_load(kept, back)
    torch.cuda.synchronize()
    zz = _np(z)
    full = _relu(zz) if act == RELU else zz
    want, codes, e = _kept(full, act)
    assert np.array_equal(_np(back), want)                  # exact in bf16, too
    assert np.array_equal(_np(a), _np(torch.from_numpy(full).to(_dtype(a_kind))))
    stored = kept.codes.cpu().numpy().reshape(rows, -1, 32).astype(np.float64)
    assert np.array_equal(stored - (0 if act == RELU else 128), codes)
    assert np.array_equal(kept.exps.cpu().numpy().astype(int), e + 127)
    if act == RELU:
        assert np.array_equal(codes.reshape(rows, -1)[:, :width] != 0, zz > 0)
    _untouched(whole, rows, width)
    _untouched(whole_b, rows, width)


@pytest.mark.parametrize("act", [RELU, IDENT])
def test_keep_extremes(act):
    """Denormals, the smallest normals and the largest finite values."""
    torch = _torch()
    vals = [1e-45, 2.0 ** -127, 2.0 ** -126, 2.0 ** -119, 3e-38, 1e38, 3.4028234e38, 0.0, -0.0, -1e-45, -3.4028234e38]
    z = torch.zeros((len(vals), 64), device="cuda")
    for i, v in enumerate(vals):
        z[i, 5] = v
        z[i, 37] = v / 3
    kept, back = api.Checkpoint8(len(vals), 64, act), torch.empty_like(z)
    api.checkpoint8_save(kept, z)
    api.checkpoint8_load(kept, back)
    zz = _np(z)
    want, _, _ = _kept(_relu(zz) if act == RELU else zz, act)
    assert np.array_equal(_np(back), want)


@pytest.mark.parametrize("act", [RELU, IDENT])
def test_keep_non_finite_blocks(act):
    """A block with an infinity or a NaN stands for no finite value; the
    blocks beside it are as ever, and a NaN lets nothing through."""
    torch = _torch()
    z = _rand(22, (6, 96)).clone()
    z[0, 40], z[1, 40], z[2, 40], z[3, 33] = float("inf"), float("nan"), -float("inf"), float("nan")
    kept, back, a = api.Checkpoint8(6, 96, act), torch.empty_like(z), torch.empty_like(z)
    api.checkpoint8_save(kept, z, a)
    api.checkpoint8_load(kept, back)
    zz, got = _np(z), _np(back)
    full = _relu(zz) if act == RELU else zz
    assert np.array_equal(_np(a), full, equal_nan=True)
    blocks = ~np.isfinite(full.reshape(6, 3, 32)).all(axis=2)
    assert blocks.sum() == (3 if act == RELU else 4)
    assert np.array_equal(kept.exps.cpu().numpy() == 255, blocks)
    want, _, _ = _kept(full, act)
    assert np.isfinite(got.reshape(6, 3, 32)[~blocks]).all()
    assert not np.isfinite(got.reshape(6, 3, 32)[blocks]).any()
    assert np.array_equal(got.reshape(6, 3, 32)[~blocks], want.reshape(6, 3, 32)[~blocks])
    if act == RELU:
        assert np.array_equal(kept.codes.cpu().numpy() != 0, zz > 0)


def test_keep_in_place_and_wide_pitches():
    torch = _torch()
    z = _rand(23, (50, 70), "bf16", pad=3)
    codes = torch.full((50, 128), 9, dtype=torch.uint8, device="cuda")
    exps = torch.full((50, 7), 9, dtype=torch.uint8, device="cuda")
    kept = api.Checkpoint8(50, 70, RELU, codes=codes, exps=exps)
    want = torch.relu(z)
    api.checkpoint8_save(kept, z, z)
    assert torch.equal(z, want)
    assert (codes[:, 96:] == 9).all() and (exps[:, 3:] == 9).all() and (codes[:, 70:96] == 0).all()


def test_keep_refusals():
    torch = _torch()
    z = _rand(24, (8, 64))
    kept = api.Checkpoint8(8, 64, RELU)
    api.checkpoint8_save(kept, z)
    with pytest.raises(_abi.HpacmlError) as e:     # rows that overlap each other
        api.checkpoint8_save(kept, z, torch.as_strided(z, (8, 64), (32, 1)))
    assert e.value.status == _abi.E_INVAL
    big = torch.zeros((9, 64), device="cuda")
    with pytest.raises(_abi.HpacmlError) as e:
        api.checkpoint8_save(kept, big[:8], big[1:])
    assert e.value.status == _abi.E_ALIAS
    with pytest.raises(ValueError):
        api.checkpoint8_save(kept, z[:, :63])
    with pytest.raises(ValueError):
        api.Checkpoint8(8, 64, RELU, codes=torch.zeros((8, 63), dtype=torch.uint8, device="cuda"))
    bad = api.Checkpoint8(8, 64, 7)
    with pytest.raises(_abi.HpacmlError) as e:
        api.checkpoint8_save(bad, z)
    assert e.value.status == _abi.E_INVAL
    odd = api.Checkpoint8(8, 64, RELU, codes=torch.zeros((8, 72), dtype=torch.uint8, device="cuda"))
    with pytest.raises(_abi.HpacmlError) as e:     # a pitch of 72 is not a multiple of 32
        api.checkpoint8_save(odd, z)
    assert e.value.status == _abi.E_INVAL
    kept.desc.rows = 1 << 20                       # beyond the buffers
    assert _abi.lib().hpacml8_checkpoint_load(kept.desc, z.data_ptr(), 0, 64, None) == _abi.E_RANGE


# ---- the backward pass ----------------------------------------------------------


def _case(rows, n_in, n_out, act, kind, pad=0, seed=30):
    """A kept activation (through the library), dy and W; all 64-bit copies."""
    torch = _torch()
    z = _rand(seed, (rows, n_in)) * torch.exp2(_rand(seed + 1, (rows, 1)))
    kept, back = api.Checkpoint8(rows, n_in, act), torch.empty((rows, n_in), device="cuda")
    api.checkpoint8_save(kept, z)
    api.checkpoint8_load(kept, back)
    dy = _rand(seed + 2, (rows, n_out), kind, pad, 1e-2)
    W = _rand(seed + 3, (n_out, n_in), kind, scale=n_in ** -0.5)
    through = _np(z) > 0 if act == RELU else np.ones((rows, n_in), bool)
    return kept, dy, W, _np(back), through


def _check_backward(kept, dy, W, a, through, kind, parts=("dw", "db", "dx"), what=""):
    torch = _torch()
    rows, n_in, n_out = kept.rows, kept.width, dy.shape[1]
    whole_w, dw = _guarded(n_out, n_in, "f32", pad=3)
    whole_x, dx = _guarded(rows, n_in, kind)
    db = torch.full((n_out,), -77.0, device="cuda")
    api.backward8(kept, dy, dw if "dw" in parts else None, db if "db" in parts else None, W=W,
                  dx=dx if "dx" in parts else None)
    torch.cuda.synchronize()
    g, w = _np(dy), _np(W)
    # products of 8-bit significands are exact in fp32; a sum of n terms in
    # any order is within n * EPS_SUM of the sum of magnitudes (for fp32, three
    # times as many terms).  dx: the six largest of nine partial products
    # leave out at most 2^-23 of a product, plus the rounding to its type.
    terms = 3 if kind == "f32" else 1
    if "dw" in parts:
        tol = (terms * rows + 2) * EPS_SUM * (np.abs(g).T @ np.abs(a)) + 1e-37
        assert (np.abs(_np(dw) - g.T @ a) <= tol).all(), what
    else:
        assert (dw == -77).all()
    if "db" in parts:
        assert (np.abs(_np(db) - g.sum(0)) <= (terms * rows + 2) * EPS_SUM * np.abs(g).sum(0) + 1e-37).all(), what
    else:
        assert (db == -77).all()
    if "dx" in parts:
        want = np.where(through, g @ w, 0)
        tol = ((6 if kind == "f32" else 1) * n_out + 2) * EPS_SUM * (np.abs(g) @ np.abs(w)) + 1e-37
        tol = tol + (EPSBF * np.abs(want) if kind == "bf16" else 0)
        got = _np(dx)
        assert (np.abs(got - want) <= tol).all(), what
        assert (got[~through] == 0).all(), what
    _untouched(whole_w, n_out, n_in)
    _untouched(whole_x, rows, n_in)


@pytest.mark.parametrize("rows", [1, 2, 31, 63, 64, 65, 200, 1111])
@pytest.mark.parametrize("n_in, n_out", [(1, 1), (5, 3), (32, 64), (33, 65), (64, 1), (1, 64), (200, 50), (96, 130), (300, 257)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward_sizes(rows, n_in, n_out, kind):
    act = (RELU, IDENT)[(rows + n_out) % 2]
    kept, dy, W, a, t = _case(rows, n_in, n_out, act, kind, pad=rows % 3)
    _check_backward(kept, dy, W, a, t, kind)


@pytest.mark.parametrize("rows, n_in, n_out", [(10007, 256, 256), (4096, 512, 512), (70001, 64, 8), (70001, 8, 64),
                                               (3000, 1024, 520), (300, 2048, 2048), (1, 2048, 4096), (100003, 35, 5)])
@pytest.mark.parametrize("kind, act", [("f32", RELU), ("bf16", RELU), ("bf16", IDENT)])
def test_backward_larger(rows, n_in, n_out, kind, act):
    kept, dy, W, a, t = _case(rows, n_in, n_out, act, kind)
    _check_backward(kept, dy, W, a, t, kind)


@pytest.mark.parametrize("rows, n_in, n_out", [(13001, 1100, 550), (12950, 1088, 512), (100101, 256, 40), (99001, 250, 33)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward_in_the_largest_tiles(rows, n_in, n_out, kind):
    kept, dy, W, a, t = _case(rows, n_in, n_out, RELU, kind)
    _check_backward(kept, dy, W, a, t, kind)


@pytest.mark.parametrize("rows, n_in, n_out", [(1024, 40, 70), (1025, 40, 70), (1, 1000, 900), (3, 1100, 511), (33, 1100, 513),
                                               (512, 64, 1111), (700, 333, 222), (65, 4097, 33), (17, 31, 4099)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward_of_few_rows(rows, n_in, n_out, kind):
    """On both sides of the sizes that one launch takes."""
    act = (RELU, IDENT)[rows % 2]
    kept, dy, W, a, t = _case(rows, n_in, n_out, act, kind, pad=rows % 3)
    _check_backward(kept, dy, W, a, t, kind)


def test_backward_of_few_rows_beside_infinite_weights_and_rows():
    """The rows of W that lie beyond a block of outputs' end, and the rows of dy
    beyond a block of rows' end, do not take part."""
    torch = _torch()
    kept, dy, W, a, t = _case(35, 40, 37, IDENT, "f32")
    W[36, 3] = float("inf")
    dy[:, 36] = torch.where(dy[:, 36] == 0, 1.0, dy[:, 36])
    dx = torch.empty((35, 40), device="cuda")
    api.backward8(kept, dy, W=W, dx=dx)
    rest = [k for k in range(40) if k != 3]
    assert torch.isfinite(dx[:, rest]).all() and not torch.isfinite(dx[:, 3]).any()
    W[36, 3] = 0.0
    dy[34, 5] = float("nan")
    dw = torch.empty((37, 40), device="cuda")
    api.backward8(kept, dy, dw, W=W, dx=dx)
    assert torch.isnan(dx[34]).all() and torch.isfinite(dx[:34]).all()
    rest = [j for j in range(37) if j != 5]
    assert torch.isnan(dw[5]).all() and torch.isfinite(dw[rest]).all()


@pytest.mark.parametrize("parts", [("dw",), ("db",), ("dx",), ("dw", "db"), ("dw", "dx"), ("db", "dx")])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward_wanted_parts(parts, kind):
    kept, dy, W, a, t = _case(500, 96, 72, RELU, kind)
    _check_backward(kept, dy, W, a, t, kind, parts)


@pytest.mark.parametrize("off", [0, 1, 4, 8])
def test_backward_alignment(off):
    """dy and W that begin at any element of wider rows."""
    kept, dy, W, a, t = _case(333, 128, 64, RELU, "bf16")
    wide, wideW = _rand(50, (333, 96), "bf16"), _rand(51, (64, 150), "bf16")
    wide[:, off:off + 64] = dy
    wideW[:, off:off + 128] = W
    _check_backward(kept, wide[:, off:off + 64], wideW[:, off:off + 128], a, t, "bf16", what="offset %d" % off)


def test_backward_ignores_what_lies_beside_its_rows():
    """NaN in the columns beside dy and in the codes' padding."""
    torch = _torch()
    for n_out in (64, 72, 40):
        kept, dy, W, a, t = _case(130, 70, n_out, RELU, "bf16")
        wide = torch.full((131, n_out + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:130, :n_out] = dy
        kept.codes[:, 70:] = 255
        _check_backward(kept, wide[:130, :n_out], W, a, t, "bf16")


def test_backward_accumulates_parts():
    torch = _torch()
    kept, dy, W, a, t = _case(400, 100, 60, RELU, "f32")
    dw, db = torch.zeros((60, 100), device="cuda"), torch.zeros(60, device="cuda")
    for i in range(0, 400, 130):
        m = min(130, 400 - i)
        part = api.Checkpoint8(m, 100, RELU, codes=kept.codes[i:i + m], exps=kept.exps[i:i + m])
        api.backward8(part, dy[i:i + m], dw, db, accumulate=True)
    g = _np(dy)
    assert (np.abs(_np(dw) - g.T @ a) <= 1300 * EPS_SUM * (np.abs(g).T @ np.abs(a))).all()
    assert (np.abs(_np(db) - g.sum(0)) <= 1300 * EPS_SUM * np.abs(g).sum(0)).all()


def test_backward_without_rows():
    torch = _torch()
    kept = api.Checkpoint8(0, 40, RELU)
    dw, db = torch.ones((20, 40), device="cuda"), torch.ones(20, device="cuda")
    dy = torch.empty((0, 20), device="cuda")
    api.backward8(kept, dy, dw, db, accumulate=True)
    assert (dw == 1).all() and (db == 1).all()
    api.backward8(kept, dy, dw, db)
    assert (dw == 0).all() and (db == 0).all()


def test_backward_infinite_weights_stay_behind_the_mask():
    """Where the ReLU let nothing through, dx is 0 whatever the product is."""
    torch = _torch()
    kept, dy, W, a, t = _case(100, 64, 32, RELU, "bf16")
    W[3, 7], W[5, 9] = float("inf"), float("nan")
    dx = torch.empty((100, 64), dtype=torch.bfloat16, device="cuda")
    api.backward8(kept, dy, W=W, dx=dx)
    got = _np(dx)
    assert (got[~t] == 0).all()
    assert not np.isfinite(got[:, [7, 9]][t[:, [7, 9]]]).any()
    rest = [k for k in range(64) if k not in (7, 9)]
    assert np.isfinite(got[:, rest]).all()


def test_backward_large_and_infinite_fp32_gradients():
    """fp32 values that round to infinity in bf16 stay finite; infinities and
    NaNs reach the gradients they belong to and no others."""
    torch = _torch()
    kept, dy, W, a, t = _case(70, 40, 8, IDENT, "f32")
    dy = torch.zeros_like(dy)
    dy[3, 0] = 3.4028234e38
    db = torch.empty(8, device="cuda")
    api.backward8(kept, dy, db=db)
    assert db[0].item() == dy[3, 0].item()
    dy[5, 1], dy[6, 2] = float("inf"), float("nan")
    dw = torch.empty((8, 40), device="cuda")
    dy[3, 0] = 1.0
    api.backward8(kept, dy, dw, db)
    assert not torch.isfinite(dw[1]).any() and torch.isnan(dw[2]).all() and torch.isfinite(dw[[0, 3, 4, 5, 6, 7]]).all()
    assert torch.isinf(db[1]) and torch.isnan(db[2])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_backward_repeats_and_streams(kind):
    torch = _torch()
    kept, dy, W, a, t = _case(20000, 256, 128, RELU, kind)
    need, outs = api.backward8_scratch_bytes(kept, dy, W), []
    for _ in range(3):
        s = torch.cuda.Stream()
        dw, db, dx = torch.empty((128, 256), device="cuda"), torch.empty(128, device="cuda"), torch.empty((20000, 256), dtype=dy.dtype, device="cuda")
        scratch = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF)
        torch.cuda.synchronize()
        api.backward8(kept, dy, dw, db, W=W, dx=dx, scratch=scratch, stream=s)
        s.synchronize()
        outs.append((dw, db, dx))
    for o in outs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(outs[0], o))


def test_backward_against_differences():
    """The gradients of a loss of a small layer, against central differences
    in 64 bits at the kept values."""
    torch = _torch()
    rows, n_in, n_out = 6, 9, 5
    kept, dy, W, a, t = _case(rows, n_in, n_out, RELU, "f32")
    w, b, r = _np(W), np.linspace(-1, 1, n_out), _np(_rand(60, (rows, n_out)))

    def loss(a, w, b):
        y = a @ w.T + b
        return (r * np.sin(y)).sum()

    dy = torch.from_numpy(r * np.cos(a @ w.T + b)).float().cuda()
    dw, db, dx = torch.empty((n_out, n_in), device="cuda"), torch.empty(n_out, device="cuda"), torch.empty((rows, n_in), device="cuda")
    api.backward8(kept, dy, dw, db, W=W, dx=dx)
    h = 1e-5

    def differences(v, f):
        out = np.zeros_like(v)
        for i in np.ndindex(*v.shape):
            p, m = v.copy(), v.copy()
            p[i] += h
            m[i] -= h
            out[i] = (f(p) - f(m)) / (2 * h)
        return out

    # h^2 / 6 of a third derivative of order |a|^3 rows, and fp32 roundings
    for got, want in ((dw, differences(w, lambda v: loss(a, v, b))), (db, differences(b, lambda v: loss(a, w, v))),
                      (dx, np.where(t, differences(a, lambda v: loss(v, w, b)), 0))):
        assert np.abs(_np(got) - want).max() <= 1e-4 * max(1, np.abs(want).max())


def test_backward_refusals():
    torch = _torch()
    kept, dy, W, a, t = _case(16, 32, 8, RELU, "f32")
    dw, dx = torch.empty((8, 32), device="cuda"), torch.empty((16, 32), device="cuda")
    with pytest.raises(_abi.HpacmlError) as e:
        api.backward8(kept, dy)                                  # nothing wanted
    assert e.value.status == _abi.E_INVAL
    with pytest.raises(_abi.HpacmlError) as e:
        api.backward8(kept, dy, dw, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == _abi.E_RANGE
    both = torch.zeros((24, 32), device="cuda")
    with pytest.raises(_abi.HpacmlError) as e:
        api.backward8(kept, dy, W=both[:8], dx=both[7:23])
    assert e.value.status == _abi.E_ALIAS
    with pytest.raises(TypeError):
        api.backward8(kept, dy, W=W.bfloat16(), dx=dx)
    with pytest.raises(TypeError):
        api.backward8(kept, dy, dw.double())
    with pytest.raises(ValueError):
        api.backward8(kept, dy, dx=dx)
    with pytest.raises(ValueError):
        api.backward8(kept, dy[:15], dw)
    with pytest.raises(ValueError):
        api.backward8(kept, dy, dw, stream=torch.cuda.Stream())   # no scratch on another stream
    n_out = _abi.MAX_WIDTH8 + 1
    assert _abi.lib().hpacml8_backward(kept.desc, dy.data_ptr(), 0, n_out, n_out, None, 0, dw.data_ptr(), 32, None, None,
                                       0, 0, None, 0, None) == _abi.E_UNSUPPORTED


# ---- graphs and long offsets -------------------------------------------------------


@pytest.mark.parametrize("rows, n_in, n_out", [(3, 200, 96), (60, 64, 64), (700, 96, 130), (5000, 256, 192), (33000, 128, 64)])
def test_replayed_from_a_graph(rows, n_in, n_out):
    """Every replay, with other inputs and eager work in between, has the eager
    calls' bits."""
    torch = _torch()
    layer = api.Linear8(_rand(70, (n_out, n_in)))
    z, dy = torch.empty((rows, n_in), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, n_out), dtype=torch.bfloat16, device="cuda")
    W = _rand(71, (n_out, n_in), "bf16")
    kept = api.Checkpoint8(rows, n_in, RELU)

    def outputs():
        return (torch.empty((rows, n_out), device="cuda"), torch.empty((rows, n_in), dtype=torch.bfloat16, device="cuda"),
                torch.empty((n_out, n_in), device="cuda"), torch.empty(n_out, device="cuda"), torch.empty_like(z))

    def calls(o, scratch, stream):
        y, a, dw, db, dx = o
        api.checkpoint8_save(kept, z, a, stream=stream)
        api.linear8(layer, a, y, RELU, scratch=scratch, stream=stream)
        api.backward8(kept, dy, dw, db, W=W, dx=dx, scratch=scratch, stream=stream)

    z.copy_(_rand(72, (rows, n_in)))
    dy.copy_(_rand(73, (rows, n_out)))
    scratch = torch.empty(max(layer.scratch_bytes(rows), api.backward8_scratch_bytes(kept, dy, W)), dtype=torch.uint8, device="cuda")
    replayed, s = outputs(), torch.cuda.Stream()
    calls(replayed, scratch, None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls(replayed, scratch, s)
    for i in range(4):
        z.copy_(_rand(80 + i, (rows, n_in)))
        dy.copy_(_rand(90 + i, (rows, n_out)))
        for t in replayed:
            t.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        eager = outputs()
        calls(eager, torch.empty_like(scratch), None)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(replayed, eager)), i


# (rows, pitch): offsets in the last rows pass 2^32 bytes; few rows, many rows, pitches beyond what a tile's offsets hold
@pytest.mark.parametrize("rows, pitch", [(40, 1 << 26), (70001, 1 << 15), (1100, 1 << 22)])
@pytest.mark.parametrize("n_in, n_out", [(64, 64), (70, 40)])
def test_rows_far_apart(rows, pitch, n_in, n_out):
    torch = _torch()

    def far(width, kind=torch.bfloat16, like=None):
        t = torch.empty((rows, pitch), dtype=kind, device="cuda")[:, pitch - 128:][:, :width]
        if like is not None:
            t.copy_(like)
        return t

    x, dy, W = _rand(74, (rows, n_in), "bf16"), _rand(75, (rows, n_out), "bf16"), _rand(76, (n_out, n_in), "bf16")
    layer = api.Linear8(_rand(77, (n_out, n_in)))
    blocks = -(-n_in // 32)
    results = []
    for apart in (False, True):
        y = far(n_out) if apart else torch.empty((rows, n_out), dtype=torch.bfloat16, device="cuda")
        api.linear8(layer, far(n_in, like=x) if apart else x, y, RELU)
        results.append([y.clone()])
        del y
        kept = api.Checkpoint8(rows, n_in, RELU, far(blocks * 32, torch.uint8), far(blocks, torch.uint8)) if apart else \
            api.Checkpoint8(rows, n_in, RELU)
        a = far(n_in) if apart else torch.empty((rows, n_in), dtype=torch.bfloat16, device="cuda")
        api.checkpoint8_save(kept, x, a)
        back = far(n_in) if apart else torch.empty_like(x)
        api.checkpoint8_load(kept, back)
        results[-1] += [a.clone(), back.clone(), kept.codes[:, :blocks * 32].clone(), kept.exps[:, :blocks].clone()]
        del a, back
        dw, db = torch.empty((n_out, n_in), device="cuda"), torch.empty(n_out, device="cuda")
        dx = far(n_in) if apart else torch.empty_like(x)
        api.backward8(kept, far(n_out, like=dy) if apart else dy, dw, db, W=W, dx=dx)
        results[-1] += [dw, db, dx.clone()]
        torch.cuda.synchronize()
        del dx, kept
    torch.cuda.empty_cache()
    assert all(torch.equal(u, v) for u, v in zip(*results)), [torch.equal(u, v) for u, v in zip(*results)]
