"""The 8-bit dense layers at the ends of their ranges: the longest operands,
the largest and smallest values, infinities, and what a training loop does
between its steps."""
import numpy as np
import pytest

from paper_2407_18352_amd import _abi, api
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

RELU, IDENT = _abi.ACT_RELU, _abi.ACT_IDENTITY


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def test_the_longest_operands_are_refused():
    """2^31 - 1 rows as far apart as can be described lie in no allocation."""
    import torch
    L, big = _abi.lib(), 2 ** 31 - 1
    layer = api.Linear8(torch.ones((8, 16)))
    x, y, s = (torch.zeros(1 << 12, device="cuda") for _ in range(3))
    args = x.data_ptr(), y.data_ptr(), s.data_ptr()

    def run(kind, n, ldx, ldy):
        return L.hpacml8_linear_run(layer.handle, args[0], kind, ldx, n, args[1], kind, ldy, 0, args[2], 1 << 60, None)

    for kind in (_abi.F32, _abi.BF16):
        assert run(kind, big, big, 8) == _abi.E_RANGE
        assert run(kind, big, 16, big) == _abi.E_RANGE
        assert run(kind, big, big, big) == _abi.E_RANGE
    kept = api.Checkpoint8(2, 32, RELU)
    kept.desc.rows = kept.desc.ld_exps = big
    kept.desc.ld_codes = big // 32 * 32
    assert L.hpacml8_checkpoint_load(kept.desc, args[0], _abi.F32, big, None) == _abi.E_RANGE
    assert L.hpacml8_checkpoint_save(kept.desc, args[0], _abi.F32, big, None, 0, 0, None) == _abi.E_RANGE
    assert L.hpacml8_backward(kept.desc, args[0], _abi.F32, big, 8, args[1], 32, None, 0, None, args[1], big, 0, args[2],
                              1 << 60, None) == _abi.E_RANGE
    torch.cuda.synchronize()
    assert not any(t.any() for t in (x, y, s))


@pytest.mark.parametrize("rows, n_in, n_out", [(1, 70, 50), (20, 70, 50), (24, 1100, 40), (60, 70, 50), (300, 130, 200),
                                               (5000, 600, 300), (33001, 70, 50), (33001, 300, 150)])
@pytest.mark.parametrize("x_kind, y_kind", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("large", ["x", "W"])
def test_linear_of_values_whose_sums_alone_leave_the_range(rows, n_in, n_out, x_kind, y_kind, large):
    """A scale times the sum of codes passes 3.4e38 long before the result
    does, when the other scale is small: points of magnitudes up to 3e38
    against weights from 1e-36, and the other way round."""
    import torch
    from test_gpu_dense8 import _check_linear, _dtype, _rand
    high = lambda n: 10.0 ** torch.linspace(38.4, 25, n, device="cuda", dtype=torch.float64)[:, None]
    low = lambda n: 10.0 ** torch.linspace(-36, -5, n, device="cuda", dtype=torch.float64)[:, None]
    unit = lambda seed, n: (_rand(seed, (n, n_in)) / 8).clamp(-1, 1).double()      # results stay below 3e38
    x = unit(1, rows) * (high if large == "x" else low)(rows)
    W = unit(2, n_out) * (low if large == "x" else high)(n_out)
    if large == "x":
        x[:, 0], W[:, 0] = x.abs().amax(1), W.abs().amax(1)      # sums that are not 0
    limit = 3.0e38 / n_in
    W *= (limit / (x.abs().max() * W.abs().max())).clamp(max=1)
    W = W.float()
    if large == "x" and rows >= 3 and n_out >= 3:
        W[2] = 0
        x[2], W[1] = 0, 0
        x[2, 1], W[1, 2] = 3e38, 3e38 * 2.0 ** -128              # a sum of 0, of a large point
    _check_linear(x.to(_dtype(x_kind)), W, _rand(3, (1, n_out))[0], IDENT, y_kind)


def _sums(a, b):
    """sum_j a_ij b_jk in 64 bits, product by product (a library's product need
    not treat infinities as sums do)."""
    with np.errstate(invalid="ignore"):
        return np.concatenate([(a[:, :, None] * b[None, :, k:k + 1]).sum(1) for k in range(b.shape[1])], 1)


def _same(got, want, tol):
    with np.errstate(invalid="ignore"):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        inf = np.isinf(want)
        assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf])
        ok = np.isfinite(want)
        assert (np.abs(got - want)[ok] <= np.broadcast_to(tol, want.shape)[ok]).all()


@pytest.mark.parametrize("rows, n_in, n_out", [(70, 40, 8), (33, 70, 200), (1100, 72, 40), (1500, 70, 100), (40000, 24, 16)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", [RELU, IDENT])
def test_backward_infinities_follow_the_formula(rows, n_in, n_out, kind, act):
    """Infinities of either sign and NaNs in dy and W, beside zeros, values
    exact in 8 bits and others: the results are infinite, and NaN, where the
    sums of the formulas are."""
    import torch
    from test_gpu_dense8 import EPS_SUM, EPSBF, _case, _np
    inf, nan = float("inf"), float("nan")
    kept, dy, W, a, through = _case(rows, n_in, n_out, act, kind)
    dy, W = dy.clone(), W.clone()
    dy[::3] = (dy[::3] * 256).round() / 256        # few bits, zeros among them
    W[:, ::2] = (W[:, ::2] * 16).round() / 16
    dy[5, 1], dy[9, 2], dy[30, 3], dy[rows - 1, 4], dy[31, 1], dy[12, 7] = inf, -inf, inf, -inf, inf, nan
    W[3, 7], W[4, 9], W[1, 11], W[6, 13], W[1, 15], W[2, 15] = inf, -inf, inf, nan, -inf, inf
    W[1, 17] = 0.0
    dw, db = torch.empty((n_out, n_in), device="cuda"), torch.empty(n_out, device="cuda")
    dx = torch.empty((rows, n_in), dtype=dy.dtype, device="cuda")
    api.backward8(kept, dy, dw, db, W=W, dx=dx)
    g, w = _np(dy), _np(W)
    fin = lambda v: np.abs(np.where(np.isfinite(v), v, 0))
    terms = 3 if kind == "f32" else 1
    want = np.where(through, _sums(g, w), 0)
    tol = (2 * terms * n_out + 2) * EPS_SUM * (fin(g) @ fin(w)) + 1e-37 + (EPSBF * fin(want) if kind == "bf16" else 0)
    _same(_np(dx), want, tol)
    _same(_np(dw), _sums(g.T, a), (terms * rows + 2) * EPS_SUM * (fin(g).T @ np.abs(a)) + 1e-37)
    with np.errstate(invalid="ignore"):
        _same(_np(db), g.sum(0), (terms * rows + 2) * EPS_SUM * fin(g).sum(0) + 1e-37)


@pytest.mark.parametrize("rows", [1, 1100])
def test_backward_terms_of_fp32_values_add_up(rows):
    """One row of values of every exponent against a kept 1 and W = 1: the sum of
    an operand's three terms, exact from 2^-110 on, within 2^-134 below."""
    import torch
    z = torch.zeros((rows, 64), device="cuda")
    z[0] = 1.0
    kept = api.Checkpoint8(rows, 64, IDENT)
    api.checkpoint8_save(kept, z)
    n = 256 * 128
    bits = torch.randint(0, 1 << 23, (n,), generator=torch.Generator().manual_seed(7), dtype=torch.int32)
    v = (bits | (torch.arange(n, dtype=torch.int32) // 128 % 255) << 23).view(torch.float32)
    v[::5] *= -1
    v[-1], v[-2] = 3.4028234663852886e38, -3.4028234663852886e38
    eye, dx = torch.eye(64, device="cuda"), torch.empty((rows, 64), device="cuda")
    dw, db = torch.empty((64, 64), device="cuda"), torch.empty(64, device="cuda")
    for part in v.split(64):
        dy = torch.zeros((rows, 64), device="cuda")
        dy[0] = part.cuda()
        api.backward8(kept, dy, dw, db, W=eye, dx=dx)
        want = part.double()
        tol = torch.where(want.abs() >= 2.0 ** -110, 0.0, 2.0 ** -134)
        for got in (dw[:, 0], dw[:, 63], db, dx[0]):
            assert ((got.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows, n_in, n_out", [(70, 100, 8), (1500, 100, 70), (40000, 96, 24), (1200, 600, 600)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", [RELU, IDENT])
def test_backward_of_kept_infinities(rows, n_in, n_out, kind, act):
    """A block of channels that was kept with an infinity or a NaN: dw is that of
    the values it stands for in bf16, and NaN in fp32; db, dx and the other
    blocks are as ever."""
    import torch
    from test_gpu_dense8 import EPS_SUM, _np, _rand
    z = _rand(51, (rows, n_in)).clone()
    z[7, 3], z[rows - 1, 70] = float("inf"), float("nan") if rows % 3 else float("inf")
    kept, back = api.Checkpoint8(rows, n_in, act), torch.empty((rows, n_in), device="cuda")
    api.checkpoint8_save(kept, z)
    api.checkpoint8_load(kept, back)
    dy, W = _rand(52, (rows, n_out), kind, 0, 1e-2).clone(), _rand(53, (n_out, n_in), kind)
    dy[7, 1] = 0
    dw, db = torch.empty((n_out, n_in), device="cuda"), torch.empty(n_out, device="cuda")
    dx = torch.empty((rows, n_in), dtype=dy.dtype, device="cuda")
    api.backward8(kept, dy, dw, db, W=W, dx=dx)
    a, g, w = _np(back), _np(dy), _np(W)
    channels = [k for k in range(n_in) if k // 32 in (0, 2)]
    assert not np.isfinite(a).all(0)[channels].any() and np.isfinite(a).all(0).sum() == n_in - len(channels)
    want = _sums(g.T, a)
    if kind == "f32":
        want[:, channels] = np.nan
    _same(_np(dw), want, (3 * rows + 2) * EPS_SUM * (np.abs(g).T @ np.abs(np.where(np.isfinite(a), a, 0))) + 1e-37)
    assert np.isfinite(_np(db)).all() and np.isfinite(_np(dx)).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("n_in, n_out", [(2048, 2048), (40, 20)])
def test_backward_without_rows_on_either_side_of_the_rule(kind, n_in, n_out):
    """Sizes that one launch takes and that take several; dx alone as well, whose
    empty tensor has no address."""
    import torch
    kind = getattr(torch, kind)
    kept = api.Checkpoint8(0, n_in, RELU)
    dw, db = torch.full((n_out, n_in), 3.0, device="cuda"), torch.full((n_out,), 3.0, device="cuda")
    dy, dx = (torch.empty((0, n), dtype=kind, device="cuda") for n in (n_out, n_in))
    W = torch.ones((n_out, n_in), dtype=kind, device="cuda")
    api.backward8(kept, dy, dw, db, W=W, dx=dx, accumulate=True)
    assert (dw == 3).all() and (db == 3).all()
    api.backward8(kept, dy, W=W, dx=dx)
    api.backward8(kept, dy, db=db)
    assert (dw == 3).all() and (db == 0).all()
    api.backward8(kept, dy, dw, db, W=W, dx=dx)
    assert (dw == 0).all() and (db == 0).all()


# ---- a training loop ----------------------------------------------------------


def _model_and_batch(dims=(6, 64, 96, 2), n=300, seed=0):
    import torch
    from paper_2407_18352_amd.surrogate8 import Surrogate8
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, dims[0]), generator=g, device="cuda")
    return Surrogate8(dims, seed=1), x, torch.randn((n, dims[-1]), generator=g, device="cuda") / n


def _grads(m):
    return [p.grad.clone() for p in m.parameters()]


@pytest.mark.parametrize("accumulate", [False, True])
def test_training_after_zero_grad(accumulate):
    """An optimizer's zero_grad takes the gradients away (None) or fills them
    with 0: the next pass has all of them, equal to a new model's."""
    import torch
    m, x, dy = _model_and_batch()
    m.forward(x)
    m.backward(dy)
    want = _grads(m)
    opt = torch.optim.SGD(m.parameters(), lr=0.0)
    for to_none in (True, False):
        opt.zero_grad(set_to_none=to_none)
        m.forward(x)
        m.backward(dy, accumulate=accumulate)
        assert all(torch.equal(u, v) for u, v in zip(_grads(m), want))
        opt.step()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_inputs_and_gradients_of_any_layout(kind):
    """Inputs that lie column after column (fields stacked one by one), rows of a
    wider record, and a gradient that is one row for all points."""
    import torch
    from paper_2407_18352_amd import surrogate8
    m, x, _ = _model_and_batch()
    x = x.to(getattr(torch, kind))
    dy = torch.tensor([[0.5, -0.25]], dtype=x.dtype, device="cuda").expand(300, 2)
    wide = torch.zeros((300, 11), dtype=x.dtype, device="cuda")
    wide[:, 2:8] = x
    layers, results = m.answering(), []
    for u, d in ((x, dy.contiguous()), (x.t().contiguous().t(), dy), (wide[:, 2:8], dy.t().contiguous().t())):
        y = m.forward(u)
        m.backward(d)
        results.append([y, surrogate8.answer(layers, u)] + _grads(m))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))


def test_a_model_used_on_one_stream_after_another():
    """Steps that follow one another on streams of their own, the first held up:
    each has the gradients it has alone."""
    import torch
    batches = [_model_and_batch(n=n, seed=n)[1:] for n in (700, 700, 300, 700)]
    m = _model_and_batch()[0]
    want = []
    for x, dy in batches:
        m.forward(x)
        m.backward(dy)
        want.append(_grads(m))
    torch.cuda.synchronize()
    forwards, backwards = [torch.cuda.Stream() for _ in batches], [torch.cuda.Stream() for _ in batches]
    got = []
    for (x, dy), f, b in zip(batches, forwards, backwards):
        with torch.cuda.stream(f):
            torch.cuda._sleep(20_000_000)
            m.forward(x)
        with torch.cuda.stream(b):
            m.backward(dy)
            got.append(_grads(m))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(w, g))


# ---- scratch memory -------------------------------------------------------------


def test_linear_scratch_is_what_the_products_read():
    """Many points of a narrow layer form their codes where they multiply them:
    the scratch memory asked for stops growing there, and never shrinks."""
    import torch
    from test_gpu_dense8 import _linear, _np, _rand
    rows = [0, 1, 32, 33, 1000, 32767, 32768, 40000, 1 << 20, 1 << 30, (1 << 30) + 1, 2 ** 31 - 1]
    for n_in, n_out, fixed in ((512, 512, True), (200, 1024, True), (513, 64, False), (64, 1025, False)):
        layer = api.Linear8(torch.ones((n_out, n_in)))
        need = [layer.scratch_bytes(n) for n in rows]
        assert need[0] == 0 and need == sorted(need)
        assert (need[8] < 2 ** 25) == fixed and need[10] >= (1 << 30) * n_in
    W, x = _rand(81, (96, 130)), _rand(82, (40000, 130), "bf16")
    layer, y = api.Linear8(W), torch.empty((40000, 96), device="cuda")
    scratch = torch.full((layer.scratch_bytes(40000) + 64,), 7, dtype=torch.uint8, device="cuda")
    api.linear8(layer, x, y, RELU, scratch=scratch[:-64])
    want, size = _linear(x.float().cpu().numpy(), W.cpu().numpy(), None, RELU)
    assert (np.abs(_np(y) - want) <= 6 * 2.0 ** -24 * size + 1e-37).all() and (scratch[-64:] == 7).all()
    with pytest.raises(_abi.HpacmlError) as e:
        api.linear8(layer, x, y, RELU, scratch=scratch[:-80])
    assert e.value.status == _abi.E_RANGE


def test_linear_weights_beyond_their_allocation_are_refused():
    """Device weights and biases that would be read past the end of what was
    allocated for them."""
    import ctypes as C
    import torch
    L, h = _abi.lib(), C.c_void_p()
    small, host = torch.zeros(256, device="cuda"), torch.zeros(1 << 15)
    n = _abi.MAX_WIDTH8
    assert L.hpacml8_linear_create(n, n, small.data_ptr(), None, C.byref(h)) == _abi.E_RANGE and not h.value
    torch.cuda.empty_cache()
    big = torch.zeros(64 << 18, device="cuda")            # 64 MB: not a piece of what torch holds, so an allocation of its own
    assert L.hpacml8_linear_create(1, 8, small.data_ptr(), big.data_ptr() + big.numel() * 4 - 28, C.byref(h)) == _abi.E_RANGE
    assert not h.value
    for W, b in ((small, big[-8:]), (host, host), (host, small), (host.pin_memory(), None)):
        assert L.hpacml8_linear_create(1, 8, W.data_ptr(), None if b is None else b.data_ptr(), C.byref(h)) == _abi.OK
        L.hpacml8_linear_destroy(h)
        h = C.c_void_p()


def test_linear_weights_of_the_device():
    """They give the layer that the same weights on the host give, also where
    another stream is still writing them, or they begin at an odd address."""
    import ctypes as C
    import torch
    from test_gpu_dense8 import _rand
    W, x = _rand(91, (2048, 4096)), _rand(92, (9, 4096), "bf16")
    want, y = torch.empty((9, 2048), device="cuda"), torch.empty((9, 2048), device="cuda")
    api.linear8(api.Linear8(W.cpu()), x, want)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        torch.cuda._sleep(10_000_000)
        late = W.clone()
    torch.cuda.empty_cache()
    layer = api.Linear8(late)
    late.zero_()                                    # nothing of it is needed any more
    api.linear8(layer, x, y)
    assert torch.equal(y, want)
    odd = torch.zeros(W.numel() * 4 + 64, dtype=torch.uint8, device="cuda")
    odd[2:2 + W.numel() * 4] = W.contiguous().view(-1).view(torch.uint8)
    torch.cuda.synchronize()
    h = C.c_void_p()
    assert _abi.lib().hpacml8_linear_create(4096, 2048, odd.data_ptr() + 2, None, C.byref(h)) == _abi.OK
    layer.close()
    layer.handle = h
    y.zero_()
    api.linear8(layer, x, y)
    assert torch.equal(y, want)


def test_a_training_step_replayed_from_a_graph():
    """A step captured after one on another stream, replayed between eager steps
    with other inputs: each has the eager steps' gradients."""
    import torch
    m, x, dy = _model_and_batch(n=1100)
    batches = [_model_and_batch(n=1100, seed=s)[1:] for s in (3, 4, 5)]
    want = []
    for u, d in batches:
        m.forward(u)
        m.backward(d)
        want.append(_grads(m))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.forward(x)
        m.backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = m.forward(x)
        m.backward(dy)
    for again in range(2):
        for (u, d), w in zip(batches, want):
            x.copy_(u)
            dy.copy_(d)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(_grads(m), w))
            eager = m.forward(u)
            m.backward(d)
            assert torch.equal(eager, y) and all(torch.equal(p, q) for p, q in zip(_grads(m), w))
