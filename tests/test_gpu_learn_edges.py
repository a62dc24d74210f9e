"""GPU tests of the layers in 8-bit floats, group norm and clipping together and
at their edges: other alignments and streams, graphs, operands that overlap,
offsets beyond 32 bits, and the class that trains with them."""
import math

import pytest
import torch

from paper_2407_18352_amd import _abi, api, surrogatef8
from test_gpu_f8 import BF16, F32, loaded, quantized, values

pytestmark = pytest.mark.gpu


def moved(t, by=1):
    """The same values at an address `by` elements further, inside wider rows."""
    room = torch.zeros((t.shape[0], t.shape[1] + by + 2), dtype=t.dtype, device="cuda")
    room[:, by : by + t.shape[1]] = t
    return room[:, by : by + t.shape[1]]


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("n, n_in, n_out", [(5, 256, 64), (300, 256, 512), (1000, 130, 33)])
def test_any_alignment_gives_the_same_bits(n, n_in, n_out, kind):
    g = torch.Generator().manual_seed(n)
    x, dy, W = values(g, n, n_in, kind), values(g, n, n_out, kind), torch.randn((n_out, n_in), generator=g)
    layer = api.LinearF8(W, torch.randn(n_out, generator=g), learn=True)
    got = []
    for move in (lambda t: t, moved, lambda t: moved(t, 3)):
        kept, y = api.MatrixF8(n_in, n), move(torch.zeros((n, n_out), dtype=kind, device="cuda"))
        api.linearf8(layer, move(x), y, _abi.ACT_RELU, kept=kept)
        dw, db, dx = move(torch.empty((n_out, n_in), device="cuda")), torch.empty(n_out, device="cuda"), move(torch.empty((n, n_in), dtype=kind, device="cuda"))
        api.backwardf8(kept, move(dy), dw, db, layer=layer, dx=dx, y=y)
        back = move(torch.empty((n_in, n), dtype=kind, device="cuda"))
        api.loadf8(kept, back)
        z, mean, rstd = move(torch.empty((n, n_out), dtype=kind, device="cuda")), torch.empty((n, 1), device="cuda"), torch.empty((n, 1), device="cuda")
        api.group_norm(y, z, 1, 1, act=_abi.ACT_SILU, mean=mean, rstd=rstd)
        dz = move(torch.empty((n, n_out), dtype=kind, device="cuda"))
        api.group_norm_backward(y, move(dy), 1, 1, mean, rstd, dz, act=_abi.ACT_SILU)
        got.append([y, dw, db, dx, back, z, dz])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n", [1, 33, 100, 300])
def test_rows_and_columns_beyond_are_left(n):
    g = torch.Generator().manual_seed(n)
    n_in, n_out = 200, 70
    layer = api.LinearF8(torch.randn((n_out, n_in), generator=g), learn=True)
    x = values(g, n, n_in, BF16)
    y, dx = torch.full((n + 3, n_out + 5), 7.0, dtype=BF16, device="cuda"), torch.full((n + 3, n_in + 5), 7.0, dtype=BF16, device="cuda")
    dw, kept = torch.full((n_out + 2, n_in + 5), 7.0, device="cuda"), api.MatrixF8(n_in, n)
    api.linearf8(layer, x, y[:n, :n_out], kept=kept)
    api.backwardf8(kept, y[:n, :n_out], dw[:n_out, :n_in], layer=layer, dx=dx[:n, :n_in])
    for t, r, c in ((y, n, n_out), (dx, n, n_in), (dw, n_out, n_in)):
        assert (t[r:] == 7).all() and (t[:, c:] == 7).all() and not (t[:r, :c] == 7).all()
    for points in (1, n):
        z = torch.full((n + 3, n_out + 5), 7.0, dtype=BF16, device="cuda")
        api.group_norm(y[:n, :n_out], z[:n, :n_out], points, 7)
        assert (z[n:] == 7).all() and (z[:, n_out:] == 7).all()


def chain(n, seed):
    """A training step's calls on buffers of their own; (the call, its outputs)."""
    g = torch.Generator().manual_seed(seed)
    n_in, n_out = 96, 128
    x, W, b = values(g, n, n_in, BF16), torch.randn((n_out, n_in), generator=g).cuda(), torch.randn(n_out, generator=g).cuda()
    gamma, beta, dy = torch.ones(n_out, device="cuda") * 1.1, torch.zeros(n_out, device="cuda"), values(g, n, n_out, BF16)
    layer, kept = api.LinearF8(W, b, learn=True), api.MatrixF8(n_in, n)
    new = lambda *s, kind=F32: torch.zeros(s, dtype=kind, device="cuda")     # noqa: E731
    z, a, dz, dx = new(n, n_out, kind=BF16), new(n, n_out, kind=BF16), new(n, n_out, kind=BF16), new(n, n_in, kind=BF16)
    mean, rstd, dgamma, dbeta, dw, db, norm = new(n, 4), new(n, 4), new(n_out), new(n_out), new(n_out, n_in), new(n_out), new(1)
    clipped = [torch.zeros_like(t) for t in (dw, db, dgamma, dbeta)]
    grads = api.GradientSet([dw, db, dgamma, dbeta], into=clipped)
    need = max(layer.scratch_bytes(n), api.backwardf8_scratch_bytes(kept, dz), api.group_norm_scratch_bytes(z, 1, 4, True), grads.scratch_bytes())
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(stream=None):
        layer.update(W, b, stream=stream)
        api.linearf8(layer, x, z, kept=kept, scratch=scratch, stream=stream)
        api.group_norm(z, a, 1, 4, gamma, beta, act=_abi.ACT_SILU, mean=mean, rstd=rstd, scratch=scratch, stream=stream)
        api.group_norm_backward(z, dy, 1, 4, mean, rstd, dz, dgamma, dbeta, gamma, beta, _abi.ACT_SILU, scratch=scratch, stream=stream)
        api.backwardf8(kept, dz, dw, db, layer=layer, dx=dx, scratch=scratch, stream=stream)
        api.clip_gradients(grads, 0.5, norm, scratch=scratch, stream=stream)

    return call, [z, a, mean, rstd, dgamma, dbeta, dw, db, dx, norm] + clipped, (x, W)


@pytest.mark.parametrize("n", [7, 500, 5000])
def test_equal_calls_give_equal_bits(n):
    call, outs, _ = chain(n, 1)
    call()
    first = [t.clone() for t in outs]
    assert all(t.isfinite().all() for t in first)
    for _ in range(3):
        for t in outs:
            t.fill_(5)
        call()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))


@pytest.mark.parametrize("n", [7, 5000])
def test_replayed_from_a_graph_between_eager_calls(n):
    call, outs, (x, W) = chain(n, 2)
    call()                                             # before the capture: everything is built
    eager, eager_outs, (ex, eW) = chain(n, 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        new = torch.randn(x.shape, generator=torch.Generator().manual_seed(k)).to(x.dtype).cuda()
        for t, w in ((x, W), (ex, eW)):
            t.copy_(new)
            w.mul_(1.25)
        graph.replay()
        eager()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager_outs))


def test_other_streams():
    call, outs, _ = chain(3000, 3)
    call()
    want = [t.clone() for t in outs]
    other, again = chain(3000, 3), chain(3000, 3)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):                                 # two at a time, each with buffers of its own
        other[0](s)
        again[0](t)
    torch.cuda.synchronize()
    for got in (other[1], again[1]):
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    layer = api.LinearF8(torch.randn(8, 16))
    x, y = torch.randn((3, 16), device="cuda"), torch.empty((3, 8), device="cuda")
    with pytest.raises(ValueError):
        api.linearf8(layer, x, y, stream=s)            # a call on a stream of its own brings its scratch memory
    with pytest.raises(ValueError):
        layer.update(torch.randn((16, 8), device="cuda").t(), stream=s)


def test_two_graphs_that_share_scratch_memory():
    """One after another on a stream they may: nothing in it lives from call to call."""
    a, b = chain(400, 4), chain(400, 5)
    for c in (a, b):
        c[0]()
    want = [[t.clone() for t in c[1]] for c in (a, b)]
    torch.cuda.synchronize()
    graphs = []
    for c in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=None if len(graphs) == 1 else graphs[0].pool()):
            c[0]()
    for _ in range(3):
        for g in (graphs[0], graphs[1], graphs[1], graphs[0]):
            g.replay()
        torch.cuda.synchronize()
        for c, w in zip((a, b), want):
            assert all(torch.equal(p, q) for p, q in zip(c[1], w))


def refused(status, call):
    with pytest.raises(_abi.HpacmlError) as e:
        call()
    assert e.value.status == status


def test_operands_that_overlap_are_refused():
    layer, kept = api.LinearF8(torch.randn(64, 64), torch.randn(64), learn=True), api.MatrixF8(64, 300)
    room = torch.randn((300, 128), device="cuda")
    x, scratch = room[:, :64], torch.empty(layer.scratch_bytes(300), dtype=torch.uint8, device="cuda")
    refused(_abi.E_ALIAS, lambda: api.linearf8(layer, x, room[:, 32:96], scratch=scratch))
    refused(_abi.E_ALIAS, lambda: api.linearf8(layer, x, x, scratch=scratch))
    api.linearf8(layer, x, room[:, 64:], scratch=scratch)                        # columns of one record
    both = torch.empty(layer.scratch_bytes(300) + (1 << 20), dtype=torch.uint8, device="cuda")
    refused(_abi.E_ALIAS, lambda: api.linearf8(layer, x, torch.empty((300, 64), device="cuda"), kept=api.MatrixF8(64, 300, codes=both), scratch=both))
    dy, dw, db = torch.randn((300, 64), device="cuda"), torch.empty((64, 64), device="cuda"), torch.empty(64, device="cuda")
    refused(_abi.E_ALIAS, lambda: api.backwardf8(kept, dy, dw, db, layer=layer, dx=dy))
    refused(_abi.E_ALIAS, lambda: api.backwardf8(kept, dy, dw, dw[0], layer=layer))
    refused(_abi.E_ALIAS, lambda: api.quantizef8(dy, api.MatrixF8(300, 64, both), api.MatrixF8(64, 300, both)))
    refused(_abi.E_ALIAS, lambda: api.productf8(kept, kept, kept.codes.view(torch.float32)[:4096].view(64, 64)))
    m, r = torch.empty((300, 4), device="cuda"), torch.empty((300, 4), device="cuda")
    refused(_abi.E_ALIAS, lambda: api.group_norm(dy, dy, 1, 4))
    refused(_abi.E_ALIAS, lambda: api.group_norm(dy, torch.empty_like(dy), 1, 4, mean=m, rstd=m))
    refused(_abi.E_ALIAS, lambda: api.group_norm_backward(x, dy, 1, 4, m, r, dy))
    refused(_abi.E_ALIAS, lambda: api.group_norm_backward(x, dy, 1, 4, m, r, None, db, db))


def test_operands_beyond_their_memory_are_refused():
    x = torch.randn((300, 64), device="cuda")
    q = api.MatrixF8(300, 64)
    q.desc.rows = 1 << 28
    refused(_abi.E_SHAPE, lambda: api.quantizef8(x, q))
    q.desc.rows, q.desc.scales = 300, q.desc.codes + 8
    refused(_abi.E_INVAL, lambda: api.quantizef8(x, q))          # not aligned
    with pytest.raises(TypeError):
        api.quantizef8(x.cpu(), api.MatrixF8(300, 64))
    with pytest.raises(TypeError):
        api.MatrixF8(300, 64, codes=torch.empty(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError):
        api.MatrixF8(300, 64, codes=torch.empty(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        api.group_norm(x, torch.empty_like(x), 7, 4)              # 300 rows are no whole images of 7
    with pytest.raises(ValueError):
        api.group_norm(x, torch.empty_like(x), 1, 4, gamma=torch.ones(63, device="cuda"))
    with pytest.raises(ValueError):
        api.backwardf8(api.MatrixF8(64, 300), x, dx=torch.empty_like(x))
    layer = api.LinearF8(torch.randn(8, 64), torch.randn(8))
    with pytest.raises(ValueError):
        layer.update(torch.randn((8, 64), device="cuda"))
    with pytest.raises(ValueError):
        api.LinearF8(torch.randn(8, 64)[:, :0])


def test_offsets_beyond_32_bits():
    """Rows whose codes, inputs and results lie more than 2^32 bytes into their buffers: as the same rows alone."""
    n, width, m = 2200000, 2048, 300
    x = torch.empty((n, width), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(0, n, 100000):
        x[i : i + 100000] = torch.randn((100000, width), generator=g, device="cuda")
    W = torch.randn((96, width), generator=torch.Generator().manual_seed(2)) / 45
    layer = api.LinearF8(W)
    q = quantized(x)
    assert q.codes.numel() > 1 << 32
    y = torch.empty((n, 96), dtype=BF16, device="cuda")
    api.productf8(q, layer.W, y)
    # (the last 300 rows start a tile of 32 of their own only in the small call: rows do not depend on each other)
    alone = torch.empty((m, 96), dtype=BF16, device="cuda")
    api.productf8(quantized(x[n - m :]), layer.W, alone)
    assert torch.equal(y[n - m :], alone)
    del q
    z, small = torch.empty_like(x), torch.empty((m, width), dtype=BF16, device="cuda")
    api.group_norm(x, z, 1, 16, act=_abi.ACT_SILU)
    api.group_norm(x[n - m :], small, 1, 16, act=_abi.ACT_SILU)
    assert torch.equal(z[n - m :], small)
    mean, rstd = torch.empty((n // 1100, 16), device="cuda"), torch.empty((n // 1100, 16), device="cuda")
    api.group_norm(x, z, 1100, 16, mean=mean, rstd=rstd)       # images of 1100 points
    v = x[n - 1100 :].double().view(1100, 16, -1)
    want = ((v - v.mean((0, 2), keepdim=True)) / v.var((0, 2), unbiased=False, keepdim=True).add(1e-5).sqrt()).view(1100, width)
    assert ((z[n - 1100 :].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2e-5).all()


def test_more_blocks_than_a_grid():
    """Integers up to 8, which codes hold exactly: what comes of them is exact."""
    wide = torch.empty((33, (1 << 26) + 1000), dtype=BF16, device="cuda").random_(-8, 9)
    back = torch.full_like(wide, 99)
    api.loadf8(quantized(wide), back)                          # 2^20 blocks of 32 rows x 128 values, and more
    assert all(torch.equal(a, b) for a, b in zip(wide, back))
    del wide, back
    n_out = (1 << 22) + 777                                    # 2^16 sums of 64 columns, and more
    dy, db = torch.empty((3, n_out), dtype=BF16, device="cuda").random_(-8, 9), torch.empty(n_out, device="cuda")
    api.backwardf8(api.MatrixF8(1, 3), dy, db=db)
    assert torch.equal(db, dy.float().sum(0))
    n_out = (1 << 24) + 33                                     # of one row: more outputs than one launch for few rows has threads for
    W, x, y = torch.empty((n_out, 5), dtype=BF16, device="cuda").random_(-8, 9), torch.empty((1, 5), device="cuda").random_(-8, 9), torch.empty((1, n_out), device="cuda")
    api.productf8(quantized(x), quantized(W), y)
    assert torch.equal(y[0], (W.float() * x).sum(1))


def test_a_product_of_few_and_many_rows_agree():
    """The forms for few rows and for many, on the same whole numbers."""
    g = torch.Generator().manual_seed(4)
    W = torch.randint(-8, 9, (600, 1000), generator=g).float()
    x = torch.randint(-8, 9, (65, 1000), generator=g).float().cuda()
    layer = api.LinearF8(W)
    for kind in (F32, BF16):
        y = torch.empty((65, 600), dtype=kind, device="cuda")
        api.linearf8(layer, x, y)
        assert torch.equal(y.cpu(), (x.cpu().double() @ W.double().t()).to(kind))
        for n in (1, 15, 16, 17, 32, 33, 64):
            few = torch.empty((n, 600), dtype=kind, device="cuda")
            api.linearf8(layer, x[:n], few)
            assert torch.equal(few, y[:n])


@pytest.mark.parametrize("n, n_in, n_out", [(16, 12200, 100), (16, 12300, 100), (17, 6100, 130), (17, 6200, 130), (32, 6100, 33), (33, 3000, 70), (33, 3100, 70),
                                            (64, 3000, 5), (64, 3100, 5), (65, 300, 40), (1, 4096, 4096), (1, 4097, 4097), (2, 130, 12288), (2, 130, 12289),
                                            (40, 1024, 4097), (40, 1025, 4097)])
def test_sizes_beside_the_rule_for_few_rows(n, n_in, n_out):
    """Whole numbers, whose sums fp32 holds."""
    g = torch.Generator().manual_seed(n + n_in)
    W, x = torch.randint(-8, 9, (n_out, n_in), generator=g).float().cuda(), torch.randint(-8, 9, (n, n_in), generator=g).float().cuda()
    b = torch.randint(-8, 9, (n_out,), generator=g).float().cuda()
    want = (x.double() @ W.double().t() + b).relu()
    layer = api.LinearF8(W, b)
    for kind in (F32, BF16):
        y = torch.empty((n, n_out), dtype=kind, device="cuda")
        api.linearf8(layer, x.to(kind), y, act=_abi.ACT_RELU)
        assert torch.equal(y, want.to(kind))
        y = torch.empty((n, n_out), dtype=kind, device="cuda")
        api.productf8(quantized(x), layer.W, y, b, act=_abi.ACT_RELU)
        assert torch.equal(y, want.to(kind))


# ---- the class that trains with them ---------------------------------------------


def norms(model, x, dy):
    """fp32 autograd's outputs and gradients of the same model (group norm from elementary operations: torch's own gives other
    gradients of its parameters here for more than 128 rows)."""
    a = x
    for l, (W, b) in enumerate(zip(model.W, model.b)):
        a = a @ W.t() + b
        if l < len(model.W) - 1:
            v = a.view(a.shape[0], model.groups, -1)
            d = v - v.mean(2, keepdim=True)
            h = (d / (d.square().mean(2, keepdim=True) + model.eps).sqrt()).view(a.shape)
            a = torch.nn.functional.silu(h * model.gamma[l] + model.beta[l])
    return a.detach(), torch.autograd.grad((a * dy).sum(), model.parameters())


def test_surrogate_gradients_and_clipping():
    """Against fp32.  An e4m3 value is off by at most 2^-4, in the mean square by less than 2^-4 / sqrt(3) (3.6 %), a product of two by 5.1 %;
    a gradient has at most three products forward and three back behind it: sqrt(6) * 5.1 % = 12.5 % of its norm."""
    g = torch.Generator().manual_seed(5)
    model = surrogatef8.SurrogateF8([5, 64, 96, 3], groups=8)
    x, dy = torch.randn((777, 5), generator=g).cuda(), torch.randn((777, 3), generator=g).cuda()
    y = model.forward(x)
    assert torch.equal(model.answer(x), y)
    want, grads = norms(model, x, dy)
    model.backward(dy)
    assert (y - want).norm() <= 0.125 * want.norm()
    for p, w in zip(model.parameters(), grads):
        assert (p.grad - w).norm() <= 0.125 * w.norm()
    kept = [p.grad.clone() for p in model.parameters()]
    model.backward(dy, accumulate=True)
    for p, k in zip(model.parameters(), kept):
        assert torch.allclose(p.grad, 2 * k, rtol=1e-6, atol=1e-6 * float(k.abs().max()))
    total = math.sqrt(sum(float(p.grad.double().square().sum()) for p in model.parameters()))
    norm = model.clip(0.1)
    assert abs(norm.item() - total) <= 1e-6 * total
    after = math.sqrt(sum(float(p.grad.double().square().sum()) for p in model.parameters()))
    assert abs(after - 0.1) <= 1e-6
    for p in model.parameters():                     # an optimizer that drops its gradients
        p.grad = None
    with pytest.raises(ValueError):
        model.clip(0.1)
    model.backward(dy)
    model.clip(1e9)
    assert all(torch.equal(p.grad, k) for p, k in zip(model.parameters(), kept))


def test_surrogate_batches_streams_and_updates():
    model, same = surrogatef8.SurrogateF8([4, 32, 2], groups=4, seed=3), surrogatef8.SurrogateF8([4, 32, 2], groups=4, seed=3)
    g = torch.Generator().manual_seed(6)
    side = torch.cuda.Stream()
    for n in (3, 100, 1, 0, 70):
        x, dy = torch.randn((n, 4), generator=g).cuda(), torch.randn((n, 2), generator=g).cuda()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = model.forward(x)
        model.backward(dy)                           # on another stream than the forward pass
        z = same.forward(x)
        same.backward(dy)
        torch.cuda.synchronize()
        assert torch.equal(y, z) and all(torch.equal(p.grad, q.grad) for p, q in zip(model.parameters(), same.parameters()))
    with torch.no_grad():
        model.W[-1].mul_(2)                          # (of the first, group norm would take it away again)
    x = torch.randn((9, 4), generator=g).cuda()
    assert torch.equal(model.forward(x), same.forward(x))       # before the update the weights laid out are the old ones
    model.update()
    assert not torch.equal(model.forward(x), same.forward(x))
    with pytest.raises(ValueError):
        surrogatef8.SurrogateF8([4, 30, 2], groups=4)


def test_surrogate_captured_into_a_graph():
    """A step's passes and its clipping replayed between eager ones of another size, whose buffers replace those of the passes before the capture."""
    g = torch.Generator().manual_seed(9)
    model, same = surrogatef8.SurrogateF8([4, 32, 2], groups=4, seed=3), surrogatef8.SurrogateF8([4, 32, 2], groups=4, seed=3)
    x, dy = torch.randn((150, 4), generator=g).cuda(), torch.randn((150, 2), generator=g).cuda()
    for _ in range(2):
        model.forward(x)
        model.backward(dy)
        model.clip(0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = model.forward(x)
        model.backward(dy)
        norm = model.clip(0.5)
    other = torch.randn((40, 4), generator=g).cuda()
    for k in range(3):
        model.forward(other)
        model.backward(dy[:40])
        taken = [torch.full((4096,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]     # what the first passes' buffers left
        x.copy_(torch.randn((150, 4), generator=g))
        graph.replay()
        want = same.forward(x)
        same.backward(dy)
        total = same.clip(0.5)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(norm, total)
        assert all(torch.equal(p.grad, q.grad) for p, q in zip(model.parameters(), same.parameters()))
        assert all(bool((t == 255).all()) for t in taken)
        with torch.no_grad():
            for m in (model, same):
                m.W[0].mul_(1.5)
                m.update()
    held = model.set
    for p in model.parameters():                     # other gradients: a set of their own, and the graph's stays
        p.grad = None
    model.backward(dy[:40])
    model.clip(0.5)
    assert model.set is not held and held.handle
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, model.answer(x)) and torch.isfinite(norm).all()


def test_surrogate_calls_out_of_order():
    model = surrogatef8.SurrogateF8([4, 32, 2], groups=4)
    with pytest.raises(ValueError):
        model.backward(torch.zeros((3, 2), device="cuda"))
    graph = torch.cuda.CUDAGraph()
    t = torch.zeros(3, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        t.add_(1)
        with pytest.raises(RuntimeError):
            api.GradientSet([t])                     # synchronises: not in a capture
    graph.replay()
    assert t.tolist() == [1, 1, 1]


def test_surrogate_command_runs():
    loss, rms = surrogatef8.main(["--points", "2000", "--dims", "5,64,64,1", "--steps", "3"])
    assert math.isfinite(loss) and math.isfinite(rms)
