"""GPU tests on whole numbers, whose sums fp32 holds: products and layers of the
large tiles, and gradients of parameters, of which a lost row, point, slab or
image shows."""
import pytest
import torch

from paper_2407_18352_amd import _abi, api
from test_gpu_f8 import BF16, F32, quantized
from test_gpu_group_norm import EPS, HALF, NONE, RELU, SILU, forward

pytestmark = pytest.mark.gpu

# n, m, width: tiles of 256 x 256, of which blocks take several, whole ones and not, few slabs and many; in parts of the width, of one length and not
LARGE = [(4099, 4001, 520), (4096, 4096, 512), (8449, 2049, 1000), (700, 66000, 601), (2049, 2049, 24700), (257, 300, 32768), (1537, 1500, 6 * 64 * 128), (1025, 1400, 131)]
# rows, in, out: the three products of a layer
LAYERS = [(32900, 520, 400), (82001, 1100, 1100), (131073, 300, 77)]


def whole(g, most, *shape):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda")


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("n, m, k", LARGE)
def test_products_of_large_tiles(n, m, k, kind):
    g = torch.Generator(device="cuda").manual_seed(n + m + k)
    blocks = -(-k // 128)
    assert k * 64 < 2 ** 24

    def matrix(rows):        # scales of their own for every row and block
        scale = torch.exp2(torch.randint(0, 2, (rows, blocks), generator=g, device="cuda").float()).repeat_interleave(128, 1)[:, :k]
        return whole(g, 4, rows, k) * scale

    p, q = matrix(n), matrix(m)
    b, old = whole(g, 50, m).float(), whole(g, 9, n, m).float()
    want = (p.double() @ q.double().t()).float()
    p, q = quantized(p), quantized(q)
    y = torch.full((n, m + 3), 7.0, dtype=kind, device="cuda")
    api.productf8(p, q, y[:, :m])
    assert torch.equal(y[:, :m], want.to(kind)) and (y[:, m:] == 7).all()
    api.productf8(p, q, y[:, :m], b, _abi.ACT_RELU)
    assert torch.equal(y[:, :m], torch.relu(want + b).to(kind)) and (y[:, m:] == 7).all()
    if kind == F32:
        y[:, :m] = old
        api.productf8(p, q, y[:, :m], accumulate=True)
        assert torch.equal(y[:, :m], want + old) and (y[:, m:] == 7).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("n, n_in, n_out", LAYERS)
def test_layers_of_large_tiles(n, n_in, n_out, kind):
    g = torch.Generator(device="cuda").manual_seed(n)
    x, dy, W, b = (whole(g, 4, n, n_in).to(kind), (whole(g, 3, n, n_out) * 2 + 1).to(kind), whole(g, 3, n_out, n_in).float(), whole(g, 20, n_out).float())
    assert n * 28 < 2 ** 24          # of the sums of rows: 4 * 7 each
    layer, kept, y = api.LinearF8(W, b, learn=True), api.MatrixF8(n_in, n), torch.empty((n, n_out), dtype=kind, device="cuda")
    api.linearf8(layer, x, y, _abi.ACT_RELU, kept=kept)
    assert torch.equal(y, torch.relu(x.double() @ W.double().t() + b).to(kind))
    dz = torch.where(y > 0, dy, torch.zeros_like(dy)).double()
    dw, db, dx = torch.full((n_out, n_in), 7.0, device="cuda"), torch.full((n_out,), 7.0, device="cuda"), torch.empty((n, n_in), dtype=kind, device="cuda")
    api.backwardf8(kept, dy, dw, db, layer=layer, dx=dx, y=y)
    assert torch.equal(dx, (dz @ W.double()).to(kind))
    want = dz.t().contiguous() @ x.double()
    assert torch.equal(dw, want.float()) and torch.equal(db, dz.sum(0).float())
    api.backwardf8(kept, dy, db=db)                  # no ReLU: every row counts, an odd number of times
    assert torch.equal(db, dy.double().sum(0).float())
    api.backwardf8(kept, dy, dw, db, y=y, accumulate=True)
    assert torch.equal(dw, 2 * want.float()) and torch.equal(db, (dy.double() + dz).sum(0).float())


#               images, points, channels, groups: of one point
ONE_POINT = [(70001, 1, 64, 8), (9001, 1, 40, 5), (4099, 1, 1024, 2), (70001, 1, 7, 7), (3, 1, 1001, 1)]
# groups in a block's registers: blocks go on to further images, which are shared out unequally
HELD = [(2500, 3, 8, 1), (1111, 16, 128, 8), (2100, 5, 45, 9), (600, 1024, 128, 8), (5000, 2, 1024, 4)]
# in parts
PARTS = [(1, 70001, 8, 2), (3, 4097, 3, 3), (1, 20000, 130, 10), (2, 300, 1024, 1), (1, 1 << 20, 1, 1), (37, 5003, 16, 4)]


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", ONE_POINT + HELD + PARTS)
def test_gradients_of_parameters_lose_no_point(case, kind):
    """x - mean and dy are odd, so that every point counts in every sum."""
    images, points, channels, groups = case
    n = images * points
    g = torch.Generator(device="cuda").manual_seed(n + channels)
    x, dy = (whole(g, 1, n, channels + 3) * 2 + 1).to(kind)[:, :channels], (whole(g, 1, n, channels + 1) * 2 + 1).to(kind)[:, :channels]
    assert n * 5 * 3 * 2 < 2 ** 26   # multiples of 4
    mean, rstd = whole(g, 1, images, groups) * 2.0, torch.full((images, groups), 4.0, device="cuda")
    d = ((x.double().view(images, points, groups, -1) - mean.double().view(images, 1, groups, 1)) * 4).view(n, channels)
    for act in (NONE, RELU):
        dz = dy.double() if act == NONE else torch.where(d > 0, dy.double(), torch.zeros_like(d))
        want = ((dz * d).sum(0).float(), dz.sum(0).float())
        for dx in (None, torch.empty((n, channels), dtype=kind, device="cuda")):
            got = torch.full((channels,), 7.0, device="cuda"), torch.full((channels,), 7.0, device="cuda")
            api.group_norm_backward(x, dy, points, groups, mean, rstd, dx, *got, act=act)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        api.group_norm_backward(x, dy, points, groups, mean, rstd, None, *got, act=act, accumulate=True)
        assert all(torch.equal(a, 2 * b) for a, b in zip(got, want))


@pytest.mark.parametrize("act", [NONE, SILU])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", HELD)
def test_blocks_that_go_from_image_to_image(case, kind, act):
    images, points, channels, groups = case
    n, per = images * points, channels // groups
    g = torch.Generator().manual_seed(n)
    level = torch.randn((images, 1, groups, 1), generator=g) * 3          # every image's and group's own
    x = (torch.randn((images, points, groups, per), generator=g) * torch.exp2(level) + level).view(n, channels).to(kind).cuda()
    dy = (torch.randn((n, channels), generator=g) * torch.exp2(level).expand(-1, points, -1, per).reshape(n, channels)).to(kind).cuda()
    gamma, beta = 1 + torch.randn(channels, generator=g).cuda() * 0.3, torch.randn(channels, generator=g).cuda()
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
    api.group_norm(x, y, points, groups, gamma, beta, EPS, act, mean, rstd)
    want, wm, wr, h, z = forward(x, points, groups, gamma, beta, act)
    # a rounding of the mean; of the variance and its reciprocal root
    assert ((mean.double() - wm).abs() <= 2.0 ** -24 * wm.abs() + 2.0 ** -40 / wr).all() and ((rstd.double() - wr).abs() <= 2.0 ** -22 * wr).all()

    def wide(t):
        return t.double().view(images, 1, groups, 1).expand(images, points, groups, per).reshape(n, channels)

    # z by the mean's rounding, rstd's, its own four; SiLU's slope is below 1.1, its own error 2^-20 of z and of |z| 2^-22
    off = 2.0 ** -24 * wide(wm * wr).abs() * gamma.abs() + 2.0 ** -20 * (h.abs() * gamma.abs() + beta.abs())
    assert ((y.double() - want).abs() <= HALF[kind] * want.abs() + 1.2 * off + (2.0 ** -20 * z.abs() * (1 + z.abs()) if act == SILU else 0) + 2.0 ** -130).all()
    alone = torch.empty_like(y)
    for i in (0, images // 2, images - 1):           # as an image alone
        rows = slice(i * points, (i + 1) * points)
        api.group_norm(x[rows], alone[rows], points, groups, gamma, beta, EPS, act)
        assert torch.equal(alone[rows], y[rows])
    api.group_norm_backward(x, dy, points, groups, mean, rstd, dx, None, None, gamma, beta, act)
    _, _, _, h, z = forward(x, points, groups, gamma, beta, act, moments=(mean, rstd))
    s = torch.sigmoid(z)
    gg = dy.double() * (s * (1 + z * (1 - s)) if act == SILU else 1) * gamma.double()

    def over(t):
        return t.view(images, points, groups, per).mean((1, 3), keepdim=True).expand(images, points, groups, per).reshape(n, channels)

    r = wide(rstd)
    want = r * (gg - over(gg) - h * over(gg * h))
    # each term by its roundings, the means by up to forty additions in a row of 2^-24 each; the slope of SiLU, below 1.1, by those of its
    # terms and by z's
    size = dy.double().abs() * gamma.double().abs() * ((1.1 + z.abs()) * (2 + z.abs()) if act == SILU else 1)
    terms = r * (size + over(size) + h.abs() * over(size * h.abs()))
    assert ((dx.double() - want).abs() <= HALF[kind] * want.abs() + 2.0 ** -18 * terms + 2.0 ** -130).all()
