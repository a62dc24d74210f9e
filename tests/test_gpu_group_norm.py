"""GPU tests of group norm with an activation and of its backward pass, against
their formulas in 64 bits."""
import math

import pytest
import torch

from paper_2407_18352_amd import _abi, api

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
NONE, RELU, SILU = _abi.ACT_IDENTITY, _abi.ACT_RELU, _abi.ACT_SILU
EPS = 1e-5


def forward(x, points, groups, gamma, beta, act, eps=EPS, moments=None):
    """(y, mean, rstd, h, z) in 64 bits, rows as x."""
    rows, channels = x.shape
    v = x.double().view(rows // points, points, groups, channels // groups)
    if moments is None:
        mean = v.mean((1, 3), keepdim=True)
        rstd = 1 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + eps)
    else:
        mean, rstd = (m.double().view(rows // points, 1, groups, 1) for m in moments)
    h = ((v - mean) * rstd).reshape(rows, channels)
    z = h * (gamma.double() if gamma is not None else 1) + (beta.double() if beta is not None else 0)
    y = {NONE: lambda: z, RELU: lambda: torch.relu(z), SILU: lambda: z * torch.sigmoid(z)}[act]()
    return y, mean.view(-1, groups), rstd.view(-1, groups), h, z


def data(g, images, points, channels, kind, pad):
    x = torch.randn((images * points, channels + pad), generator=g) * 2 + torch.randn(channels + pad, generator=g)
    dy = torch.randn((images * points, channels + pad), generator=g)
    return x.to(kind).cuda()[:, :channels], dy.to(kind).cuda()[:, :channels]


#        images, points, channels, groups
CASES = [(1, 1, 1, 1), (3, 1, 8, 2), (5, 1, 7, 7), (1, 1, 16384, 4), (70, 1, 512, 16), (1000, 1, 64, 2), (33, 1, 30, 5), (2, 3, 8, 1), (7, 49, 45, 9),
         (2, 1000, 24, 3), (1, 70001, 8, 2), (3, 4097, 3, 3), (2, 300, 1024, 1), (1, 5, 16384, 1), (130, 16, 128, 8), (2, 2500, 96, 32), (1, 20000, 130, 10)]


def bound(kind, want, h, n):
    """fp32 error of (x - mean) * (rstd * gamma) + beta and what follows: mean's rounding and that of the sums behind it (a handful of
    roundings each of the size of the values), the type's own rounding."""
    return HALF[kind] * want.abs() + 2.0 ** -24 * (64 + 8 * h.abs()) + 2.0 ** -130


@pytest.mark.parametrize("act", [NONE, RELU, SILU])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, kind, act):
    images, points, channels, groups = case
    pad = 0 if channels % 8 == 0 and channels > 24 else 3
    g = torch.Generator().manual_seed(channels + points)
    x, _ = data(g, images, points, channels, kind, pad)
    gamma, beta = 1 + torch.randn(channels, generator=g).cuda() * 0.3, torch.randn(channels, generator=g).cuda()
    y = torch.full((images * points, channels + 5), 9.0, dtype=kind, device="cuda")
    mean, rstd = torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
    for par in ((gamma, beta), (None, None)):
        api.group_norm(x, y[:, :channels], points, groups, *par, EPS, act, mean, rstd)
        want, wm, wr, h, _ = forward(x, points, groups, *par, act)
        assert (y[:, channels:] == 9).all()
        most = x.double().abs().max()
        assert ((mean.double() - wm).abs() <= 2.0 ** -22 * most).all()
        # the variance's relative error, twice the size of rstd's: 64-bit joins of fp32 sums of squares about a near value
        assert ((rstd.double() - wr).abs() <= 2.0 ** -20 * wr).all()
        scale = wr.abs().max() * most * (1 + gamma.abs().max())      # an error of mean and x - mean, as z sees it
        assert ((y[:, :channels].double() - want).abs() <= bound(kind, want, h, points) + 2.0 ** -22 * scale).all()
    again = torch.empty((images * points, channels), dtype=kind, device="cuda")
    api.group_norm(x, again, points, groups, act=act)        # without moments: the same
    assert torch.equal(again, y[:, :channels])


@pytest.mark.parametrize("act", [NONE, RELU, SILU])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", CASES)
def test_backward(case, kind, act):
    images, points, channels, groups = case
    pad = 0 if channels % 8 == 0 and channels > 24 else 3
    g = torch.Generator().manual_seed(channels + points + 1)
    x, dy = data(g, images, points, channels, kind, pad)
    gamma, beta = 1 + torch.randn(channels, generator=g).cuda() * 0.3, torch.randn(channels, generator=g).cuda()
    y = torch.empty((images * points, channels), dtype=kind, device="cuda")
    mean, rstd = torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
    for par in ((gamma, beta), (None, None)):
        api.group_norm(x, y, points, groups, *par, EPS, act, mean, rstd)
        dx = torch.full((images * points, channels + 5), 9.0, dtype=kind, device="cuda")
        dgamma, dbeta = torch.ones(channels, device="cuda"), torch.ones(channels, device="cuda")
        api.group_norm_backward(x, dy, points, groups, mean, rstd, dx[:, :channels], dgamma, dbeta, *par, act)
        assert (dx[:, channels:] == 9).all()
        _, _, _, h, z = forward(x, points, groups, *par, act, moments=(mean, rstd))
        s = torch.sigmoid(z)
        if act == RELU:      # z as fp32 operands give it
            v = x.float().view(images, points, groups, -1)
            d = (v - mean.view(images, 1, groups, 1)).double()
            a = (rstd.view(images, 1, groups, 1) * (par[0] if par[0] is not None else torch.ones_like(gamma)).view(1, 1, groups, -1)).double()
            z = (d * a).reshape(z.shape) + (par[1].double() if par[1] is not None else 0)
        gz = dy.double() * {NONE: torch.ones_like(z), RELU: (z > 0).double(), SILU: s * (1 + z * (1 - s))}[act]
        gg = gz * (par[0].double() if par[0] is not None else 1)

        def over(t):
            return t.view(images, points, groups, -1).mean((1, 3), keepdim=True).expand(images, points, groups, channels // groups).reshape(t.shape)

        wide = rstd.double().view(images, 1, groups, 1).expand(images, points, groups, channels // groups).reshape(z.shape)
        want = wide * (gg - over(gg) - h * over(gg * h))
        # a few fp32 roundings of each term
        terms = wide * (gg.abs() + over(gg.abs()) + h.abs() * over((gg * h).abs()))
        z_off = 2.0 ** -21 * wide * (gg.abs() + over(gg.abs())) * (1 + z.abs()) if act == SILU else 0
        assert ((dx[:, :channels].double() - want).abs() <= HALF[kind] * want.abs() + 2.0 ** -20 * terms + z_off + 2.0 ** -130).all()
        rows = images * points
        # s (1 + z (1 - s)) passes zero: its error is that of its terms, s (1 + |z| (1 - s)), by a few roundings and by z's own, which
        # moves it by less than |z| 2^-22
        size = dy.double().abs() * (s * (1 + z.abs() * (1 - s)) + z.abs() if act == SILU else 1)
        for got, each, most in ((dgamma, gz * h, size * h.abs()), (dbeta, gz, size)):
            tol = (2.0 ** -24 * (math.log2(rows + 1) + 64) * 8) * (most + 2.0 ** -20).sum(0)
            assert ((got.double() - each.sum(0)).abs() <= tol).all()
        for which in ("dx", "dgamma", "dbeta"):
            t = {"dx": torch.empty_like(y), "dgamma": torch.empty_like(dgamma), "dbeta": torch.empty_like(dbeta)}[which]
            api.group_norm_backward(x, dy, points, groups, mean, rstd, **{which: t}, gamma=par[0], beta=par[1], act=act)
            assert torch.equal(t, {"dx": dx[:, :channels], "dgamma": dgamma, "dbeta": dbeta}[which])
        more = [dgamma.clone(), dbeta.clone()]
        api.group_norm_backward(x, dy, points, groups, mean, rstd, None, *more, *par, act, accumulate=True)
        assert torch.equal(more[0], 2 * dgamma) and torch.equal(more[1], 2 * dbeta)


def test_gradients_by_differences():
    """The gradients against central differences of the formula's forward pass in 64 bits."""
    g = torch.Generator().manual_seed(3)
    images, points, channels, groups = 2, 6, 12, 3
    x, dy = data(g, images, points, channels, F32, 0)
    gamma, beta = 1 + torch.randn(channels, generator=g).cuda() * 0.3, torch.randn(channels, generator=g).cuda()
    mean, rstd, y, dx = (torch.empty(s, device="cuda") for s in ((images, groups), (images, groups), x.shape, x.shape))
    dgamma, dbeta = torch.empty(channels, device="cuda"), torch.empty(channels, device="cuda")
    api.group_norm(x, y, points, groups, gamma, beta, EPS, SILU, mean, rstd)
    api.group_norm_backward(x, dy, points, groups, mean, rstd, dx, dgamma, dbeta, gamma, beta, SILU)
    at = [x.double(), gamma.double(), beta.double()]

    def loss(v):
        return (forward(v[0], points, groups, v[1], v[2], SILU)[0] * dy.double()).sum().item()

    for which, got in enumerate((dx, dgamma, dbeta)):
        for i in range(0, got.numel(), 7):
            step = 1e-4
            ends = []
            for s in (step, -step):
                v = [t.clone() for t in at]
                v[which].view(-1)[i] += s
                ends.append(loss(v))
            assert abs(got.view(-1)[i].item() - (ends[0] - ends[1]) / (2 * step)) <= 1e-4


@pytest.mark.parametrize("points", [1, 5, 5000])
def test_infinities_and_nans_stay_in_their_group(points):
    x = torch.randn((3 * points, 64), generator=torch.Generator().manual_seed(1)).cuda()
    for bad in (math.inf, math.nan):
        v = x.clone()
        v[points, 20] = bad                   # image 1, group 1 of 4
        y = torch.empty_like(v)
        api.group_norm(v, y, points, 4)
        nan = torch.isnan(y).view(3, points, 4, 16)
        assert nan[1, :, 1].all() and nan.sum() == points * 16


def test_far_from_zero():
    """Values 1e4 away from zero with a spread of 1: fp32 keeps 2^-10 of it, the statistics of those values are right."""
    g = torch.Generator().manual_seed(2)
    for images, points, channels, groups in ((50, 1, 256, 4), (2, 3000, 16, 2)):
        x = (torch.randn((images * points, channels), generator=g) + 1e4).cuda()
        y, mean, rstd = torch.empty_like(x), torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
        api.group_norm(x, y, points, groups, mean=mean, rstd=rstd)
        want, wm, wr, _, _ = forward(x, points, groups, None, None, NONE)
        assert ((mean.double() - wm).abs() <= 2.0 ** -23 * 1e4).all()
        assert ((rstd.double() - wr).abs() <= 2e-5 * wr).all()
        assert ((y.double() - want).abs() <= 2e-3).all()      # mean's own rounding: 2^-24 of 1e4


def test_one_value_has_no_gradient():
    x, dy = torch.randn((9, 5), device="cuda"), torch.randn((9, 5), device="cuda")
    mean, rstd, y, dx = torch.empty((9, 5), device="cuda"), torch.empty((9, 5), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    api.group_norm(x, y, 1, 5, mean=mean, rstd=rstd)
    dgamma, dbeta = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    api.group_norm_backward(x, dy, 1, 5, mean, rstd, dx, dgamma, dbeta)
    assert (y == 0).all() and (dx == 0).all() and (dgamma == 0).all()


def test_no_images():
    x = torch.empty((0, 8), device="cuda")
    dgamma, dbeta, m = torch.ones(8, device="cuda"), torch.ones(8, device="cuda"), torch.empty((0, 2), device="cuda")
    api.group_norm(x, x, 3, 2)
    api.group_norm_backward(x, x, 3, 2, m, m, x, dgamma, dbeta, accumulate=True)
    assert (dgamma == 1).all() and (dbeta == 1).all()
    api.group_norm_backward(x, x, 3, 2, m, m, x, dgamma, dbeta)
    assert (dgamma == 0).all() and (dbeta == 0).all()


@pytest.mark.parametrize("images, channels, groups", [(1, 64, 8), (777, 64, 8), (9001, 256, 8), (1000, 24, 3), (1000, 8, 8), (513, 40, 5), (20000, 4, 1), (77, 1024, 2)])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_few_groups_of_one_point(images, channels, groups, kind):
    """Several rows share a wave where a row has few groups."""
    g = torch.Generator().manual_seed(images + channels)
    x, dy = data(g, images, 1, channels, kind, 0)
    gamma, beta = 1 + torch.randn(channels, generator=g).cuda() * 0.3, torch.randn(channels, generator=g).cuda()
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
    dgamma, dbeta = torch.empty(channels, device="cuda"), torch.empty(channels, device="cuda")
    api.group_norm(x, y, 1, groups, gamma, beta, EPS, NONE, mean, rstd)
    api.group_norm_backward(x, dy, 1, groups, mean, rstd, dx, dgamma, dbeta, gamma, beta)
    want, wm, wr, h, _ = forward(x, 1, groups, gamma, beta, NONE)
    assert ((y.double() - want).abs() <= HALF[kind] * want.abs() + 2.0 ** -20 * (1 + wr.max()) * (8 + h.abs())).all()
    assert ((mean.double() - wm).abs() <= 2.0 ** -21 * 10).all() and ((rstd.double() - wr).abs() <= 2.0 ** -19 * wr * (1 + wr)).all()
    h = forward(x, 1, groups, gamma, beta, NONE, moments=(mean, rstd))[3]
    for got, each in ((dgamma, dy.double() * h), (dbeta, dy.double())):
        assert ((got.double() - each.sum(0)).abs() <= 2.0 ** -19 * (each.abs() + 2.0 ** -20).sum(0)).all()
    gg = (dy.double() * gamma.double()).view(images, groups, -1)
    hh = h.view(images, groups, -1)
    want = (rstd.double()[:, :, None] * (gg - gg.mean(2, keepdim=True) - hh * (gg * hh).mean(2, keepdim=True))).view(x.shape)
    terms = (rstd.double()[:, :, None] * (gg.abs() + gg.abs().mean(2, keepdim=True) + hh.abs() * (gg * hh).abs().mean(2, keepdim=True))).view(x.shape)
    assert ((dx.double() - want).abs() <= HALF[kind] * want.abs() + 2.0 ** -20 * terms + 2.0 ** -130).all()
