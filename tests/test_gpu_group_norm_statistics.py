"""GPU tests of group norm's statistics where 32-bit sums do not do: groups of
one value, values far from zero beside their spread, and values whose squares
leave the range of fp32; in each of its forms."""
import math

import pytest
import torch

from paper_2407_18352_amd import api
from test_gpu_group_norm import BF16, EPS, F32, HALF, NONE, RELU, forward

pytestmark = pytest.mark.gpu

#             images, points, channels, groups: one point (a few lanes a group)
IN_REGISTERS = [(5, 1, 7, 1), (33, 1, 45, 1), (700, 1, 96, 8), (9, 1, 512, 1), (3, 1, 2048, 4),
                # groups in a block's registers
                (4, 221, 9, 1), (37, 221, 45, 9), (3, 45, 16, 2), (2, 4096, 1, 1), (5, 64, 256, 32)]
# parts of an image; wide groups of one point
IN_PARTS = [(1, 20000, 8, 2), (2, 5000, 3, 1), (3, 1, 1989, 1), (1, 70001, 130, 10), (2, 4097, 3, 3), (6, 300, 1024, 1)]


def normed(x, points, groups, beta=None, act=NONE):
    images = x.shape[0] // points
    y, mean, rstd = torch.empty_like(x), torch.empty((images, groups), device="cuda"), torch.empty((images, groups), device="cuda")
    api.group_norm(x, y, points, groups, None, beta, EPS, act, mean, rstd)
    return y, mean, rstd


def constants(case, level, kind, g):
    """A value near `level` for every image and group, of all bits that its type has."""
    images, points, channels, groups = case
    c = (level * (1 + torch.rand((images, 1, groups, 1), generator=g))).to(kind)
    return c, c.expand(images, points, groups, channels // groups).reshape(images * points, channels).cuda()


def one_value(case, kind):
    g = torch.Generator().manual_seed(sum(case))
    images, points, channels, groups = case
    beta = torch.randn(channels, generator=g).cuda()
    for level in (1.0, 1e3, 1e5, 1e6):
        c, x = constants(case, level, kind, g)
        for act, f in ((NONE, lambda b: b), (RELU, torch.relu)):
            y, mean, rstd = normed(x, points, groups, beta, act)
            assert torch.equal(mean.cpu(), c.float().view(images, groups))
            # a rounding to fp32 and the reciprocal root's ulp
            assert ((rstd.double() * math.sqrt(EPS) - 1).abs() <= 2.0 ** -22).all()
            assert torch.equal(y, f(beta).to(kind).expand_as(y))


def compared(x, points, groups, kind):
    """Sums in 64 bits; mean and variance rounded to fp32, the reciprocal root 2^-23 off.  In parts a run's mean is rounded about one of
    its values, within six standard deviations, and its deviation: 2^-24 of each, less than 2^-21 of rstd with the rest."""
    y, mean, rstd = normed(x, points, groups)
    want, wm, wr, _, _ = forward(x, points, groups, None, None, NONE)
    mean_off = 2.0 ** -24 * wm.abs() + 2.0 ** -21 / wr
    assert ((mean.double() - wm).abs() <= mean_off).all()
    assert ((rstd.double() - wr).abs() <= 2.0 ** -21 * wr).all()
    off = (mean_off * wr)[:, None, :, None].expand(-1, points, -1, x.shape[1] // groups).reshape(x.shape)
    # (x - mean) and its product rounded, rstd as above
    assert ((y.double() - want).abs() <= off + 2.0 ** -20 * want.abs() + HALF[kind] * want.abs() + 2.0 ** -130).all()


def far(case, kind):
    images, points, channels, groups = case
    g = torch.Generator().manual_seed(sum(case) + 1)
    for level, spread in ((1e3, 1.0), (1e5, 0.1), (1e5, 0.02), (1e6, 1.0)):
        _, x = constants(case, level, F32, g)
        if kind == BF16:
            spread = level / 64               # a few of its steps
        compared((x + spread * torch.randn(x.shape, generator=g).cuda()).to(kind), points, groups, kind)
    # a border of zeros around values far from them
    x = (1e5 + 0.1 * torch.randn((images * points, channels), generator=g)).to(kind).cuda()
    x.view(images, points, channels)[:, 0] = 0
    x.view(images, points, channels)[:, :, 0] = 0
    compared(x, points, groups, kind)


def large(case, kind):
    images, points, channels, groups = case
    g = torch.Generator().manual_seed(sum(case) + 2)
    for e in (60, 64, 80, 120):
        x = ((torch.randn((images * points, channels), generator=g) + 1) * 2.0 ** e).to(kind).cuda()
        compared(x, points, groups, kind)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", IN_REGISTERS)
@pytest.mark.parametrize("check", [one_value, far, large])
def test_in_registers(check, case, kind):
    check(case, kind)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("case", IN_PARTS)
@pytest.mark.parametrize("check", [one_value, far, large])
def test_in_parts(check, case, kind):
    check(case, kind)
