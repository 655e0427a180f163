"""SiLU and its slope value by value, far beyond what norms of ordinary nets give them.

A weight of 0 makes z the bias, exactly, so a sample's results are act(bias) and, where dy is 1 in one pixel and 0 elsewhere, dbias is
act'(bias).  Bounds: with e = 2^-24, the exponential's argument is off by two roundings of it, so exp(-z) by (|z| + 2) 2 e of itself (the
instruction's own error included), g = 1 / (1 + exp(-z)) by that times 1 - g and four roundings and a reciprocal, 8 e; so is h = 1 - g, with g:
    d_g = (1 - g) (|z| + 2) 2 e + 8 e,  d_h = g (|z| + 2) 2 e + 8 e        of g and h
    silu = z g: |z g| (d_g + 2 e);     slope = g (1 + z h): g (1 + |z| h) (d_g + 4 e) + g |z| h d_h
and numbers below 2^-126 count as 0: |z| 2^-125 more.
"""
import pytest
import torch

from paper_2007_13221_b200 import layers

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
E = 2.0 ** -24
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: E}


def results(z, dtype, pixels, groups):
    """silu and its slope at each of z, one a channel; the groups' statistics do not matter."""
    c = z.numel()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    x = torch.randn((1, 1, pixels, c), generator=gen, device="cuda").to(dtype)
    op = layers.GroupNorm(1, 1, c, groups, "silu", dtype=dtype)
    weight, dy = torch.zeros((1, c), device="cuda"), torch.zeros_like(x)
    dy[0, 0, pixels // 2] = 1
    y, stats = op.apply(x, weight, z[None])
    return y[0, 0, 0].double(), op.grad(x, dy, stats, weight, z[None])[2][0].double()


def check(z, dtype, pixels, groups, of=slice(None)):
    """The results at the channels `of` against the bounds; all results."""
    every = results(z, dtype, pixels, groups)
    y, slope, z = every[0][of], every[1][of], z[of]
    v = z.double()
    g, h = torch.sigmoid(v), torch.sigmoid(-v)
    d_g, d_h = h * (v.abs() + 2) * 2 * E + 8 * E, g * (v.abs() + 2) * 2 * E + 8 * E
    want = v * g
    flush = v.abs() * 2.0 ** -125
    rounded = U[dtype] * want.abs() + (2.0 ** -25 if dtype is HF else 2.0 ** -133)
    off = (y - want).abs() - (want.abs() * (d_g + 2 * E) + flush + 1.01 * rounded)
    assert bool((off <= 0).all()), (float(z[off.argmax()]), float(y[off.argmax()]), float(want[off.argmax()]))
    want = g * (1 + v * h)
    off = (slope - want).abs() - (g * (1 + v.abs() * h) * (d_g + 4 * E) + g * v.abs() * h * d_h + flush + 2.0 ** -126)
    assert bool((off <= 0).all()), (float(z[off.argmax()]), float(slope[off.argmax()]), float(want[off.argmax()]))
    return every


# one walk with vectors of 16 bytes, of fewer, and several walks
PLANS = [(F32, 4, 64), (BF, 4, 64), (HF, 9, 64), (F32, 5, 1), (BF, 6, 1), (F32, 2000, 1), (BF, 1500, 1)]


@pytest.mark.parametrize("plan", PLANS, ids=str)
def test_slopes_of_large_values(plan):
    """From where 1 - g begins to lose digits up to where exp(-z) is no number any more: g (1 + z (1 - g)) is 1 + z exp(-z) there."""
    dtype, pixels, groups = plan
    top = 1000.0 if dtype is not HF else 6e4
    z = torch.cat([torch.linspace(-20, 110, 2048), torch.logspace(0, 3, 2048).clamp(max=top)])
    z = z[torch.randperm(4096, generator=torch.Generator().manual_seed(1))]
    check(z.cuda(), dtype, pixels, groups)


@pytest.mark.parametrize("plan", PLANS, ids=str)
def test_values_far_below_zero(plan):
    """z / (1 + exp(-z)) goes to 0 there, and so does its slope."""
    dtype, pixels, groups = plan
    z = -torch.cat([torch.linspace(30, 130, 2048), torch.logspace(1, 30, 2048)])
    z = z[torch.randperm(4096, generator=torch.Generator().manual_seed(1))]
    z[torch.arange(0, 4096, 5)] = torch.linspace(-10, 10, 820)      # and beside ordinary ones
    check(z.cuda(), dtype, pixels, groups)


@pytest.mark.parametrize("plan", PLANS, ids=str)
def test_values_that_are_no_numbers_spoil_no_neighbour(plan):
    dtype, pixels, groups = plan
    z = torch.linspace(-60, 60, 4096)
    bad = torch.arange(0, 4096, 5)
    z[bad] = torch.tensor([float("nan"), float("inf"), -float("inf")]).repeat(274)[:820]
    z = z.cuda()
    fine = torch.ones(4096, dtype=torch.bool)
    fine[bad] = False
    y, slope = check(z, dtype, pixels, groups, fine.cuda())
    assert bool(y[z == float("inf")].isposinf().all()) and bool(y[z.isnan() | z.isneginf()].isnan().all()) and bool(slope[z.isnan()].isnan().all())
