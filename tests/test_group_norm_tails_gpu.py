"""SiLU far below zero in the group norm, forward and backward, by every route: gamma = 0 makes beta the activation's
argument exactly, so nothing but the activation's own evaluation is compared."""
import pytest
import torch

from paper_2203_10991_b200 import binding

gpu = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -149
FAR = [-41.0, -41.5, -41.6, -42.0, -45.0, -50.0, -60.0, -80.0, -87.0, -87.4, -88.0, -90.0, -100.0, -103.0, -104.0, -120.0, -200.0,
       -1e4, -1e10, -1e20, -3e38]
NEAR = [0.0, -0.5, 1.0, -3.0, 7.5, -20.0, 30.0, -35.0, 100.0, 1e10, 3e38]


def arguments(c):
    """c of them, two far ones and a near one in turn: far ones have near and far neighbours on either side."""
    far, near = 3 * (FAR + FAR), 3 * (NEAR + NEAR)
    return torch.tensor([near[i // 3] if i % 3 == 0 else far[2 * (i // 3) + i % 3 - 1] for i in range(c)], dtype=torch.float32)


def silu64(z):
    z = z.double()
    s = torch.sigmoid(z)
    # the exponential's argument is rounded (|z| U, and as much for the constant), exp and quotient to 2 units, a handful of
    # products; below 2^-126 the sigmoid has an absolute grid
    rel = (2 * z.abs() + 16) * U
    return z * s, z.abs() * s * rel + (1 + z.abs()) * 4 * TINY, s * (1 + z * (1 - s)), (1 + z.abs()) * (s * rel + 4 * TINY)


#                n, s, c, groups: sums in a warp (folded), values per channel, several blocks to a sample, through memory
ROUTES = [(2, 9, 64, 8), (2, 9, 56, 8), (1, 5000, 64, 4), (2, 9, 63, 7), (2, 9, 34, 2)]


@gpu
@pytest.mark.parametrize("n,s,c,groups", ROUTES)
def test_silu_far_below_zero(n, s, c, groups):
    z = arguments(c).cuda()
    x = torch.randn(n, s, c, generator=torch.Generator().manual_seed(1)).cuda()
    gamma = torch.zeros(c, device="cuda")
    y, mean, rstd = binding.mvue_group_norm_act(x, groups, gamma, z, act="silu")
    want, bound, slope, slope_bound = (t.cuda() for t in silu64(z.cpu()))
    assert bool(((y.double() - want).abs() <= bound).all())
    dy = torch.zeros_like(x)
    dy[0, s // 2] = 1.0
    dx, dgamma, dbeta = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, gamma, z, act="silu")
    assert bool(((dbeta.double() - slope).abs() <= slope_bound).all())
    assert float(dx.abs().max()) == 0


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n,s,c,groups", ROUTES)
def test_a_neighbour_that_is_not_finite(n, s, c, groups, bad):
    # two sigmoids may share a reciprocal: what is not finite on one side stays there
    z = arguments(c)
    z[1::4] = bad
    fine = torch.isfinite(z)
    x = torch.randn(n, s, c, generator=torch.Generator().manual_seed(1)).cuda()
    gamma = torch.zeros(c, device="cuda")
    y, mean, rstd = binding.mvue_group_norm_act(x, groups, gamma, z.cuda(), act="silu")
    want, bound, slope, slope_bound = silu64(torch.where(fine, z, torch.zeros_like(z)))
    off = (y.double().cpu() - want).abs()
    assert bool((off <= bound)[..., fine].all())
    got = y.cpu()[..., ~fine]
    assert bool((got == bad).all() if bad > 0 else torch.isnan(got).all())
    dy = torch.zeros_like(x)
    dy[0, s // 2] = 1.0
    _, _, dbeta = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, gamma, z.cuda(), act="silu")
    assert bool(((dbeta.double().cpu() - slope).abs() <= slope_bound)[fine].all())


@gpu
@pytest.mark.parametrize("n,s,c,groups", ROUTES)
def test_in_place(n, s, c, groups):
    z = arguments(c)
    z[3::16] = float("nan")
    fine = torch.isfinite(z)
    x = torch.randn(n, s, c, generator=torch.Generator().manual_seed(1)).cuda()
    gamma = torch.zeros(c, device="cuda")
    want, bound, _, _ = silu64(torch.where(fine, z, torch.zeros_like(z)))
    y = x.clone()
    _, mean, rstd = binding.mvue_group_norm_act(y, groups, gamma, z.cuda(), act="silu", out=y)
    assert bool(((y.double().cpu() - want).abs() <= bound)[..., fine].all()) and bool(torch.isnan(y[..., ~fine.cuda()]).all())
    # gamma of ordinary size and the far arguments in beta: dx in the place of dy as well as beside it
    gamma = torch.ones(c, device="cuda")
    z = arguments(c).cuda()
    dy = torch.randn(n, s, c, generator=torch.Generator().manual_seed(2)).cuda()
    apart = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, gamma, z, act="silu")
    inside = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, gamma, z, act="silu", out=dy)
    # the two ways differ by the sigmoids' last places, 8 units of the largest term at most
    assert float((apart[0] - inside[0]).abs().max()) <= 8 * 2.0 ** -23 * float(apart[0].abs().max())
    assert all(torch.equal(p, q) for p, q in zip(apart[1:], inside[1:]))
