"""AdamW where the second moment is below the smallest normal number (2^-126): gradients of 1e-20 to 1e-18 on fresh states.
The root of such a v' is an ordinary number, and with eps = 0 it is all that the step is divided by."""
import numpy as np
import pytest
import torch

from paper_2203_10991_b200 import optim
from tests.helpers import adamw_ref as ref, adamw_torch

gpu = pytest.mark.gpu
U = 2.0 ** -24
LR = 1e-3


def gradients(n):
    # v' = g^2 / 1000 from 10^-44 (seven times the smallest subnormal) to 10^-39 (a tenth of the smallest normal)
    gen = torch.Generator().manual_seed(2)
    size = 10 ** (-20.5 + 2.5 * torch.rand(n, generator=gen, dtype=torch.float64))
    return (size * torch.randn(n, generator=gen).sign()).float()


def check(param, m, v, eps, step):
    """The param (zero before) against 64 bits from the moments m, v in binary32: the root and the quotient are within
    2 units of their last places (8 U), the constants and products of the update take six more roundings."""
    want = -LR / (1 - 0.9 ** step) * m / (np.sqrt(v) / np.sqrt(1 - 0.999 ** step) + eps)
    assert np.all(np.abs(param - want) <= 16 * U * np.abs(want))


@gpu
@pytest.mark.parametrize("eps", [0.0, 1e-20, 1e-8])
@pytest.mark.parametrize("state_bits", [32, 8])
def test_moments_below_the_smallest_normal(state_bits, eps):
    n = 8192
    g = gradients(n)
    p = [torch.zeros(n, device="cuda")]
    plan = optim.AdamWPlan.zeros(p, state_bits=state_bits)
    plan.step([g.cuda()], step=1, lr=LR, eps=eps, weight_decay=0.0, seed=11)
    zero = np.zeros(n, np.float32)
    m1, v1 = ref.moments32(g.numpy(), zero, zero, 0.9, 0.999)
    assert np.all(v1 > 0) and np.all(v1 < 2.0 ** -126)
    check(p[0].double().cpu().numpy(), m1.astype(np.float64), v1.astype(np.float64), eps, 1)
    if state_bits == 32:
        assert np.array_equal(plan.exp_avgs[0].cpu().numpy(), m1) and np.array_equal(plan.exp_avg_sqs[0].cpu().numpy(), v1)
        return
    want = adamw_torch.States(n, "cpu")
    want.step(g, 0.9, 0.999, 11)
    assert torch.equal(plan.exp_avg_scales[0].cpu(), want.ms) and torch.equal(plan.exp_avg_sq_scales[0].cpu(), want.vs)
    assert torch.equal(plan.exp_avgs[0].view(torch.uint8).cpu(), want.m)
    assert torch.equal(plan.exp_avg_sqs[0].view(torch.uint8).cpu(), want.v)


@gpu
@pytest.mark.parametrize("state_bits", [32, 8])
def test_ordinary_and_small_gradients_side_by_side(state_bits):
    # one element in seven is small; the others' steps are what they are without it
    n = 4096
    small = gradients(n)
    gen = torch.Generator().manual_seed(4)
    g = 1e-3 * torch.randn(n, generator=gen)
    g[::7] = small[::7]
    p = [torch.zeros(n, device="cuda")]
    optim.AdamWPlan.zeros(p, state_bits=state_bits).step([g.cuda()], step=1, lr=LR, eps=0.0, weight_decay=0.0, seed=12)
    zero = np.zeros(n, np.float32)
    m1, v1 = ref.moments32(g.numpy(), zero, zero, 0.9, 0.999)
    check(p[0].double().cpu().numpy(), m1.astype(np.float64), v1.astype(np.float64), 0.0, 1)
