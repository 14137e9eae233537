"""Group norm of maps whose values are beyond the root of the largest binary32 number: squares of the values overflow, squares
of their distances from the mean do not."""
import pytest
import torch

from paper_2203_10991_b200 import binding

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent", [10, 63, 65, 90, 100])
@pytest.mark.parametrize("n,s,c,groups", [(2, 64, 4, 1), (1, 4096, 2, 1), (3, 32, 12, 3), (2, 64, 16, 2), (2, 64, 64, 8), (1, 8192, 64, 1)])
def test_constant_groups(n, s, c, groups, dtype, exponent):
    # powers of two in numbers that are powers of two: every sum and mean is exact, the variance is zero, y is beta
    x = torch.full((n, s, c), 2.0 ** exponent, device="cuda", dtype=dtype)
    x[..., c // 2:] *= -1 if groups == 1 and exponent < 60 else 1
    beta = torch.arange(c, device="cuda", dtype=torch.float32) / 8
    y, mean, rstd = binding.mvue_group_norm_act(x, groups, None, beta, act="none", eps=1.0)
    if groups == 1 and exponent < 60:                       # two values of either sign: the mean 0, the variance 2^(2 exponent)
        want = x.double() / (4.0 ** exponent + 1.0) ** 0.5 + beta
        assert float((y.double() - want).abs().max()) <= float(want.abs().max()) * 2.0 ** (-7 if dtype == torch.bfloat16 else -21)
        return
    assert torch.equal(mean, torch.full_like(mean, 2.0 ** exponent)) and torch.equal(rstd, torch.ones_like(rstd))
    assert torch.equal(y, beta.to(dtype).expand_as(y))
