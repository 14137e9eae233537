"""Group norm over groups of one element (one position, one channel to a group): the output does not depend on the input, so dx
is zero, not what two roundings of the same product leave of it times rstd (316 at the default eps)."""
import pytest
import torch

from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype,affine", [(torch.float32, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("n,c", [(7, 8), (5, 7), (3, 10), (2, 64), (400, 1000), (1, 4096), (33, 1)])
def test_no_gradient_through_groups_of_one(n, c, dtype, affine, act):
    gen = torch.Generator().manual_seed(n + c)
    x, dy = (torch.randn(n, 1, c, generator=gen).to(dtype).cuda() for _ in range(2))
    w, b = ((1 + torch.randn(c, generator=gen)).to(affine).cuda() for _ in range(2))
    y, mean, rstd = binding.mvue_group_norm_act(x, c, w, b, act=act)
    assert torch.equal(mean, x.reshape(n, c).float())
    dx, dw, db = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, c, w, b, act=act)
    assert float(dx.float().abs().max()) == 0 and float(dw.abs().max()) == 0
    # what is not a number stays visible
    dy[0, 0, 0] = float("nan")
    dx, _, _ = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, c, w, b, act="none")
    assert bool(torch.isnan(dx[0, 0, 0])) and float(dx.float().reshape(-1)[1:].abs().nan_to_num(9.0).max() if dx.numel() > 1 else 0.0) == 0
