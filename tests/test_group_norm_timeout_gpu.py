"""The bounded wait between the blocks of a group norm's cluster, made to run out without a fault: the blocks send one another
nothing, every wait gives up after some polls, the status word says so, the outputs are NaN and not something that looks like a
result, and the next call gives the same bits as before."""
import ctypes

import pytest
import torch

from paper_2203_10991_b200 import binding

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
#          n, s, c, groups, dtype: groups of whole pieces (folded) and others, one unit to a cluster and several
SHAPES = [(1, 5000, 64, 4, BF16), (200, 3136, 64, 8, BF16), (1, 1031, 56, 8, F32), (400, 1031, 56, 8, F32), (2, 4099, 16, 1, F32),
          (150, 6000, 24, 2, BF16)]


@gpu
@pytest.mark.parametrize("polls", [1, 200, 3000])
@pytest.mark.parametrize("n,s,c,groups,dtype", SHAPES)
def test_unanswered_waits_expire(n, s, c, groups, dtype, polls):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(n, s, c, generator=gen, device="cuda").to(dtype) for _ in range(2))
    y, mean, rstd = binding.mvue_group_norm_act(x, groups, eps=1.0)
    back = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups)
    torch.cuda.synchronize()

    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, bad_mean, bad_rstd = torch.zeros_like(x), torch.zeros_like(mean), torch.zeros_like(rstd)
    binding.mvue_selftest_group_norm_timeout(polls, x, groups, bad_mean, bad_rstd, out, status)
    torch.cuda.synchronize()                                 # the launch ends by itself
    assert int(status) == -10
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(bad_mean).all()) and bool(torch.isnan(bad_rstd).all())
    status.zero_()
    out.zero_()
    binding.mvue_selftest_group_norm_timeout(polls, x, groups, mean, rstd, out, status, dy=dy)
    torch.cuda.synchronize()
    assert int(status) == -10 and bool(torch.isnan(out).all())

    status.zero_()
    again = binding.mvue_group_norm_act(x, groups, eps=1.0, dev_status=status)
    back_again = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd, *back), (*again, *back_again)))


def test_refusals_before_any_launch():
    L, p = binding.lib(), ctypes.c_void_p

    def call(polls=10, x=4096, dy=None, dtype=1, n=1, s=5000, c=64, groups=4, mean=8192, out=1 << 14, ws=1 << 15, status=1 << 16):
        return L.mvue_selftest_group_norm_timeout(polls, p(x), p(dy), dtype, n, s, c, groups, p(mean), p(mean), p(out), p(ws), 1 << 30,
                                                  p(status), None)

    assert call(polls=0) == -3 and call(polls=(1 << 16) + 1) == -3 and call(n=0) == -3
    assert call(s=4) == -3                                   # one block holds the sample
    assert call(c=63, groups=7) == -3                        # through memory
    assert call(s=100000) == -3                              # no cluster holds it
    assert call(x=None) == -1 and call(mean=None) == -1 and call(out=None) == -1 and call(status=None) == -1
    assert call(x=4104) == -4 and call(dy=4104) == -4 and call(dtype=3) == -5 and call(ws=None, dy=4096) == -7
