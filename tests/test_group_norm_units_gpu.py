"""Group norm where clusters of two or more blocks take several samples in turn: the two places of the blocks' exchange alternate,
the next sample's copies replace the last one's, and the sums for the gradients of gamma and beta go on from sample to sample.
Every sample has its own mean and width, and all of them are compared with 64 bits."""
import ctypes

import pytest
import torch

from paper_2203_10991_b200 import binding
from tests.helpers import norm_ref as ref

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
#        n, s, c, groups, dtype, act: groups that are no whole pieces of eight channels, and such that are; the last slab of a
#        sample narrower than the others (120 of 48s, 80 of 32s) or not
SHAPES = [(400, 1031, 56, 8, F32, "silu"), (200, 2500, 120, 10, BF16, "gelu"), (250, 2100, 36 * 2, 6, BF16, "relu"),
          (700, 1000, 64, 2, BF16, "silu"), (300, 2100, 80, 10, BF16, "silu"), (130, 3136, 96, 6, F32, "relu")]


@pytest.mark.parametrize("n,s,c,groups,dtype,act", SHAPES)
def test_the_shapes_are_of_that_kind(n, s, c, groups, dtype, act):
    # the self-test of the blocks' exchange takes only shapes that have one: here it is refused for want of a workspace
    # (before anything is launched), with four positions for its shape
    p = ctypes.c_void_p

    def call(s):
        return binding.lib().mvue_selftest_group_norm_timeout(1, p(4096), p(4096), int(dtype is BF16), n, s, c, groups, p(4096), p(4096),
                                                              p(4096), None, 0, p(4096), None)

    assert call(s) == -7 and call(4) == -3


@gpu
@pytest.mark.parametrize("n,s,c,groups,dtype,act", SHAPES)
def test_many_samples_to_a_cluster(n, s, c, groups, dtype, act):
    gen = torch.Generator(device="cuda").manual_seed(n + c)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    x = ((0.3 + torch.rand(n, 1, c, generator=gen, device="cuda")) * normal(n, s, c) + normal(n, 1, c)).to(dtype)
    dy = normal(n, s, c).to(dtype)
    w, b = 1 + 0.3 * normal(c), 0.3 * normal(c)
    got = binding.mvue_group_norm_act(x, groups, w, b, act=act)
    want, bound = ref.forward(x, groups, w, b, 1e-5, act)
    for g, t, e in zip(got, want, bound):
        assert ref.inside(g, t, e)
    del want, bound
    _, mean, rstd = got
    back = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, w, b, act=act)
    want, bound = ref.backward(dy, x, mean, rstd, groups, w, b, act)
    for g, t, e in zip(back, want, bound):
        assert ref.inside(g, t, e)
    del want, bound
    again = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, w, b, act=act)
    assert all(torch.equal(p, q) for p, q in zip(back, again))
