"""8-bit AdamW states against the definition, bit for bit over tensors of a layer's size and several steps: a code that
falls on the wrong side of its threshold once in millions, and the scales that follow from it, show up here."""
import numpy as np
import pytest
import torch

from paper_2203_10991_b200 import optim
from tests.helpers import adamw_ref, adamw_torch

gpu = pytest.mark.gpu


def u8(t):
    return t.view(torch.uint8)


def test_the_two_references_agree():
    # the torch form that runs on the device against the numpy form of the small tests
    gen = torch.Generator().manual_seed(1)
    g = torch.randn(1024, generator=gen) * 1e-3
    g[256:512] = 0.0
    s = adamw_torch.States(1024, "cpu")
    m0, v0 = np.zeros(1024, np.float32), np.zeros(1024, np.float32)
    values = adamw_ref.e4m3_values().astype(np.float32)
    for seed in (3, 0xFEDCBA9876543210, 5):
        r = adamw_ref.random16(0, 128, seed)
        assert np.array_equal(adamw_torch.random16(128, seed, "cpu").numpy(), r.astype(np.int64))
        s.step(g, 0.9, 0.999, seed)
        m1, v1 = adamw_ref.moments32(g.numpy(), m0, v0 * v0, 0.9, 0.999)
        swapped = (r & 255) << 8 | r >> 8
        for x, one, codes, scales in ((m1, False, s.m, s.ms), (np.sqrt(v1), True, s.v, s.vs)):
            want, scale = adamw_ref.quantise(x, swapped, one)
            assert np.array_equal(codes.numpy(), want) and np.array_equal(scales.numpy(), scale)
        m0 = values[s.m.numpy()] * np.repeat(s.ms.numpy(), 256)
        v0 = values[s.v.numpy()] * np.repeat(s.vs.numpy(), 256)


@gpu
@pytest.mark.parametrize("kind", ["dense", "zero blocks", "wide"])
def test_codes_and_scales_of_a_large_tensor_over_eight_steps(kind):
    # 2^25 elements: a root that is one unit off where it should be rounded moves about ten codes a step
    n = 1 << 25
    gen = torch.Generator(device="cuda").manual_seed(7)
    p = [torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
    plan = optim.AdamWPlan.zeros(p, state_bits=8)
    want = adamw_torch.States(n, "cuda")
    for step in range(1, 9):
        g = torch.randn(n, generator=gen, device="cuda").mul_(1e-3)
        if kind == "wide":                                  # magnitudes over many binades: codes below 2^-6 are common
            g *= torch.exp(4 * torch.randn(n, generator=gen, device="cuda"))
        if kind == "zero blocks":                           # rows of a table that no batch has named, single zeros in the others
            g.view(-1, 2, 256)[:, 0] = 0.0
            g[300::512] = 0.0
        plan.step([g], step=step, lr=1e-3, seed=1000 + step)
        want.step(g, 0.9, 0.999, 1000 + step)
        assert int((u8(plan.exp_avgs[0]) != want.m).sum()) == 0
        assert int((u8(plan.exp_avg_sqs[0]) != want.v).sum()) == 0
        assert torch.equal(plan.exp_avg_scales[0], want.ms) and torch.equal(plan.exp_avg_sq_scales[0], want.vs)
