"""AdamWPlan as an object: seeds, refused gradients."""
import pytest
import torch

from paper_2203_10991_b200 import optim

gpu = pytest.mark.gpu
BF16 = torch.bfloat16


@gpu
def test_slow_average_moves_without_a_seed_of_ones_own():
    # sqrt(v) = 4 q, gradients of size q: v falls to q^2 at the rate beta2 = 0.999.  With the same random numbers each step
    # every element has a fixed threshold, and the average stays where it is.
    n, q = 4096, 1e-3
    plan = optim.AdamWPlan.zeros([torch.zeros(n, device="cuda")], state_bits=8)
    plan.exp_avg_sqs[0].view(torch.uint8).fill_(0x60)                       # 2^(12-7) = 32 in units of the scale
    plan.exp_avg_sq_scales[0].fill_(4 * q / 32)
    g = [torch.full((n,), q, device="cuda")]
    g[0][::256] = 40 * q                                                    # one large value a block keeps the scale up
    for t in range(1, 1001):
        plan.step(g, step=t, lr=0.0, weight_decay=0.0)
    root = (plan.exp_avg_sqs[0].double() * plan.exp_avg_sq_scales[0].double().repeat_interleave(256)).reshape(-1, 256)[:, 1:]
    exact = (16 * 0.999 ** 1000 + (1 - 0.999 ** 1000)) ** 0.5 * q
    # v follows the average of the squared codes, which the rounding's spread (a few per cent of sqrt(v) a step) raises a little
    assert abs(float(root.mean()) / exact - 1) < 0.15


@gpu
def test_bf16_params_drift_in_the_mean_without_a_seed_of_ones_own():
    # updates of 2^-16 on params of 1 (half a unit there is 2^-9): 256 steps move the mean by 2^-8 (32-bit states, v' = m'^2 = 1)
    n, steps, lr = 65536, 256, 2.0 ** -16
    p = [torch.ones(n, device="cuda", dtype=BF16)]
    plan = optim.AdamWPlan.zeros(p)
    g = [torch.ones(n, device="cuda")]
    for t in range(1, steps + 1):
        plan.step(g, step=t, lr=lr, weight_decay=0.0, stochastic_rounding=True)
    # each element falls by 2^-8 with probability 2^-8 a step: the mean's deviation is 2^-8 sqrt(256 / 256 / 65536) = 2^-16
    assert abs(float((1 - p[0].double()).mean()) - steps * lr) < 8 * 2.0 ** -16
    # and is not the same for all: with fixed thresholds 1 in 256 would fall at every step
    assert float((1 - p[0].double()).max()) < 0.1


@gpu
def test_refused_gradients_leave_the_plan_as_it_is():
    def plan_of():
        p = [torch.full((300,), 0.5, device="cuda"), torch.full((8, 64), 0.5, device="cuda")]
        return p, optim.AdamWPlan.zeros(p)

    first = [torch.full((300,), 0.1, device="cuda"), torch.full((8, 64), 0.2, device="cuda")]
    other = torch.full((300,), -7.0, device="cuda")
    p, plan = plan_of()
    q, want = plan_of()
    plan.step(first, step=1, lr=1e-2)
    want.step(first, step=1, lr=1e-2)
    for bad in ([other, torch.zeros(8, 128, device="cuda")[:, ::2]], [other, torch.zeros(8, 64)], [other, torch.zeros(8, 65, device="cuda")], [other]):
        with pytest.raises(ValueError):
            plan.step(bad, step=2, lr=1e-2)
    with pytest.raises(TypeError):
        plan.step([other, torch.zeros(8, 64, device="cuda", dtype=torch.float16)], step=2, lr=1e-2)
    plan.step(step=2, lr=1e-2)
    want.step(first, step=2, lr=1e-2)
    assert all(torch.equal(a, b) for a, b in zip(p, q))


@gpu
def test_exchanged_memory_is_refused_and_never_written_after_it_was_freed():
    p = [torch.full((4096,), 0.5, device="cuda"), torch.full((4096,), 0.5, device="cuda")]
    g = [torch.full((4096,), 0.1, device="cuda") for _ in p]
    plan = optim.AdamWPlan.zeros(p, grads=g)
    plan.step(step=1, lr=1e-2)
    after = p[1].clone()
    p[1].data = p[1].data.clone()
    with pytest.raises(ValueError):
        plan.step(g, step=2, lr=1e-2)
    # the old memory is the plan's: nothing else is given it, and the step without gradients stays inside
    others = [torch.full((4096,), 7.0, device="cuda") for _ in range(64)]
    plan.step(step=2, lr=1e-2)
    assert all(bool((t == 7).all()) for t in others) and torch.equal(p[1], after)
    again = optim.AdamWPlan(p, plan.exp_avgs, plan.exp_avg_sqs)
    again.step(g, step=3, lr=1e-2)
    assert not torch.equal(p[1], after)
    g[0].data = g[0].data.clone()
    with pytest.raises(ValueError):
        again.step(step=4, lr=1e-2)
    again.step(g, step=4, lr=1e-2)
