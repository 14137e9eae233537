"""Which layouts AdamWPlan takes for one another: dimensions of size zero and one, dimension orders, gaps."""
import pytest
import torch

from paper_2203_10991_b200 import optim


@pytest.mark.parametrize("shape", [(0,), (0, 5), (5, 0), (3, 0, 2), (2, 3, 0)])
def test_empty_tensors_are_dense(shape):
    t = torch.empty(shape)
    assert optim._dense(t) and optim._dense(t.transpose(0, -1)) and optim._same_layout(t, torch.empty(shape))


def test_dense_in_any_order_and_not_with_gaps():
    t = torch.empty(4, 3, 5, 2)
    for u in (t, t.permute(2, 0, 3, 1), t.to(memory_format=torch.channels_last), t[:, :1].squeeze(1)[:1], torch.empty(1, 7).t(), torch.empty(())):
        assert optim._dense(u)
    for u in (t[:, :2], t[..., ::2], torch.empty(4, 1).expand(4, 3), torch.empty(7).as_strided((2, 2), (1, 1))):
        assert not optim._dense(u)


def test_strides_of_dimensions_of_size_one_do_not_count():
    # the same memory order, other strides where there is nothing to step over
    a = torch.empty_strided((8, 1, 3, 2), (6, 1, 1, 3))
    b = torch.empty_strided((8, 1, 3, 2), (6, 6, 1, 3))
    assert not a.is_contiguous() and optim._dense(a) and optim._dense(b)
    assert optim._same_layout(a, b) and optim._same_layout(b, a)
    c = torch.empty_strided((8, 1, 3, 2), (6, 6, 2, 1))
    assert c.is_contiguous() and not optim._same_layout(a, c)
    assert not optim._same_layout(a, torch.empty_strided((8, 1, 2, 3), (6, 6, 1, 2)))
    assert optim._same_layout(torch.empty(6), torch.empty(2, 3))


@pytest.mark.gpu
def test_a_step_with_empty_and_thin_params():
    p = [torch.zeros(5, 0, device="cuda"), torch.zeros(3, 0, 2, device="cuda"), torch.empty_strided((8, 1, 3, 2), (6, 1, 1, 3), device="cuda").zero_()]
    g = [torch.zeros_like(p[0]), torch.zeros_like(p[1]), torch.empty_strided((8, 1, 3, 2), (6, 6, 1, 3), device="cuda").copy_(
        torch.arange(48, device="cuda").reshape(8, 1, 3, 2) - 20.5)]
    for state_bits in (32, 8):
        optim.AdamWPlan.zeros(p, state_bits=state_bits).step(g, step=1, lr=1e-2, weight_decay=0.0)
    # the first step of fresh states moves every element by lr against its gradient's sign (m / sqrt(v) = g / |g|)
    assert float((p[2] + 2e-2 * g[2].sign()).abs().max()) < 1e-6
