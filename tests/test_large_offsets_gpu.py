"""Tables, maps and parameter lists whose offsets pass 32 bits: what lies beyond equals what a small call gives."""
import pytest
import torch

from paper_2203_10991_b200 import binding, optim

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_embedding_rows_beyond_four_gigabytes():
    vocab, cols = 600_000, 4096                              # 4.9 GB of bf16, 9.8 GB of fp32; element numbers beyond 2^31
    w = torch.empty(vocab, cols, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 0, 550_001, vocab - 1, 131_072], device="cuda")
    rows = torch.randn(5, cols, device="cuda").to(torch.bfloat16)
    rows[3] = rows[0]
    w[ids] = rows
    assert torch.equal(binding.mvue_embedding(ids, w, scale=2.0), (rows.float() * 2).to(torch.bfloat16))
    dw = binding.mvue_embedding_grad(ids, rows, vocab)
    want = rows.float()
    assert torch.equal(dw[vocab - 1], want[0] + want[3]) and torch.equal(dw[0], want[1]) and torch.equal(dw[550_001], want[2])
    # everything else is zero (whole numbers of rows: the sums of magnitudes by row)
    named = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    named[ids] = True
    assert float(dw.abs().amax(1)[~named].max()) == 0


@pytest.mark.parametrize("state_bits", [8, 32])
def test_adamw_elements_beyond_two_to_the_31(state_bits):
    n, tail = 2**31 + 5000, 6000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    start = (n - tail) // 256 * 256                          # a scale block's first element
    gen = torch.Generator().manual_seed(1)
    p[start:] = torch.randn(n - start, generator=gen).to(torch.bfloat16).cuda()
    g[start:] = torch.randn(n - start, generator=gen).to(torch.bfloat16).cuda()
    small_p, small_g = [p[start:].clone()], [g[start:].clone()]
    plan = optim.AdamWPlan.zeros([p], state_bits=state_bits)
    plan.step([g], step=1, lr=1e-2)
    assert int(torch.count_nonzero(p[:start])) == 0
    if state_bits == 32:
        small = optim.AdamWPlan.zeros(small_p, state_bits=32)
        small.step(small_g, step=1, lr=1e-2)
        assert torch.equal(p[start:], small_p[0]) and torch.equal(plan.exp_avgs[0][start:], small.exp_avgs[0])
    else:                                                    # other random bits there, the same params (rounded to nearest) and scales
        small = optim.AdamWPlan.zeros(small_p, state_bits=8)
        small.step(small_g, step=1, lr=1e-2)
        assert torch.equal(p[start:], small_p[0])
        assert torch.equal(plan.exp_avg_scales[0][start // 256:], small.exp_avg_scales[0])


@pytest.mark.parametrize("c", [64, 62])                      # samples in shared memory; element by element through memory
def test_group_norm_samples_beyond_four_gigabytes(c):
    n, s = 40_000, 1000                                      # 5 GB of bf16, 2.5 10^9 elements
    x = torch.zeros(n, s, c, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(2)
    last = torch.randn(2, s, c, generator=gen).to(torch.bfloat16).cuda()
    x[-2:] = last
    w, b = torch.randn(c, generator=gen).cuda(), torch.randn(c, generator=gen).cuda()
    y, mean, rstd = binding.mvue_group_norm_act(x, 2, w, b, act="silu", out=torch.empty_like(x))
    few = torch.nn.functional.silu(torch.nn.functional.group_norm(last.double().transpose(1, 2), 2, w.double(), b.double())).transpose(1, 2)
    # bf16 keeps eight digits: half a unit is 2^-9 of a power of two above the value
    assert float(((y[-2:].double() - few).abs() - 2.0 ** -8 * few.abs()).max()) < 1e-5
    assert torch.equal(y[0], y[n // 2])
    dx, dw, db = binding.mvue_group_norm_act_backward(x, x, mean, rstd, 2, w, b, act="silu", out=y)
    alone = binding.mvue_group_norm_act_backward(last, last, mean[-2:].contiguous(), rstd[-2:].contiguous(), 2, w, b, act="silu")
    assert float((dx[-2:].float() - alone[0].float()).abs().max()) <= 2.0 ** -6 * float(alone[0].float().abs().max())
    assert float(dx[0].float().abs().max()) == 0             # dy = 0 there
