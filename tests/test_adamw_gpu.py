"""The AdamW step over many tensors: both moments bit for bit against numpy binary32, the params against 64 bits, the
8-bit states' codes bit for bit, odd sizes and alignments, refusals, streams and graphs."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2203_10991_b200 import binding, optim
from tests.helpers import adamw_ref as ref

U = 2.0 ** -24                     # half a unit in the last place, relative
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
F32, BF16 = torch.float32, torch.bfloat16

gpu = pytest.mark.gpu


def bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).cpu().numpy().reshape(-1)


def f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def tensors(sizes, dtype, std, seed, offset=0):
    """Views that start `offset` elements behind an allocation's start."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for n in sizes:
        buf = torch.empty(n + offset, dtype=dtype, device="cuda")
        buf[offset:] = (std * torch.randn(n, generator=gen)).to(dtype).cuda()
        out.append(buf[offset:])
    return out


def check_param(got, want, moved, stored="f32"):
    """got against the 64-bit want.  Roundings on the way (each at most U of its own result): decay * param and its
    constant (2), the constant and product and quotient of the update with its approximate root and reciprocal
    (2 + 2 ulp = 4 + 4 U, six more roundings: 14 U of the update), the difference (1).  Rounding is monotone, so what is
    stored lies between the ends of that interval rounded the same way ("random": down and up)."""
    bound = (4 * U * np.abs(want) + 16 * U * moved) * (1 + 1e-6) + 1e-45
    lo, hi = want - bound, want + bound
    if stored != "f32":
        lo, hi = (torch.from_numpy(x).float() for x in (lo, hi))
        if stored == "bf16":
            lo, hi = lo.to(BF16), hi.to(BF16)
        else:
            cut = [(x.view(torch.int32) & -65536) for x in (lo, hi)]                       # towards zero
            away = [(x.view(torch.int32) + 0xFFFF) & -65536 for x in (lo, hi)]
            lo = torch.where(lo >= 0, cut[0], away[0]).view(F32)
            hi = torch.where(hi >= 0, away[1], cut[1]).view(F32)
        lo, hi = lo.double().numpy(), hi.double().numpy()
    assert np.all((lo <= got) & (got <= hi)), float(np.maximum(lo - got, got - hi).max())


@gpu
@pytest.mark.parametrize("offset", [0, 1, 8])
@pytest.mark.parametrize("sizes", [[1], [7, 8, 9], [255, 256, 257, 2047, 2048, 2049, 4099], [13] * 40 + [3000], [70001]])
@pytest.mark.parametrize("form", ["f32", "bf16", "master"])
@pytest.mark.parametrize("grad_dtype", [F32, BF16])
def test_32bit_states(sizes, form, grad_dtype, offset):
    p = tensors(sizes, F32 if form == "f32" else BF16, 0.05, 1, offset)
    w = tensors(sizes, F32, 0.05, 2, offset) if form == "master" else None
    g = tensors(sizes, grad_dtype, 1e-3, 3, offset)
    m, v = tensors(sizes, F32, 1e-3, 4, offset), [x.square_() for x in tensors(sizes, F32, 1e-3, 5, offset)]
    before = [[x.clone() for x in q] for q in (w or p, g, m, v)]
    optim.AdamWPlan(p, m, v, masters=w).step(g, step=7, **HYPER, grad_scale=0.5)
    torch.cuda.synchronize()
    for i in range(len(sizes)):
        p0, g0, m0, v0 = (q[i].float().cpu().numpy() for q in before)
        m1, v1 = ref.moments32(g0, m0, v0, 0.9, 0.999, 0.5)
        assert np.array_equal(m[i].cpu().numpy(), m1) and np.array_equal(v[i].cpu().numpy(), v1)
        want, m64, v64 = ref.step64(p0, g0, m0, v0, step=7, **HYPER, grad_scale=0.5)
        # two products, their constants' roundings and a sum
        assert np.all(np.abs(m1 - m64) <= 4 * U * (np.abs(0.9 * m0) + np.abs(0.05 * g0)) + 1e-45)
        assert np.all(np.abs(v1 - v64) <= 6 * U * v64 + 1e-45)
        moved = np.abs(want - p0.astype(np.float64) * (1 - HYPER["lr"] * HYPER["weight_decay"]))
        if form == "master":
            check_param(f64(w[i]), want, moved)
            assert torch.equal(p[i], w[i].to(BF16))
        else:
            check_param(f64(p[i]), want, moved, form)
        assert np.array_equal(bits(g[i]), bits(before[1][i]))


@gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("sizes", [[1], [9, 256, 257], [2049, 4, 700]])
@pytest.mark.parametrize("form", ["f32", "bf16", "bf16_random", "master"])
def test_8bit_states(sizes, form, offset):
    p = tensors(sizes, F32 if form == "f32" else BF16, 0.05, 1, offset)
    w = tensors(sizes, F32, 0.05, 2, offset) if form == "master" else None
    g = tensors(sizes, F32, 1e-3, 3, offset)
    plan = optim.AdamWPlan.zeros(p, state_bits=8)
    if offset:
        codes = [[torch.zeros(n + offset, dtype=torch.uint8, device="cuda")[offset:].view(torch.float8_e4m3fn) for n in sizes] for _ in range(2)]
        plan = optim.AdamWPlan(p, *codes, masters=w, exp_avg_scales=plan.exp_avg_scales, exp_avg_sq_scales=plan.exp_avg_sq_scales)
    elif w is not None:
        plan = optim.AdamWPlan(p, plan.exp_avgs, plan.exp_avg_sqs, masters=w, exp_avg_scales=plan.exp_avg_scales,
                               exp_avg_sq_scales=plan.exp_avg_sq_scales)
    values = ref.e4m3_values().astype(np.float32)
    state = [[np.zeros(n, np.float32) for n in sizes] for _ in range(2)]           # m, sqrt(v) as the codes say
    for step, seed in ((1, 5), (2, 0x123456789ABCDEF0)):
        p0 = [x.float().cpu().numpy() for x in (w or p)]
        for x in g:
            x.mul_(-0.7)
        plan.step(g, step=step, **HYPER, seed=seed, stochastic_rounding=form == "bf16_random")
        torch.cuda.synchronize()
        unit = 0
        for i, n in enumerate(sizes):
            blocks = -(-n // 256)
            random = ref.random16(unit, blocks * 32, seed)[:n]
            unit += blocks * 32
            m1, v1 = ref.moments32(g[i].cpu().numpy(), state[0][i], state[1][i] * state[1][i], 0.9, 0.999)
            root = np.sqrt(v1)
            swapped = (random & 255) << 8 | random >> 8
            for x, codes, scales, floor_one, k in ((m1, plan.exp_avgs[i], plan.exp_avg_scales[i], False, 0),
                                                   (root, plan.exp_avg_sqs[i], plan.exp_avg_sq_scales[i], True, 1)):
                want_codes, want_scale = ref.quantise(x, swapped, floor_one)
                assert np.array_equal(scales.cpu().numpy(), want_scale)
                assert np.array_equal(bits(codes), want_codes)
                state[k][i] = values[want_codes] * np.repeat(want_scale, 256)[:n]
            want, _, _ = ref.step64(p0[i], np.zeros(n), m1.astype(np.float64) / 0.9, v1.astype(np.float64) / 0.999, step=step, **HYPER)
            moved = np.abs(want - p0[i].astype(np.float64) * (1 - HYPER["lr"] * HYPER["weight_decay"]))
            if form == "master":
                check_param(f64(w[i]), want, moved)
            else:
                check_param(f64(p[i]), want, moved, form)


def test_codes_are_unbiased_over_all_random_numbers():
    # the reference that the kernel's codes equal bit for bit, over every 16-bit random number: the mean code value is the
    # value itself up to the grid of the random numbers (a step / 2^16), in every binade and below the smallest
    y = np.concatenate([[448.0], np.float32(2.0) ** np.linspace(-12, 8.8, 40, dtype=np.float32), [0.0]]).astype(np.float32)
    values = ref.e4m3_values()
    total = np.zeros(y.size)
    for r in range(65536):
        codes, scale = ref.quantise(y, np.full(y.size, r), False)
        total += values[codes]
    assert float(scale[0]) == 1.0
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-9))), -6) - 3)
    diff = total / 65536 - y.astype(np.float64)
    assert np.all(diff <= 0) and np.all(diff >= -step / 65536)


@gpu
def test_param_rounded_at_random_is_the_fp32_result_plus_its_half_word():
    n, seed = 3000, 77
    p16, g = tensors([n], BF16, 0.05, 1)[0], tensors([n], BF16, 1e-3, 2)[0]
    p32 = p16.float()
    for bits_ in (8, 32):
        a, b = [p16.clone()], [p32.clone()]
        optim.AdamWPlan.zeros(a, state_bits=bits_).step([g], step=1, **HYPER, seed=seed, stochastic_rounding=True)
        optim.AdamWPlan.zeros(b, state_bits=bits_).step([g], step=1, **HYPER, seed=seed, stochastic_rounding=True)
        random = ref.random16(0, -(-n // 256) * 32, seed)[:n].astype(np.int64)
        assert np.array_equal(bits(a[0]).view(np.uint16), ((bits(b[0]).view(np.uint32).astype(np.int64) + random) >> 16).astype(np.uint16))


@gpu
def test_slow_average_moves_in_8_bits():
    # sqrt(v) = 4 q, gradients of size q: v falls to q^2 at the rate beta2 = 0.999, which nearest rounding never shows
    n, q = 4096, 1e-3
    p = [torch.zeros(n, device="cuda")]
    plan = optim.AdamWPlan.zeros(p, state_bits=8)
    plan.exp_avg_sqs[0].view(torch.uint8).fill_(0x60)                       # 2^(12-7) = 32 in units of the scale
    plan.exp_avg_sq_scales[0].fill_(4 * q / 32)
    g = [torch.full((n,), q, device="cuda")]
    g[0][::256] = 40 * q                                                    # one large value a block keeps the scale up
    for t in range(1, 1001):
        plan.step(g, step=t, lr=0.0, weight_decay=0.0, seed=t)
    root = f64(plan.exp_avg_sqs[0].float() * plan.exp_avg_sq_scales[0].repeat_interleave(256)).reshape(-1, 256)[:, 1:]
    exact = np.sqrt(16 * 0.999 ** 1000 + (1 - 0.999 ** 1000)) * q
    # v follows the average of the squared codes, which the rounding's spread (a few per cent of sqrt(v) a step) raises a little
    assert abs(root.mean() / exact - 1) < 0.15
    assert abs(4 * q / exact - 1) > 0.5                                     # where it would have stayed


@gpu
def test_masked_edges_zero_blocks_and_non_finite():
    n = 600
    p = [torch.full((n,), 0.5, device="cuda")]
    plan = optim.AdamWPlan.zeros(p, state_bits=8)
    g = [torch.zeros(n, device="cuda")]
    g[0][300] = float("inf")                                                # the second of three blocks
    plan.step(g, step=1, lr=1e-2, weight_decay=0.0)
    assert torch.equal(p[0][:256], torch.full((256,), 0.5, device="cuda"))  # 0 / (0 + eps): no move
    assert torch.equal(p[0][512:], torch.full((88,), 0.5, device="cuda"))
    assert torch.isnan(p[0][300]) and int(torch.isnan(p[0]).sum()) == 1
    s = plan.exp_avg_scales[0]
    assert float(s[0]) == 0 and float(s[2]) == 0 and torch.isnan(s[1]) and torch.isnan(plan.exp_avg_sq_scales[0][1])
    assert int(plan.exp_avgs[0].view(torch.uint8)[:256].max()) == 0
    # a NaN gradient reaches a bf16 param as NaN, whatever the random bits
    q = [torch.ones(64, device="cuda", dtype=BF16)]
    g = [torch.full((64,), float("nan"), device="cuda")]
    plan = optim.AdamWPlan.zeros(q)
    plan.step(g, step=1, lr=1e-2, seed=3, stochastic_rounding=True)
    assert bool(torch.isnan(q[0]).all())


@gpu
def test_empty_lists_empty_tensors_and_more_than_one_launch():
    optim.AdamWPlan([], [], []).step([], step=1, lr=1.0)
    sizes = [0, 5, 0] + [3 + i % 5 for i in range(700)] + [0]
    p = tensors(sizes, BF16, 1.0, 1)
    g = tensors(sizes, F32, 1.0, 2)
    plan = optim.AdamWPlan.zeros(p, state_bits=8)
    plan.step(g, step=1, lr=1e-2, seed=9, stochastic_rounding=True)
    # the numbering of the random bits runs through all tensors, across launches
    flat_p = torch.zeros(703 * 256, dtype=BF16, device="cuda")
    flat_g = torch.zeros(703 * 256, device="cuda")
    full = [i for i, n in enumerate(sizes) if n]
    again = tensors(sizes, BF16, 1.0, 1)
    for k, i in enumerate(full):
        flat_p[k * 256:k * 256 + sizes[i]] = again[i]
        flat_g[k * 256:k * 256 + sizes[i]] = g[i]
    one = optim.AdamWPlan.zeros([flat_p], state_bits=8)
    one.step([flat_g], step=1, lr=1e-2, seed=9, stochastic_rounding=True)
    for k, i in enumerate(full):
        assert torch.equal(flat_p[k * 256:k * 256 + sizes[i]], p[i])
        assert np.array_equal(bits(one.exp_avgs[0])[k * 256:k * 256 + sizes[i]], bits(plan.exp_avgs[i]))


@gpu
def test_dimension_orders_streams_graphs_and_device_scale():
    gen = torch.Generator().manual_seed(3)
    w = torch.randn(8, 16, 3, 3, generator=gen).cuda().to(memory_format=torch.channels_last)
    g = torch.randn(8, 16, 3, 3, generator=gen).cuda().to(memory_format=torch.channels_last)
    a, b = [w.clone()], [w.clone().contiguous()]
    assert not a[0].is_contiguous()
    scale = torch.tensor([0.25], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pa = optim.AdamWPlan.zeros(a)
    pb = optim.AdamWPlan.zeros(b)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.step([g], step=1, lr=1e-2, dev_grad_scale=scale)
    torch.cuda.current_stream().wait_stream(side)
    pb.step([g.contiguous()], step=1, lr=1e-2, grad_scale=0.25)
    assert torch.equal(a[0], b[0])
    # captured and replayed: the same bits as the call
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.step([g], step=2, lr=1e-2, dev_grad_scale=scale)
    graph.replay()
    pb.step([g.contiguous()], step=2, lr=1e-2, grad_scale=0.25)
    assert torch.equal(a[0], b[0])
    with pytest.raises(ValueError):
        pa.step([g.contiguous()], step=3, lr=1e-2)                          # another dimension order than the param's
    with pytest.raises(ValueError):
        optim.AdamWPlan.zeros([torch.zeros(8, 8, device="cuda")[:, :4]])    # gaps
    with pytest.raises(TypeError):
        optim.AdamWPlan.zeros([torch.zeros(8, device="cuda", dtype=torch.float16)])


def test_refusals_before_any_launch():
    L = binding.lib()
    T, C = binding.AdamWTensor, binding.AdamWConfig

    def call(count=1, t=None, c=None, null=False):
        entry = dict(param=4096, grad=8192, exp_avg=1 << 14, exp_avg_sq=1 << 15, numel=16, param_dtype=0, grad_dtype=0)
        conf = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, grad_scale=1.0, state_bits=32)
        arr = (T * 1)(T(**{**entry, **(t or {})}))
        return L.mvue_adamw_step(None if null else arr, count, C(**{**conf, **(c or {})}), None)

    assert call(null=True) == -1 and L.mvue_adamw_step(None, 0, None, None) == -1
    assert call(count=-1) == -3 and call(c=dict(step=0)) == -3 and call(t=dict(numel=-1)) == -3
    assert call(t=dict(grad=None)) == -1 and call(t=dict(exp_avg=None)) == -1
    assert call(c=dict(state_bits=8)) == -1                                 # no scales
    assert call(c=dict(state_bits=16)) == -5 and call(t=dict(param_dtype=2)) == -5 and call(t=dict(master=4096)) == -5
    assert call(c=dict(options=2)) == -12 and call(c=dict(beta1=1.0)) == -12 and call(c=dict(beta2=-0.1)) == -12
    assert call(t=dict(grad=8194)) == -4 and call(t=dict(param=4097, param_dtype=1)) == -4
    if not torch.cuda.is_available():
        assert call() in (-8, -9)
