"""Newton-Schulz orthogonalisation and the Muon step.

Two comparisons.  With the same arithmetic in 64 bits but the binary16 roundings of the operands, for one and two steps: the kernel differs
where a sum in binary32 (off by sqrt(K) 2^-24, 2^-19 for K = 1024) falls on the other side of a rounding (half a step, 2^-12), one entry in a
hundred and twenty at most, by a step of 2^-11: 4.5e-5 of the norm.  The second step multiplies that by up to 3.4 and flips a share of
4.5e-5 / 2^-12 = 18 % of its own roundings, 0.18^0.5 * 2^-11 / 3^0.5 each for three operands: 1.5e-4 + 2e-4.  After that the two are like two
draws of the roundings.  With the definition, five steps: an operand's rounding is off by up to 2^-12, 2^-12 / 3^0.5 on average, three
operands a step, slopes of 12 over the last two steps: 12 * 3^0.5 * 2^-12 / 3^0.5 = 3e-3, and twice that where few entries leave nothing to
average.  More steps wander: between 0.7 and 1.2 the polynomial's slope is above one in places."""
import numpy as np
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding, optim

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def spectra(rows, cols, gen):
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    yield "noise", normal(rows, cols)
    r = max(1, min(rows, cols) // 16)
    yield "few large directions", normal(rows, r) @ normal(r, cols) + 0.1 * normal(rows, cols)
    yield "fewer", normal(rows, 1) @ normal(1, cols) + 0.01 * normal(rows, cols)
    yield "rows of very different size", normal(rows, cols) * torch.exp(2 * normal(rows, 1))
    yield "rank one", normal(rows, 1) @ normal(1, cols)


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm().clamp(min=1e-300))


# vectors, one small cluster's tiles and their edges, pair tiles and theirs, wide and tall
SHAPES = [(1, 1), (1, 40), (33, 1), (16, 16), (64, 65), (128, 200), (130, 128), (256, 256), (250, 1000), (256, 1025), (257, 257), (300, 520), (777, 1111), (1030, 512)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for name, x in spectra(rows, cols, gen):
        got = binding.mvue_orthogonalize(x, dev_status=status)
        assert got.dtype is F32 and got.shape == x.shape
        assert rel(got, ref.orthogonalize(x)) < 6e-3, name
        assert torch.equal(got, binding.mvue_orthogonalize(x))
        b = binding.mvue_orthogonalize(x, out_dtype=BF16)
        assert bool(((b.double() - got.double()).abs() <= got.double().abs() * 2.0 ** -8).all())
    assert int(status) == 0


@pytest.mark.parametrize("steps", [1, 2, 3, 8, 16])
@pytest.mark.parametrize("rows,cols", [(17, 17), (100, 140), (256, 1000), (520, 300), (600, 1000)])
def test_numbers_of_steps(steps, rows, cols):
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    got = binding.mvue_orthogonalize(x, steps=steps)
    if steps <= 2:
        assert rel(got, ref.orthogonalize_rounded(x, steps)) < (1e-4, 5e-4)[steps - 1]
    if steps <= 5:
        assert rel(got, ref.orthogonalize(x, steps)) < 6e-3
    else:
        # the singular vectors stay, the values stay between the polynomial's least and greatest on its own range
        u, _, v = torch.linalg.svd(x.double(), full_matrices=False)
        core = u.T @ got.double() @ v.T
        assert float((core - core.diag().diag()).norm() / core.norm()) < 2e-2
        assert 0.5 < float(core.diag().min()) and float(core.diag().max()) < 1.3


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_batches_strides_and_in_place(dtype):
    gen = torch.Generator(device="cuda").manual_seed(4)
    for shape in ((5, 70, 90), (2, 3, 300, 130), (70, 33, 20)):
        x = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        got = binding.mvue_orthogonalize(x)
        flat = x.reshape(-1, *shape[-2:])
        for i in (0, flat.shape[0] - 1):
            assert torch.equal(got.reshape(flat.shape)[i], binding.mvue_orthogonalize(flat[i]))
        y = x.clone()
        assert torch.equal(binding.mvue_orthogonalize(y, out=y), got) and torch.equal(y, got)
        big = torch.full((*shape[:-1], shape[-1] + 11), 3.0, dtype=dtype, device="cuda")
        view = big[..., 3:3 + shape[-1]]
        view.copy_(x)
        out = torch.full_like(big, -2.0)
        binding.mvue_orthogonalize(view, out=out[..., 3:3 + shape[-1]])
        # (the norm is summed up in another order, and a last bit there changes the roundings)
        assert rel(out[..., 3:3 + shape[-1]], ref.orthogonalize(x)) < 6e-3 + (2.0 ** -8 if dtype is BF16 else 0)
        out[..., 3:3 + shape[-1]] = -2.0
        assert bool((out == -2.0).all())


@pytest.mark.parametrize("rows,cols", [(40, 60), (300, 270)])
def test_sizes_of_numbers(rows, cols):
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    for scale in (1e-20, 1e-12, 1e-8, 1e-6, 1e6, 1e15):
        got = binding.mvue_orthogonalize(x * scale)
        assert rel(got, ref.orthogonalize(x * scale)) < 6e-3, scale          # also where eps outweighs the norm
    assert not bool(binding.mvue_orthogonalize(x * 0).any())


@pytest.mark.parametrize("rows,cols", [(40, 60), (300, 270)])
def test_what_is_not_finite_stays_in_its_matrix(rows, cols):
    x = torch.randn(4, rows, cols, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    want = binding.mvue_orthogonalize(x)
    x[1, 3, 5], x[2, 0, 0] = float("nan"), float("inf")
    got = binding.mvue_orthogonalize(x)
    assert torch.equal(got[[0, 3]], want[[0, 3]]) and bool(got[[1, 2]].isnan().all())


def test_singular_values_and_vectors():
    x = torch.randn(200, 500, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    y = binding.mvue_orthogonalize(x).double()
    s = torch.linalg.svdvals(y)
    assert 0.65 < float(s.min()) and float(s.max()) < 1.25                   # the polynomial's fifth iterate on (0.01, 1) is in (0.68, 1.21)
    u, _, v = torch.linalg.svd(x.double(), full_matrices=False)
    core = u.T @ y @ v.T
    assert float((core - core.diag().diag()).norm() / core.norm()) < 6e-3


# ---- the step -----------------------------------------------------------------------------------------------------------
def step64(p, m, g, lr, mu, decay, rule, nesterov=True, grad_scale=1.0):
    p, m, g = p.double(), m.double(), g.double() * grad_scale
    m = mu * m + (1 - mu) * g
    u = mu * m + (1 - mu) * g if nesterov else m
    rows, cols = p.shape
    s = 0.2 * max(rows, cols) ** 0.5 if rule == "rms" else max(1.0, rows / cols) ** 0.5
    update = lr * s * ref.orthogonalize(u)
    return p * (1 - lr * decay) - update, m, update


def problem(shapes, param, grad, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    p = [(0.02 * normal(s)).to(BF16 if param != "f32" else F32) for s in shapes]
    masters = [(t.float() * (1 + 2.0 ** -10)) for t in p] if param == "bf16+f32" else None
    return p, masters, [1e-3 * normal(s) for s in shapes], [(1e-3 * normal(s)).to(grad) for s in shapes]


MIXED = [(60, 100), (100, 60), (60, 100), (300, 280), (1, 50), (60, 100), (280, 300), (7, 9), (300, 280)]


@pytest.mark.parametrize("param", ["f32", "bf16", "bf16+f32"])
@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("rule,nesterov", [("rms", True), ("shape", False)])
def test_step(param, grad, rule, nesterov):
    p, masters, m, g = problem(MIXED, param, grad)
    before = [(w if masters is None else v).clone() for w, v in zip(p, masters or p)]
    m0 = [t.clone() for t in m]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = optim.MuonPlan(p, m, masters=masters, grads=g)
    lr, mu, decay, gs = 0.03, 0.9, 0.1, 0.5
    plan.step(lr=lr, momentum=mu, weight_decay=decay, scale=rule, nesterov=nesterov, grad_scale=2 * gs, dev_grad_scale=torch.full((1,), 0.5, device="cuda"),
              dev_status=status)
    for i, (w, v, x) in enumerate(zip(p, before, g)):
        want, moment, update = step64(v, m0[i], x, lr, mu, decay, rule, nesterov, gs)
        assert bool(((m[i].double() - moment).abs() <= 4 * U * (m0[i].double().abs() + x.double().abs())).all())
        # the update within 6e-3 of its norm, a rounding of the param besides
        got = w if masters is None else masters[i]
        room = 6e-3 * float(update.norm()) + 4 * U * float(want.norm()) + (2.0 ** -8 * float(want.norm()) if param == "bf16" else 0)
        assert float((got.double() - want).norm()) <= room
        if masters is not None:
            assert torch.equal(w, masters[i].to(BF16))
    assert int(status) == 0


def test_momentum_over_steps_and_new_gradients():
    p, _, m, _ = problem([(40, 90), (400, 300)], "f32", F32)
    plan = optim.MuonPlan.zeros(p)
    m = [torch.zeros_like(t) for t in p]
    w = [t.double() for t in p]
    for k in range(3):
        g = problem([(40, 90), (400, 300)], "f32", F32, seed=10 + k)[3]
        plan.step(g, lr=0.01, weight_decay=0.0)
        for i in range(2):
            w[i], m[i], update = step64(w[i], m[i], g[i], 0.01, 0.95, 0.0, "rms")
            assert rel(plan.momentums[i], m[i]) < 1e-6
            assert float((p[i].double() - w[i]).norm()) < 6e-3 * (k + 1) * float(update.norm())


@pytest.mark.parametrize("shapes", [MIXED, [(64, 128)], [(33, 40), (129, 130)]])
def test_stochastic_rounding_bit_for_bit(shapes):
    # the same step on fp32 params gives the values that are rounded; matrices are numbered through, each padded to 256 elements
    p, _, m, g = problem(shapes, "bf16", F32)
    wide = [t.float() for t in p]
    optim.MuonPlan(wide, [t.clone() for t in m], grads=g).step(lr=0.03)
    optim.MuonPlan(p, m, grads=g).step(lr=0.03, stochastic_rounding=True, seed=77)
    first = 0
    for w, v in zip(p, wide):
        n = v.numel()
        padded = -(-n // 256) * 256
        r = ref.philox_halves(np.arange(first // 8, (first + padded) // 8), 2, 77).reshape(-1)[:n]
        bits = v.cpu().numpy().reshape(-1).view(np.uint32).astype(np.int64)
        want = ((bits + r) >> 16).astype(np.uint16)
        np.testing.assert_array_equal(w.cpu().view(torch.int16).numpy().view(np.uint16).reshape(-1), want)
        first += padded


def test_more_matrices_than_go_together():
    shapes = [(20, 30)] * 70 + [(30, 20)] * 3
    p, _, m, g = problem(shapes, "f32", F32)
    single = [t.clone() for t in p]
    optim.MuonPlan(p, [t.clone() for t in m], grads=g).step(lr=0.02)
    for i in (0, 63, 64, 69, 70, 72):
        optim.MuonPlan([single[i]], [m[i].clone()], grads=[g[i]]).step(lr=0.02)
        assert torch.equal(single[i], p[i])


def test_captured_and_replayed_beside_another_plan():
    p, _, m, g = problem([(130, 200), (300, 260)], "f32", F32)
    q, _, mq, gq = problem([(130, 200), (300, 260)], "f32", F32, seed=5)
    want = [t.clone() for t in p]
    again = optim.MuonPlan(want, [t.clone() for t in m], grads=g)
    want_q = [t.clone() for t in q]
    again_q = optim.MuonPlan(want_q, [t.clone() for t in mq], grads=gq)
    plan, other = optim.MuonPlan(p, m, grads=g), optim.MuonPlan(q, mq, grads=gq)
    graphs = []
    for each in (plan, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            each.step(lr=0.02)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):                                                       # both at once: each plan has a workspace of its own
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _ in range(3):
        again.step(lr=0.02)
        again_q.step(lr=0.02)
    assert all(torch.equal(a, b) for a, b in zip([*p, *q], [*want, *want_q]))


def test_plan_refuses():
    p = [torch.zeros(8, 16, device="cuda")]
    ok = torch.zeros(8, 16, device="cuda")
    for args, kw in (((p, []), {}), ((p, [ok.half()]), {}), ((p, [ok.T]), {}), ((p, [ok.cpu()]), {}), (([ok[0]], [ok[0]]), {}), (([ok[:, ::2]], [ok[:, :8]]), {}),
                     ((p, [ok]), {"masters": [ok]}), (([ok.cpu()], [ok.cpu()]), {}), ((p, [ok]), {"grads": [ok, ok]}), ((p, [ok]), {"grads": [ok.T]})):
        with pytest.raises(ValueError):
            optim.MuonPlan(*args, **kw)
    plan = optim.MuonPlan.zeros(p)
    for kw in ({"grads": None}, {"grads": [ok], "stochastic_rounding": True}, {"grads": [ok], "scale": "other"}, {"grads": [ok], "dev_grad_scale": torch.ones(1)},
               {"grads": [ok], "dev_status": torch.zeros(1, device="cuda")}):
        with pytest.raises(ValueError):
            plan.step(lr=0.1, **kw)
    for kw, status in (({"ns_steps": 0}, -3), ({"ns_steps": 17}, -3), ({"momentum": 1.0}, -12)):
        with pytest.raises(binding.MvueError) as e:
            plan.step([ok], lr=0.1, **kw)
        assert e.value.status == status
    p[0].data = torch.zeros(8, 16, device="cuda")
    with pytest.raises(ValueError):
        plan.step([ok], lr=0.1)
    optim.MuonPlan([], []).step([], lr=0.1)
    empty = [torch.zeros(0, 5, device="cuda")]
    optim.MuonPlan.zeros(empty).step(empty, lr=0.1)
    for bad in (lambda: binding.mvue_orthogonalize(ok[0]), lambda: binding.mvue_orthogonalize(ok.T), lambda: binding.mvue_orthogonalize(ok.cpu())):
        with pytest.raises(ValueError):
            bad()
    assert binding.mvue_orthogonalize(torch.zeros(3, 0, 5, device="cuda")).shape == (3, 0, 5)


def test_results_side_by_side_and_results_that_overlap():
    x = torch.randn(3, 40, 24, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda")
    beside = torch.full((40, 3, 24), 7.0, device="cuda")
    binding.mvue_orthogonalize(x, out=beside.transpose(0, 1))
    assert torch.equal(beside.transpose(0, 1), binding.mvue_orthogonalize(x))
    same = torch.randn(40, 24, generator=torch.Generator(device="cuda").manual_seed(10), device="cuda").expand(3, 40, 24)
    assert torch.equal(binding.mvue_orthogonalize(same)[2], binding.mvue_orthogonalize(same[0]))        # read three times
    for out in (torch.zeros(40, 24, device="cuda").expand(3, 40, 24), torch.zeros(4000, device="cuda").as_strided((3, 40, 24), (900, 24, 1)),
                torch.zeros(4000, device="cuda").as_strided((3, 40, 24), (20, 72, 1))):
        with pytest.raises(binding.MvueError) as e:
            binding.mvue_orthogonalize(x, out=out)
        assert e.value.status == -3


def test_a_plan_refuses_tensors_that_share_memory():
    a, b, c = (torch.zeros(8, 16, device="cuda") for _ in range(3))
    for params, momentums in (([a, a], [b, c]), ([a, b], [c, c]), ([a], [a]), ([a[:4], a[3:7]], [b[:4], c[:4]])):
        with pytest.raises(ValueError):
            optim.MuonPlan(params, momentums)
    optim.MuonPlan([a[:4], a[4:]], [b[:4], b[4:]])


def test_a_plan_dropped_after_a_step_on_another_stream():
    p, _, m, g = problem([(300, 260), (40, 500)], "f32", F32)
    want = [t.clone() for t in p]
    again = optim.MuonPlan(want, [t.clone() for t in m], grads=g)
    again.step(lr=0.02)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    plan = optim.MuonPlan(p, m, grads=g)
    need = plan._workspace.numel()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        plan.step(lr=0.02)
    del plan
    junk = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]      # would be the plan's workspace
    torch.cuda.synchronize()
    assert len(junk) == 3 and all(torch.equal(a, b) for a, b in zip(p, want))


@pytest.mark.parametrize("steps", [1, 2, 3, 5])
@pytest.mark.parametrize("batch,rows,cols", [(2, 321, 3274), (30, 300, 520), (12, 520, 300), (5, 1030, 512), (3, 600, 2000), (7, 197, 3708), (2, 2100, 1050), (40, 100, 2500)])
def test_products_of_every_tile_in_batches(batch, rows, cols, steps):
    # X X^T, A A and B X each go through the tiles that suit their own number: all small, all of pairs, or some of each
    gen = torch.Generator(device="cuda").manual_seed(batch + rows)
    x = torch.randn(batch, rows, cols, generator=gen, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = binding.mvue_orthogonalize(x, steps=steps, dev_status=status)
    assert torch.equal(got, binding.mvue_orthogonalize(x, steps=steps)) and int(status) == 0
    for i in {0, batch // 2, batch - 1}:
        want = ref.orthogonalize(x[i], steps)
        # 3^0.5 roundings of 2^-12 / 3^0.5 a step, by the slopes of later steps: 3.4 each from small values, 12 for the last two together
        assert rel(got[i], want) < 6e-3, (i, rel(got[i], want))
        if steps <= 2:                               # (sums of 4096 instead of 1024: twice as many roundings flip, 2^0.5 of 4.5e-5 and 2.5e-4)
            assert rel(got[i], ref.orthogonalize_rounded(x[i], steps)) < (1e-4, 5e-4)[steps - 1]
