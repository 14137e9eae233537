"""Group norm with an activation on channels-last maps, forward and backward, against 64 bits: odd channel counts and
group sizes, one position to many, strides and alignments, means that are large against the deviation, refusals."""
import ctypes

import pytest
import torch

from paper_2203_10991_b200 import binding
from tests.helpers import norm_ref as ref

F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu"]
#        n, s, c, groups
SHAPES = [(1, 1, 1, 1), (2, 1, 8, 1), (3, 1, 64, 32), (2, 2, 24, 3), (3, 5, 7, 7), (2, 9, 30, 5), (1, 49, 512, 32), (2, 63, 96, 6),
          (5, 100, 80, 8), (2, 257, 33, 11), (1, 1000, 320, 32), (3, 1031, 56, 8), (2, 4099, 16, 1), (1, 20011, 64, 8), (300, 3, 40, 4)]


def inputs(n, s, c, dtype, affine, seed, shift=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, s, c, generator=gen) * (0.5 + torch.rand(c, generator=gen)) + shift * torch.randn(c, generator=gen)
    dy = torch.randn(n, s, c, generator=gen)
    w, b = 1 + 0.3 * torch.randn(c, generator=gen), 0.3 * torch.randn(c, generator=gen)
    return x.to(dtype).cuda(), dy.to(dtype).cuda(), w.to(affine).cuda(), b.to(affine).cuda()


def check_forward(got, x, groups, w, b, act, eps=1e-5):
    want, bound = ref.forward(x, groups, w, b, eps, act)
    for g, t, e in zip(got, want, bound):
        assert ref.inside(g, t, e)


def check_backward(got, dy, x, mean, rstd, groups, w, b, act):
    want, bound = ref.backward(dy, x, mean, rstd, groups, w, b, act)
    for g, t, e in zip(got, want, bound):
        assert ref.inside(g, t, e)


@gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,affine", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,s,c,groups", SHAPES)
def test_forward_and_backward(n, s, c, groups, dtype, affine, act):
    x, dy, w, b = inputs(n, s, c, dtype, affine, s + c)
    got = binding.mvue_group_norm_act(x, groups, w, b, act=act)
    check_forward(got, x, groups, w, b, act)
    _, mean, rstd = got
    back = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, w, b, act=act)
    check_backward(back, dy, x, mean, rstd, groups, w, b, act)
    again = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, groups, w, b, act=act)
    assert all(torch.equal(p, q) for p, q in zip(back, again))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_means_and_constant_groups(dtype):
    # deviations of a thousandth of the mean (as far as bf16 holds them), and channels that do not vary at all
    x, dy, w, b = inputs(2, 700, 32, F32, F32, 3)
    x = (x + 300).to(dtype)
    dy = dy.to(dtype)
    got = binding.mvue_group_norm_act(x, 4, w, b, act="none")
    check_forward(got, x, 4, w, b, "none")
    flat = torch.full((2, 50, 16), 5.0, device="cuda", dtype=dtype)
    y, mean, rstd = binding.mvue_group_norm_act(flat, 2, w[:16], b[:16], act="none", eps=1e-3)
    assert torch.equal(mean, torch.full_like(mean, 5.0))
    assert torch.equal(y.float(), b[:16].to(dtype).float().expand(2, 50, 16))
    zero = torch.zeros(1, 3, 8, device="cuda", dtype=dtype)
    assert float(binding.mvue_group_norm_act(zero, 1, act="silu")[0].abs().max()) == 0


@gpu
def test_without_affine_and_with_either():
    x, dy, w, b = inputs(2, 130, 48, BF16, F32, 8)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y = binding.mvue_group_norm_act(x, 6, ww, bb, act="silu")
        check_forward(y, x, 6, one if ww is None else ww, zero if bb is None else bb, "silu")
        back = binding.mvue_group_norm_act_backward(dy, x, y[1], y[2], 6, ww, bb, act="silu")
        check_backward(back, dy, x, y[1], y[2], 6, one if ww is None else ww, zero if bb is None else bb, "silu")


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lo", [0, 8, 3])
def test_channel_slices_images_and_in_place(dtype, lo):
    # a slice of the channels of a wider map: row stride and alignment of their own; [n, h, w, c] as well as [n, s, c]
    big, dyb, w, b = inputs(3, 12 * 11, 72, dtype, F32, 9)
    w, b = w[:40].contiguous(), b[:40].contiguous()
    x, dy = (t.reshape(3, 12, 11, 72)[..., lo:lo + 40] for t in (big, dyb))
    flat, dflat = big[..., lo:lo + 40], dyb[..., lo:lo + 40]
    out = torch.full((3, 12, 11, 72), 9.0, device="cuda", dtype=dtype)
    y, mean, rstd = binding.mvue_group_norm_act(x, 5, w, b, act="gelu", out=out[..., lo:lo + 40])
    check_forward((y.reshape(3, 132, 40), mean, rstd), flat, 5, w, b, "gelu")
    assert bool((out[..., :lo] == 9).all()) and bool((out[..., lo + 40:] == 9).all())
    dx, dw, db = binding.mvue_group_norm_act_backward(dy, x, mean, rstd, 5, w, b, act="gelu")
    check_backward((dx.reshape(3, 132, 40), dw, db), dflat, flat, mean, rstd, 5, w, b, "gelu")
    other = dyb.clone().reshape(3, 12, 11, 72)[..., lo:lo + 40]       # the same alignment and strides: the same route, the same bits
    same = binding.mvue_group_norm_act_backward(other, x, mean, rstd, 5, w, b, act="gelu", out=other)
    assert torch.equal(same[0], dx)
    inplace = big.clone().reshape(3, 12, 11, 72)[..., lo:lo + 40]
    binding.mvue_group_norm_act(inplace, 5, w, b, act="gelu", out=inplace)
    assert torch.equal(inplace, y)
    nchw = torch.randn(2, 16, 5, 7, device="cuda").to(dtype).to(memory_format=torch.channels_last)
    z = binding.mvue_group_norm_act(nchw.permute(0, 2, 3, 1), 4)[0]
    check = torch.nn.functional.group_norm(nchw.float(), 4).permute(0, 2, 3, 1)
    assert float((z.float() - check).abs().max()) < (2e-2 if dtype == BF16 else 1e-5)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lo,c,groups", [(2, 90, 30), (2, 64, 8), (1, 34, 17), (0, 10, 1), (4, 258, 6)])
def test_rows_that_allow_pairs(dtype, lo, c, groups):
    big, dyb, w, b = inputs(2, 333, c + 6, dtype, F32, c)
    w, b = w[:c].contiguous(), b[:c].contiguous()
    x, dy = big[..., lo:lo + c], dyb[..., lo:lo + c]
    got = binding.mvue_group_norm_act(x, groups, w, b, act="silu")
    check_forward(got, x, groups, w, b, "silu")
    out = torch.full_like(big, 4.0)
    back = binding.mvue_group_norm_act_backward(dy, x, got[1], got[2], groups, w, b, act="silu", out=out[..., lo:lo + c])
    check_backward(back, dy, x, got[1], got[2], groups, w, b, "silu")
    assert bool((out[..., :lo] == 4).all()) and bool((out[..., lo + c:] == 4).all())


@gpu
def test_empty_batch_stream_and_graph():
    w = torch.ones(16, device="cuda")
    x = torch.empty(0, 4, 16, device="cuda")
    y, mean, rstd = binding.mvue_group_norm_act(x, 2, w, w)
    assert y.shape == x.shape and mean.shape == (0, 2)
    dx, dw, db = binding.mvue_group_norm_act_backward(x, x, mean, rstd, 2, w, w)
    assert float(dw.abs().max()) == 0 and float(db.abs().max()) == 0
    x, dy, w, b = inputs(4, 300, 64, BF16, F32, 4)
    want = binding.mvue_group_norm_act(x, 8, w, b, act="silu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = binding.mvue_group_norm_act(x, 8, w, b, act="silu")
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    out = torch.empty_like(x)
    ws = torch.empty(binding.mvue_group_norm_workspace_bytes(4, 300, 64, 8), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mvue_group_norm_act(x, 8, w, b, act="silu", out=out, workspace=ws)
    graph.replay()
    assert torch.equal(out, want[0])


@gpu
def test_status_is_left_alone():
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    for shape in ((2, 3136, 64), (2, 20000, 64), (3, 10, 7)):
        x = torch.randn(shape, device="cuda")
        _, mean, rstd = binding.mvue_group_norm_act(x, 1, dev_status=status)
        binding.mvue_group_norm_act_backward(x, x, mean, rstd, 1, dev_status=status)
    assert int(status) == 7


@gpu
def test_a_bad_sample_stays_by_itself():
    x, dy, w, b = inputs(3, 40, 32, F32, F32, 5)
    clean = binding.mvue_group_norm_act(x, 4, w, b, act="relu")[0]
    x[1, 7, 9] = float("nan")
    y = binding.mvue_group_norm_act(x, 4, w, b, act="relu")[0]
    assert bool(torch.isnan(y[1, :, 8:16]).all())
    y[1, :, 8:16] = clean[1, :, 8:16]
    assert torch.equal(y, clean)


@pytest.mark.parametrize("act", ACTS)
def test_the_formula_against_differences(act):
    # the 64-bit backward pass that the kernels are held to, against central differences of the 64-bit forward pass
    gen = torch.Generator().manual_seed(1)
    n, s, c, groups, eps = 2, 6, 12, 3, 1e-3
    x, v, dy = (torch.randn(n, s, c, generator=gen, dtype=torch.float64) for _ in range(3))
    w, b, vw, vb = (torch.randn(c, generator=gen, dtype=torch.float64) for _ in range(4))

    def loss(t):
        y = ref.forward(x + t * v, groups, w + t * vw, b + t * vb, eps, act)[0][0]
        return float((y * dy).sum())

    (_, mean, rstd), _ = ref.forward(x, groups, w, b, eps, act)
    (dx, dw, db), _ = ref.backward(dy, x, mean, rstd, groups, w, b, act)
    h = 1e-6
    # third derivatives of order 10 to 100 times h^2, and 1e-16 x 100 / h of rounding; ReLU has no element within h of its step
    assert abs((loss(h) - loss(-h)) / (2 * h) - float((dx * v).sum() + (dw * vw).sum() + (db * vb).sum())) < 1e-6


def test_refusals_before_any_launch():
    L = binding.lib()
    p = ctypes.c_void_p

    def fwd(x=4096, dtype=1, n=2, s=4, c=16, ldx=16, groups=4, w=8192, aff=0, act=1, y=16384, ldy=16, ws=32768, nws=1 << 20):
        return L.mvue_group_norm_act(p(x), dtype, n, s, c, ldx, groups, p(w), p(w), aff, 1e-5, act, p(y), ldy, None, None, p(ws), nws, None, None)

    assert fwd(x=None) == -1 and fwd(y=None) == -1
    assert fwd(n=-1) == -3 and fwd(s=0) == -3 and fwd(c=0) == -3 and fwd(groups=5) == -3 and fwd(groups=0) == -3
    assert fwd(ldx=15) == -3 and fwd(ldy=15) == -3
    assert fwd(dtype=2) == -5 and fwd(aff=7) == -5 and fwd(act=4) == -14 and fwd(act=-1) == -14
    assert fwd(x=4097) == -4 and fwd(w=8194) == -4
    assert fwd(ws=None) == -7 and fwd(nws=8) == -7 and fwd(ws=32776) == -7
    assert fwd(n=0, x=None) == 0

    def bwd(dy=4096, lddy=16, x=8192, mean=1 << 14, dx=1 << 15, ld=16, act=2, dg=1 << 16, ws=1 << 17, nws=1 << 20):
        return L.mvue_group_norm_act_backward(p(dy), lddy, p(x), 16, 1, 2, 4, 16, 4, p(mean), p(mean), None, None, 0, act, p(dx), ld, p(dg), p(dg),
                                              p(ws), nws, None, None)

    assert bwd(dy=None) == -1 and bwd(x=None) == -1 and bwd(mean=None) == -1 and bwd(dx=None) == -1
    assert bwd(lddy=8) == -3 and bwd(ld=8) == -3 and bwd(act=9) == -14 and bwd(dg=65538) == -4 and bwd(ws=None) == -7
    assert binding.mvue_group_norm_workspace_bytes(0, 4, 16, 4) == 0
    with pytest.raises(binding.MvueError):
        binding.mvue_group_norm_workspace_bytes(1, 4, 16, 3)
    with pytest.raises(ValueError):
        binding._positions(torch.empty(2, 3, 4, 8).permute(0, 2, 1, 3))
