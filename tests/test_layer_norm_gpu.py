"""Layer norm and its backward pass against the formulas in 64 bits, element for element within the bounds of tests/helpers/layer_ref.py."""
import itertools

import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def inputs(rows, cols, dtype, affine, seed=0, shift=0.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x = (normal(rows, cols) * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda")) + shift * normal(rows, 1)).to(dtype)
    w, b = (None, None) if affine is None else ((1 + 0.2 * normal(cols)).to(affine), (0.2 * normal(cols)).to(affine))
    return x, w, b, (1e-3 * normal(rows, cols)).to(dtype)


def within(got, want, bound, dtype=F32, what=""):
    off = (got.double() - want).abs()
    room = bound * 1.01 + want.abs() * ref.HALF_STEP[dtype] + 1e-38
    assert bool((off <= room).all()), (what, float((off / room).max()))


def check(x, w, b, dy, eps=1e-5, **kw):
    cols = x.shape[-1]
    y, mean, rstd = binding.mvue_layer_norm(x, w, b, eps=eps, **kw)
    assert y.shape == x.shape and mean.shape == rstd.shape == x.shape[:-1]
    want, bounds = ref.layer_norm(x, w, b, eps)
    for name, g, v, e, t in zip(("y", "mean", "rstd"), (y, mean, rstd), want, bounds, (x.dtype, F32, F32)):
        within(g, v, e, t, name)
    dx, dw, db = binding.mvue_layer_norm_backward(dy, x, mean, rstd, w)
    want, bounds = ref.layer_norm_backward(dy, x, mean, rstd, w)
    within(dx.reshape(-1, cols), want[0], bounds[0], x.dtype, "dx")
    within(dw, want[1], bounds[1], F32, "dw")
    within(db, want[2], bounds[2], F32, "db")
    return y, mean, rstd, dx, dw, db


# every route: few and many rows, one and several teams of a block, rows that a team covers exactly and not, pieces of eight, two
# and one, rows wider than a block's threads
SHAPES = [(1, 1), (1, 8), (3, 17), (2, 256), (7, 1000), (300, 30), (5000, 64), (4099, 256), (2500, 768), (3001, 1024), (1300, 1111), (1025, 2048),
          (601, 4096), (1200, 4104), (640, 4864), (150, 8192), (161, 8200), (5, 12288), (333, 16384), (160, 14336), (37, 9001), (400, 9000), (21, 30000), (3, 24577)]


@pytest.mark.parametrize("dtype,affine", [(BF16, F32), (F32, BF16), (BF16, None), (F32, F32)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_against_64_bits(rows, cols, dtype, affine):
    check(*inputs(rows, cols, dtype, affine, seed=rows + cols))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shapes_and_strides(dtype):
    # [n, s, c] as it is, rows of a wider matrix, odd strides and starts
    x, w, b, dy = inputs(6, 96, dtype, F32)
    check(x.reshape(2, 3, 96), w, b, dy.reshape(2, 3, 96))
    check(x[0], w, b, dy[0])
    for pad, first in itertools.product((0, 1, 2, 8, 13), (0, 1, 2, 8)):
        big = torch.full((700, first + 256 + pad), 7.0, dtype=dtype, device="cuda")
        big_dy = big.clone()
        xs, _, _, dys = inputs(700, 256, dtype, None, seed=pad)
        x_view, dy_view = big[:, first:first + 256], big_dy[:, first:first + 256]
        x_view.copy_(xs)
        dy_view.copy_(dys)
        out = torch.full_like(big, -3.0)
        y, mean, rstd = binding.mvue_layer_norm(x_view, out=out[:, first:first + 256])
        plain = binding.mvue_layer_norm(xs)
        within(y, ref.layer_norm(xs, None, None, 1e-5)[0][0], ref.layer_norm(xs, None, None, 1e-5)[1][0], dtype)
        within(plain[0], ref.layer_norm(xs, None, None, 1e-5)[0][0], ref.layer_norm(xs, None, None, 1e-5)[1][0], dtype)
        out[:, first:first + 256] = -3.0
        assert bool((out == -3.0).all())                                    # nothing beside the rows was written
        dx, dw, db = binding.mvue_layer_norm_backward(dy_view, x_view, mean, rstd, out=out[:, first:first + 256])
        want, bounds = ref.layer_norm_backward(dys, xs, mean, rstd, None)
        within(dx, want[0], bounds[0], dtype)
        within(dw, want[1], bounds[1])
        out[:, first:first + 256] = -3.0
        assert bool((out == -3.0).all())


@pytest.mark.parametrize("rows,cols", [(3, 100), (2000, 512), (700, 1111), (20, 9000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place(rows, cols, dtype):
    x, w, b, dy = inputs(rows, cols, dtype, F32)
    y, mean, rstd, dx, dw, db = check(x, w, b, dy)
    z = x.clone()
    assert torch.equal(binding.mvue_layer_norm(z, w, b, out=z)[0], y) and torch.equal(z, y)
    for target in (0, 1):
        g, a = dy.clone(), x.clone()
        got = binding.mvue_layer_norm_backward(g, a, mean, rstd, w, out=(g, a)[target])
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))


def test_rows_of_equal_numbers_and_rows_far_from_zero():
    # no variance: eps alone; a mean a thousand times the spread
    x = torch.full((500, 768), 3.25, device="cuda")
    x[1] = 0
    x[2:] += torch.randn(498, 768, device="cuda") * 3e-3
    for dtype in (BF16, F32):
        y = check(x.to(dtype), None, None, torch.randn_like(x).to(dtype))[0]
        assert not bool(y[:2].any())


@pytest.mark.parametrize("rows,cols", [(6, 48), (1500, 1024), (900, 300), (9, 9000)])
def test_what_is_not_finite_stays_in_its_row(rows, cols):
    x, w, b, dy = inputs(rows, cols, F32, F32)
    clean = binding.mvue_layer_norm(x, w, b)
    x[1, cols // 2], x[4, 3] = float("nan"), float("inf")
    y, mean, rstd = binding.mvue_layer_norm(x, w, b)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[1, 4]] = True
    assert bool(y[bad].isnan().all())
    for g, v in zip((y, mean, rstd), clean):
        assert torch.equal(g[~bad], v[~bad])
    dx = binding.mvue_layer_norm_backward(dy, x, mean, rstd, w)[0]
    assert bool(dx[bad].isnan().all()) and bool(dx[~bad].isfinite().all())


def test_gradient_against_differences():
    # 64-bit differences of the 64-bit formula, at a point that binary32 holds
    x, w, b, dy = inputs(4, 24, F32, F32, seed=9)
    dy = dy * 1e3
    _, mean, rstd = binding.mvue_layer_norm(x, w, b)
    dx, dw, db = binding.mvue_layer_norm_backward(dy, x, mean, rstd, w)
    loss = lambda x, w, b: (ref.layer_norm(x, w, b, 1e-5)[0][0] * dy.double()).sum()  # noqa: E731
    h = 1e-5
    for t, grad in ((x, dx), (w, dw), (b, db)):
        flat = t.double().reshape(-1)
        args = {id(x): x.double(), id(w): w.double(), id(b): b.double()}
        for i in range(0, flat.numel(), 7):
            up, down = flat.clone(), flat.clone()
            up[i] += h
            down[i] -= h
            values = [loss(*(v.reshape(t.shape) if u is t else args[id(u)] for u in (x, w, b))) for v in (up, down)]
            # the differences are off by h^2 times the third derivative (of order one) and 2^-52 / h; the kernel by its bounds
            assert abs(float((values[0] - values[1]) / (2 * h)) - float(grad.reshape(-1)[i])) < 2e-5 * (1 + float(grad.abs().max()))


def test_empty_and_refused():
    w = torch.ones(16, device="cuda")
    y, mean, rstd = binding.mvue_layer_norm(torch.empty(0, 16, device="cuda"), w, w)
    assert y.shape == (0, 16) and mean.shape == (0,)
    dx, dw, db = binding.mvue_layer_norm_backward(y, y, mean, rstd, w)
    assert not bool(dw.any()) and not bool(db.any()) and dx.shape == (0, 16)
    x = torch.zeros(4, 16, device="cuda")
    for call in (lambda: binding.mvue_layer_norm(x.T), lambda: binding.mvue_layer_norm(x, torch.ones(15, device="cuda")),
                 lambda: binding.mvue_layer_norm(torch.zeros(2, 3, 4, 16, device="cuda")[:, :, ::3]), lambda: binding.mvue_layer_norm(x.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.mvue_layer_norm(x.half()), lambda: binding.mvue_layer_norm(x, w, w.to(BF16))):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(binding.MvueError) as e:
        binding.mvue_layer_norm(torch.zeros(4, 0, device="cuda"))
    assert e.value.status == -3


def test_two_streams_and_a_captured_graph():
    x, w, b, dy = inputs(2000, 1024, BF16, F32)
    want = check(x, w, b, dy)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            y, mean, rstd = binding.mvue_layer_norm(x, w, b)
            got.append((y, mean, rstd, *binding.mvue_layer_norm_backward(dy, x, mean, rstd, w)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, v) for a, v in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, mean, rstd = binding.mvue_layer_norm(x, w, b)
        out = (y, mean, rstd, *binding.mvue_layer_norm_backward(dy, x, mean, rstd, w))
    for t in out:
        t.fill_(5)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, v) for a, v in zip(out, want))


def test_offsets_beyond_32_bits():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB of device memory")
    rows, cols = 2_200_000, 1024                                            # 2.25e9 elements
    x = torch.empty(rows, cols, dtype=BF16, device="cuda")
    x[:: rows // 4] = 1
    tail = torch.randn(300, cols, device="cuda").to(BF16)
    x[:-300] = 0
    x[-300:] = tail
    y, mean, rstd = binding.mvue_layer_norm(x, out=x)
    want = binding.mvue_layer_norm(tail)
    (v, _, _), (e, _, _) = ref.layer_norm(tail, None, None, 1e-5)
    within(y[-300:], v, e, BF16)
    assert not bool(y[:-300].any()) and torch.allclose(rstd[-300:], want[2], rtol=1e-5)
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,cols,dtype", [(3000, 1024, BF16), (3000, 1024, F32), (2000, 4864, BF16), (500, 9000, F32), (300, 1000, BF16), (9, 25000, F32)])
def test_workspace_of_any_allowed_alignment(rows, cols, dtype):
    x, w, b, dy = inputs(rows, cols, dtype, F32)
    _, mean, rstd = binding.mvue_layer_norm(x, w, b)
    want = binding.mvue_layer_norm_backward(dy, x, mean, rstd, w)
    room = torch.empty(binding.mvue_layer_norm_workspace_bytes(rows, cols) + 16, dtype=torch.uint8, device="cuda")
    got = binding.mvue_layer_norm_backward(dy, x, mean, rstd, w, workspace=room[16:])
    assert all(torch.equal(a, v) for a, v in zip(got, want))
    with pytest.raises(binding.MvueError) as e:
        binding.mvue_layer_norm_backward(dy, x, mean, rstd, w, workspace=room[8:-8])
    assert e.value.status == -7


@pytest.mark.parametrize("rows,cols", [(1, 16), (2, 17), (3, 23), (9, 31), (17, 40), (100, 77), (4001, 250), (2005, 1001), (40, 4081)])
@pytest.mark.parametrize("first,pad", [(0, 0), (1, 0), (3, 2), (0, 5), (8, 8)])
def test_what_lies_beside_a_row_does_not_count(rows, cols, first, pad):
    # rows at any distance from an aligned address in a matrix of NaN, alone and in place; and a row of NaN among others
    x, w, b, dy = inputs(rows, cols, BF16, F32, seed=rows)
    big_x, big_dy, big_y = (torch.full((rows, first + cols + pad), float("nan"), dtype=BF16, device="cuda") for _ in range(3))
    cut = slice(first, first + cols)
    big_x[:, cut], big_dy[:, cut] = x, dy
    y, mean, rstd = binding.mvue_layer_norm(big_x[:, cut], w, b, out=big_y[:, cut])
    want, bounds = ref.layer_norm(x, w, b, 1e-5)
    for g, v, e, t in zip((y, mean, rstd), want, bounds, (BF16, F32, F32)):
        within(g, v, e, t)
    assert int(big_y.isnan().sum()) == rows * (first + pad)
    dx, dw, db = binding.mvue_layer_norm_backward(big_dy[:, cut], big_x[:, cut], mean, rstd, w)
    want, bounds = ref.layer_norm_backward(dy, x, mean, rstd, w)
    for g, v, e, t in zip((dx, dw, db), want, bounds, (BF16, F32, F32)):
        within(g, v, e, t)
    again = binding.mvue_layer_norm_backward(big_dy[:, cut], big_x[:, cut], mean, rstd, w, out=big_dy[:, cut])
    if first == 0 and pad == 0:                       # (dx apart has another layout, and its sums another order, where there are gaps)
        assert all(torch.equal(a, v) for a, v in zip(again, (dx, dw, db)))
    within(again[0], want[0], bounds[0], BF16)
    assert int(big_dy.isnan().sum()) == rows * (first + pad)
    same, _, _ = binding.mvue_layer_norm(big_x[:, cut], w, b, out=big_x[:, cut])
    assert torch.equal(same, y)
    if rows > 2:
        bad = x.clone()
        bad[rows // 2] = float("nan")
        y_bad = binding.mvue_layer_norm(bad, w, b)[0]
        keep = torch.arange(rows, device="cuda") != rows // 2
        assert bool(y_bad[rows // 2].isnan().all()) and torch.equal(y_bad[keep], binding.mvue_layer_norm(x, w, b)[0][keep])
