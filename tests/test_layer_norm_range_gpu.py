"""Layer norm at the ends of binary32's range: right while squares about the mean have room, and beyond that as the header says."""
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu
SHAPES = [(5, 64), (7, 1111), (2000, 1024), (700, 1000), (3, 9000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_large_values(rows, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    noise, beta = torch.randn(rows, cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    # squares of 5e16, 1e5 of them, are below 3.4e38
    x = (noise * 1e16).to(dtype)
    y, mean, rstd = binding.mvue_layer_norm(x, None, beta)
    (want, want_mean, want_rstd), (d_y, d_mean, d_rstd) = ref.layer_norm(x, None, beta, 1e-5)
    for g, v, e, t in ((y, want, d_y, dtype), (mean, want_mean, d_mean, torch.float32), (rstd, want_rstd, d_rstd, torch.float32)):
        assert bool(((g.double() - v).abs() <= 1.01 * e + v.abs() * ref.HALF_STEP[t] + 1e-38).all())
    # values of 1e25: their squares are not
    y, mean, rstd = binding.mvue_layer_norm((noise * 1e25).to(dtype), None, beta)
    assert not bool(rstd.any()) and torch.equal(y, beta.to(dtype).expand_as(y))
    # equal ones have a mean and no squares
    y, mean, rstd = binding.mvue_layer_norm(torch.full((rows, cols), 2.0 ** 100, dtype=dtype, device="cuda"), None, beta, eps=1.0)
    assert bool(((mean.double() / 2.0 ** 100 - 1).abs() <= ref.DEPTH * ref.U).all())


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_small_values(rows, cols):
    # far below eps: y is next to beta, whatever became of the squares
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, beta = torch.randn(rows, cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    for scale in (1e-18, 1e-25, 1e-40):
        y, _, rstd = binding.mvue_layer_norm(x * scale, None, beta)
        assert torch.allclose(y, beta.expand_as(y), rtol=0, atol=1e-14) and bool(((rstd.double() * 1e-5 ** 0.5 - 1).abs() < 8 * ref.U).all())
