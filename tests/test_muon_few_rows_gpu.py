"""Newton-Schulz orthogonalisation of matrices of a few rows or columns.  Their result hangs on a few singular values.  A rounding of X, A or the
matrix that multiplies X in one of five steps (2^-12 at most) reaches the last value multiplied by the slopes of the steps after it; summed up over all
roundings and at the worst first value these are 109, so an entry is off by 109 * 2^-12 = 2.7e-2 at most to first order.  The root of the sum of
their squares, averaged over first values, is 1.6e-3 (roundings of 2^-12 / 3^0.5): the median is a few times that at most."""
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(2, 2), (2, 33), (33, 2), (3, 17), (3, 381), (287, 4), (4, 1020), (8, 8), (20, 8), (2, 4000)])
def test_few_rows(rows, cols):
    x = torch.randn(2000, rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows + cols), device="cuda")
    got, want = binding.mvue_orthogonalize(x).double(), ref.orthogonalize(x)
    off = (got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert float(off.max()) < 2.7e-2 and float(off.median()) < 5e-3
    if min(rows, cols) >= 8:                                 # the worst of eight values, the others with it: a third
        assert float(off.max()) < 2.7e-2 / 3


def test_from_sixteen_rows_on():
    gen = torch.Generator(device="cuda").manual_seed(0)
    for rows, cols in ((16, 16), (16, 500), (40, 17), (31, 1000)):
        for r in (1, 2, 5, 16):                              # directions above the noise
            x = torch.randn(200, rows, r, generator=gen, device="cuda") @ torch.randn(200, r, cols, generator=gen, device="cuda")
            x += 0.03 * torch.randn(200, rows, cols, generator=gen, device="cuda")
            got, want = binding.mvue_orthogonalize(x).double(), ref.orthogonalize(x)
            assert float(((got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)).max()) < 6e-3
