"""A matrix orthogonalised alone and among others of its extents: below 1024 columns (two shares of eight steps of 64) the same bits, from there
on sums may be split otherwise, and both are as near to the definition."""
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows,cols", [(64, 16, 4096), (40, 81, 3850), (24, 128, 2500), (14, 300, 2048), (9, 4096, 700), (64, 100, 1000), (20, 256, 1024), (14, 700, 1000)])
def test_alone_and_among_others(batch, rows, cols):
    x = torch.randn(batch, rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda")
    got = binding.mvue_orthogonalize(x)
    assert torch.equal(got, binding.mvue_orthogonalize(x))
    for i in (0, batch - 1):
        alone = binding.mvue_orthogonalize(x[i])
        want = ref.orthogonalize(x[i])
        for y in (alone, got[i]):
            assert float((y.double() - want).norm() / want.norm()) < 6e-3
        if max(rows, cols) < 1024:
            assert torch.equal(alone, got[i])
