"""Newton-Schulz orthogonalisation and the Muon step of updates whose squares binary32 cannot hold: so small that they come out as zero
(a weight without gradient, whose momentum decays from step to step), or beyond the largest number."""
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding, optim

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# one small cluster's tiles, tiles of a product a launch, tiles of pairs
SHAPES = [(40, 60), (256, 256), (1000, 128), (100, 2500), (300, 270), (600, 2000)]


def noise(rows, cols, seed=2):
    return torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("scale", [1e-18, 1e-22, 2e-23, 1e-23, 5e-24, 2e-24, 1e-24, 3e-25, 1e-25, 1e-27, 1e-32, 1e-40, 1e17, 1e20, 1e25, 1e33, 3e37])
def test_orthogonalize(rows, cols, scale):
    # the bound of other magnitudes (five steps: 3e-3, twice that for few entries); 1e-40 is what binary32 holds of it
    x = noise(rows, cols) * scale
    assert bool(x.isfinite().all()) and bool(x.any())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = binding.mvue_orthogonalize(x, dev_status=status)
    assert bool(got.isfinite().all()) and rel(got, ref.orthogonalize(x)) < 6e-3 and int(status) == 0


@pytest.mark.parametrize("steps", [1, 3, 16])
def test_numbers_of_steps(steps):
    for scale in (5e-24, 3e-25, 1e-40, 1e30):
        x = noise(200, 300) * scale
        got = binding.mvue_orthogonalize(x, steps=steps)
        assert bool(got.isfinite().all())
        if scale < 1:                                       # the polynomial's first term alone: no step wanders
            assert rel(got, ref.orthogonalize(x, steps)) < 6e-3


@pytest.mark.parametrize("scale", [1e-24, 1e30])
def test_magnitudes_side_by_side(scale):
    # one piece of eight neighbours beside pieces of another magnitude, and zeros
    x = torch.zeros(64, 128, device="cuda")
    x[:, :8] = noise(64, 8) * scale
    x[:, 16:24] = noise(64, 8, seed=3) * scale * 1e3
    assert rel(binding.mvue_orthogonalize(x), ref.orthogonalize(x)) < 6e-3
    x[:32, 64:] = noise(32, 64, seed=4)
    assert rel(binding.mvue_orthogonalize(x), ref.orthogonalize(x)) < 6e-3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_momentum_that_decays(rows, cols, dtype):
    # no gradient: the momentum goes through all magnitudes down to zero; the update is what the definition says, next to nothing
    p = (0.02 * noise(rows, cols, seed=5)).to(dtype)
    m, g = 2e-22 * noise(rows, cols), torch.zeros(rows, cols, dtype=dtype, device="cuda")
    plan = optim.MuonPlan([p], [m], grads=[g])
    want = p.clone()
    for _ in range(12):
        plan.step(lr=0.02, momentum=0.5, weight_decay=0.0)
        # ||x|| / 1e-7 * 3.4445^5 <= 1.1e-9, times 0.2 lr max(rows, cols)^0.5 = 0.18, twice that over steps that halve: 4e-10; a param's own
        # roundings besides (a bf16 param far above goes back to what it was)
        assert bool(((p.double() - want.double()).abs() <= 1e-9 + 12 * U * want.double().abs()).all())
    assert float(m.abs().max()) < 1e-24


def test_not_finite_is_still_seen():
    x = noise(300, 270) * 1e-24
    x[3, 5] = float("inf")
    assert bool(binding.mvue_orthogonalize(x).isnan().all())
    x[3, 5] = float("nan")
    assert bool(binding.mvue_orthogonalize(x).isnan().all())
