"""e4m3 codes and scales bit for bit as the definition says (whole-number arithmetic on the host), both block shapes, both roundings."""
import numpy as np
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def same(x, block_rows, seed=None, **kw):
    codes, scales = binding.mvue_quantize_e4m3(x, block_rows, seed=seed, **kw)
    assert codes.dtype is torch.float8_e4m3fn and codes.shape == x.shape and scales.dtype is torch.uint8
    want, want_scales = ref.quantize(x.float().cpu().numpy(), block_rows, seed)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)
    np.testing.assert_array_equal(codes.contiguous().view(torch.uint8).cpu().numpy(), want)
    return codes, scales


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("seed", [None, 7, 2**63 + 11])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 17), (33, 129), (130, 300), (257, 1000), (64, 2050)])
def test_bits(rows, cols, block_rows, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(rows * cols)
    # heavy tails, rows of very different size, zeros: subnormal codes, carries into the next binade, ties
    x = torch.randn(rows, cols, generator=gen, device="cuda") ** 3 * torch.exp(4 * torch.randn(rows, 1, generator=gen, device="cuda"))
    x[torch.rand(rows, cols, generator=gen, device="cuda") < 0.3] = 0
    same(x.to(dtype), block_rows, seed)


@pytest.mark.parametrize("seed", [None, 3])
def test_every_code_and_every_tie(seed):
    # the values of all codes, their neighbours and their midpoints, beside a top that fixes the scale
    finite = [c for c in range(256) if c & 0x7F != 0x7F]
    values = torch.tensor(finite, dtype=torch.uint8).view(torch.float8_e4m3fn).double().sort().values
    mids = (values[1:] + values[:-1]) / 2
    points = torch.cat([values, mids, mids * (1 + 2.0 ** -20), mids * (1 - 2.0 ** -20)]).float()
    for k in (-120, -20, 0, 20, 118):
        x = torch.zeros(1, 128 * (-(-points.numel() // 127)))
        x.view(-1, 128)[:, 0] = 448.0
        x.view(-1, 128)[:, 1:] = torch.nn.functional.pad(points, (0, x.shape[1] // 128 * 127 - points.numel())).view(-1, 127)
        same((x * 2.0 ** k).cuda(), 1, seed)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_extremes(block_rows, dtype):
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x = torch.zeros(6, 256, dtype=dtype)
    x[0, 3], x[0, 200] = big, -big                      # the largest numbers there are
    x[1] = tiny                                         # at the least scale
    x[2, ::2] = tiny * 2.0 ** -6                        # subnormal
    x[3, 5], x[3, 6], x[3, 7] = float("inf"), -1.5, float("nan")
    x[4, 129], x[4, 130] = float("-inf"), 0.0           # nothing finite but zeros beside it
    x[5] = -0.0
    for seed in (None, 5):
        codes, scales = same(x.cuda(), block_rows, seed)
        assert bool(codes[3, [5, 7]].float().isnan().all()) and int(codes.float().isnan().sum()) == 3


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_given_outputs(dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    big = torch.randn(140, 400, generator=gen, device="cuda").to(dtype)
    for first, cols in ((0, 256), (1, 256), (2, 255), (8, 300), (3, 17)):
        for block_rows in (1, 128):
            same(big[:, first:first + cols], block_rows, 4)
            pitch = cols + 5
            room = torch.full((140, pitch), 0x55, dtype=torch.uint8, device="cuda")
            codes = room.view(torch.float8_e4m3fn)[:, :cols]
            same(big[:, first:first + cols], block_rows, None, codes=codes)
            assert bool((room[:, cols:] == 0x55).all())


def test_random_rounding_has_no_bias():
    # 2000 seeds: a code's mean is off by at most half the distance of two codes / sqrt(2000) at one deviation
    x = torch.randn(4, 256, device="cuda")
    total = torch.zeros(4, 256, dtype=torch.float64, device="cuda")
    for seed in range(2000):
        codes, scales = binding.mvue_quantize_e4m3(x, 1, seed=seed)
        total += ref.dequantize(codes, scales, 1)
    scale = torch.exp2(scales.double().T.repeat_interleave(128, 1) - 127)
    step = torch.exp2(torch.floor(torch.log2((x.double().abs() / scale).clamp(min=2.0 ** -6))) - 3) * scale
    z = (total / 2000 - x.double()) / step * (2000 ** 0.5 / 0.5)
    assert float(z.abs().max()) < 6 and abs(float(z.mean())) < 6 / 32


def test_empty_and_refused():
    for shape in ((0, 256), (5, 0)):
        codes, scales = binding.mvue_quantize_e4m3(torch.empty(shape, device="cuda"), 1)
        assert codes.shape == shape
    x = torch.zeros(4, 256, device="cuda")
    for bad in (lambda: binding.mvue_quantize_e4m3(x.T), lambda: binding.mvue_quantize_e4m3(x[None]), lambda: binding.mvue_quantize_e4m3(x.cpu()),
                lambda: binding.mvue_quantize_e4m3(x, scales=torch.zeros(4, 2, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        binding.mvue_quantize_e4m3(x.half())
    with pytest.raises(binding.MvueError) as e:
        binding.mvue_quantize_e4m3(x, 64)
    assert e.value.status == -3


def test_captured_and_replayed():
    x = torch.randn(300, 1000, device="cuda").to(BF16)
    want = binding.mvue_quantize_e4m3(x, 1, seed=9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.mvue_quantize_e4m3(x, 1, seed=9)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])
