"""Dense products of e4m3 codes with block scales against 64-bit products of what the codes stand for.

The products of two codes and their scales are exact in binary32; sums of K of them, in whatever order the tensor cores take and each
addition off by at most a unit in the last place, are within K 2^-23 of the sum of magnitudes.  Entries where that is much looser than what
roundings do are held by the norm: 2^-23 of a sum that has grown over K / 32 instructions, so K / 32 2^-24 of the result's norm and a few."""
import pytest
import torch

from tests.helpers import layer_ref as ref
from paper_2203_10991_b200 import binding

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def operands(tokens, out, inp, way, seed=0, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    a = normal(tokens, inp if way == "forward" else out) * torch.exp(spread * normal(tokens, 1))
    w = normal(out, inp) * torch.exp(spread * normal(out, 1))
    return (*binding.mvue_quantize_e4m3(a, 1, seed=seed), *binding.mvue_quantize_e4m3(w, 128))


def product(way, *args, **kw):
    return (binding.mvue_scaled_forward_gemm if way == "forward" else binding.mvue_scaled_backward_gemm)(*args, **kw)


def check(got, way, a, a_scales, w, w_scales):
    x, v = ref.dequantize(a, a_scales, 1), ref.dequantize(w, w_scales, 128)
    v = v.T if way == "forward" else v
    want, room = x @ v, x.abs() @ v.abs()
    k = x.shape[1]
    off = (got.double() - want).abs()
    assert bool((off <= k * 2.0 ** -23 * room + want.abs() * ref.HALF_STEP[got.dtype] + 1e-38).all())
    bound = (k / 32 + 8) * 2.0 ** -24 + ref.HALF_STEP[got.dtype]
    assert float((got.double() - want).norm()) <= bound * float(want.norm()), float((got.double() - want).norm() / want.norm())


# one token to several tiles of pairs; extents that end inside a tile, a scale block, sixteen codes; splits of the reduction with empty parts
SHAPES = [(1, 1, 1), (1, 17, 130), (8, 128, 128), (16, 300, 1111), (17, 129, 5000), (64, 777, 333), (65, 256, 2048), (128, 4096, 512), (129, 257, 385),
          (300, 700, 9000), (500, 2000, 640), (1000, 1111, 777), (2049, 2300, 300), (3000, 4100, 129), (4096, 4096, 1024), (70, 130, 20000)]


@pytest.mark.parametrize("way", ["forward", "backward"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inp", SHAPES)
def test_against_64_bits(tokens, out, inp, dtype, way):
    args = operands(tokens, out, inp, way, seed=tokens + out)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = product(way, *args, out_dtype=dtype, dev_status=status)
    assert got.shape == (tokens, out if way == "forward" else inp) and got.dtype is dtype
    check(got, way, *args)
    assert torch.equal(got, product(way, *args, out_dtype=dtype))           # equal inputs, equal bits
    assert int(status) == 0


@pytest.mark.parametrize("way", ["forward", "backward"])
@pytest.mark.parametrize("tokens,out,inp", [(5, 200, 300), (1500, 1300, 700)])
def test_scales_anywhere_in_their_range(tokens, out, inp, way):
    a, a_scales, w, w_scales = operands(tokens, out, inp, way, spread=0.0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    # rows of A up to 2^40 apart, blocks of W too; products stay within binary32
    a_scales = (a_scales.int() + torch.randint(-40, 41, a_scales.shape, generator=gen, device="cuda")).to(torch.uint8)
    w_scales = (w_scales.int() + torch.randint(-40, 41, w_scales.shape, generator=gen, device="cuda")).to(torch.uint8)
    check(product(way, a, a_scales, w, w_scales, out_dtype=F32), way, a, a_scales, w, w_scales)


@pytest.mark.parametrize("way", ["forward", "backward"])
@pytest.mark.parametrize("tokens,out,inp", [(4, 300, 260), (1100, 1500, 1030)])
def test_nan_reaches_its_row_or_column_only(tokens, out, inp, way):
    a, a_scales, w, w_scales = operands(tokens, out, inp, way)
    clean = product(way, a, a_scales, w, w_scales, out_dtype=F32)
    a.view(torch.uint8)[2, 7] = 0x7F
    n = 55 if way == "forward" else 61
    if way == "forward":
        w.view(torch.uint8)[n, 9] = 0xFF
    else:
        w.view(torch.uint8)[9, n] = 0xFF
    got = product(way, a, a_scales, w, w_scales, out_dtype=F32)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[2], bad[:, n] = True, True
    assert bool(got[bad].isnan().all()) and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens", [7, 1024])
def test_outputs_of_any_stride_and_pitched_codes(tokens, dtype):
    for way in ("forward", "backward"):
        args = operands(tokens, 520, 1100, way)
        want = product(way, *args, out_dtype=dtype)
        for first, pad in ((0, 0), (0, 5), (1, 2), (4, 4), (8, 24)):
            big = torch.full((tokens, first + want.shape[1] + pad), -5.0, dtype=dtype, device="cuda")
            view = big[:, first:first + want.shape[1]]
            assert product(way, *args, out=view) is view and torch.equal(view, want)
            view.fill_(-5.0)
            assert bool((big == -5.0).all())
        # codes in wider rows, with whatever beside them
        wide = torch.full((tokens, 2048), 0x7F, dtype=torch.uint8, device="cuda")
        wide[:, 16:16 + args[0].shape[1]] = args[0].view(torch.uint8)
        assert torch.equal(product(way, wide[:, 16:16 + args[0].shape[1]], *args[1:], out_dtype=dtype), want)


def test_what_lies_behind_the_scales_and_codes_does_not_count():
    # blocks at the edges are short: NaN where a wrong index would read
    a, a_scales, w, w_scales = operands(200, 300, 300, "forward")
    want = binding.mvue_scaled_forward_gemm(a, a_scales, w, w_scales)
    room = torch.full((a_scales.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    room[2048:2048 + a_scales.numel()] = a_scales.reshape(-1)
    w_room = torch.full((w_scales.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    w_room[2048:2048 + w_scales.numel()] = w_scales.reshape(-1)
    got = binding.mvue_scaled_forward_gemm(a, room[2048:2048 + a_scales.numel()].view(a_scales.shape), w,
                                           w_room[2048:2048 + w_scales.numel()].view(w_scales.shape))
    assert torch.equal(got, want)


def test_empty_and_refused():
    a, a_scales, w, w_scales = operands(8, 32, 64, "forward")
    assert binding.mvue_scaled_forward_gemm(a[:0], a_scales[:, :0].contiguous(), w, w_scales).shape == (0, 32)
    ok = (a, a_scales, w, w_scales)
    for i, bad in ((0, a.float()), (0, a[None]), (0, a.T), (1, a_scales.int()), (1, a_scales[:, :7].contiguous()), (2, w.view(torch.int8)), (3, w_scales.T.expand(1, 2)),
                   (0, a[:, :63]), (0, a.cpu()), (3, w_scales.cpu())):
        with pytest.raises(ValueError):
            binding.mvue_scaled_forward_gemm(*(bad if j == i else t for j, t in enumerate(ok)))
    with pytest.raises(TypeError):
        binding.mvue_scaled_forward_gemm(*ok, out_dtype=torch.float16)
    odd = torch.zeros(8, 72, dtype=torch.uint8, device="cuda")
    for codes in (odd[:, :64], torch.zeros(8 * 80 + 1, dtype=torch.uint8, device="cuda")[1:].view(8, 80)[:, :64]):       # pitch; base
        with pytest.raises(binding.MvueError) as e:
            binding.mvue_scaled_forward_gemm(codes, *ok[1:])
        assert e.value.status == -4


@pytest.mark.parametrize("tokens", [16, 2000])
def test_two_streams_and_a_captured_graph(tokens):
    args = operands(tokens, 2048, 1024, "backward")
    want = binding.mvue_scaled_backward_gemm(*args)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(s):
            got.append(binding.mvue_scaled_backward_gemm(*args))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got.append(binding.mvue_scaled_backward_gemm(*args))
        got.append(binding.mvue_scaled_backward_gemm(*args))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_offsets_beyond_32_bits():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB of device memory")
    tokens, out, inp = 2_300_000, 1024, 128                                  # 2.36e9 results
    a = torch.zeros(tokens, inp, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    tail, tail_scales, w, w_scales = operands(300, out, inp, "forward")
    a[-300:] = tail
    a_scales = torch.full((1, tokens), 127, dtype=torch.uint8, device="cuda")
    a_scales[:, -300:] = tail_scales
    got = binding.mvue_scaled_forward_gemm(a, a_scales, w, w_scales)
    check(got[-300:], "forward", tail, tail_scales, w, w_scales)
    assert not bool(got[:-300].any())
    del got, a
    torch.cuda.empty_cache()
