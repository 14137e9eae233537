"""Embedding lookup and its gradient by sorted tokens: against plain 64-bit sums, token counts from none to several
radix-sort tiles, hot ids that cross chunks, odd widths, strides, unknown ids, padding, refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2203_10991_b200 import binding

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu


def id_list(kind, tokens, vocab, gen, dtype=torch.int64):
    if kind == "one":
        ids = torch.full((tokens,), vocab - 1)
    elif kind == "hot":                                   # half of the tokens share an id, the rest are spread by their logarithm
        ids = (torch.exp(torch.rand(tokens, generator=gen, dtype=torch.float64) * np.log(vocab)) - 1).long().clamp(0, vocab - 1)
        ids[torch.rand(tokens, generator=gen) < 0.5] = vocab // 3
    elif kind == "sorted":
        ids = torch.arange(tokens) * vocab // max(1, tokens)
    else:
        ids = torch.randint(0, vocab, (tokens,), generator=gen)
    return ids.to(dtype).cuda()


@gpu
@pytest.mark.parametrize("w_dtype,out_dtype", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("cols", [1, 7, 8, 33, 256, 1100, 4096, 9000])
@pytest.mark.parametrize("tokens", [0, 1, 37])
def test_lookup(tokens, cols, w_dtype, out_dtype):
    gen = torch.Generator().manual_seed(cols + tokens)
    w = torch.randn(101, cols, generator=gen).to(w_dtype).cuda()
    for id_dtype in (torch.int32, torch.int64):
        ids = id_list("spread", tokens, 101, gen, id_dtype)
        got = binding.mvue_embedding(ids, w, scale=27.7, out_dtype=out_dtype)
        want = (w[ids.long()].float() * 27.7).to(out_dtype)         # one product, one rounding: the same bits
        assert got.shape == (tokens, cols) and torch.equal(got, want)


@gpu
def test_lookup_strides_shapes_and_unknown_ids():
    big = torch.randn(50, 96, device="cuda").to(BF16)
    for w in (big[:, :64], big[:, 1:65], big[:, 3:40]):
        ids = torch.randint(0, 50, (3, 5), device="cuda")
        assert torch.equal(binding.mvue_embedding(ids, w), w[ids])
        out = torch.full((15, 80), 7.0, device="cuda", dtype=BF16)
        binding.mvue_embedding(ids, w, out=out[:, :w.shape[1]])
        assert torch.equal(out[:, :w.shape[1]], w[ids.reshape(-1)]) and bool((out[:, w.shape[1]:] == 7).all())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.mvue_embedding(torch.tensor([0, 49], device="cuda"), big, dev_status=status)
    assert int(status) == 0
    got = binding.mvue_embedding(torch.tensor([-1, 3, 50, 2**40], device="cuda"), big, dev_status=status)
    assert int(status) == -13
    assert torch.equal(got[1], big[3]) and float(got[[0, 2, 3]].abs().max()) == 0


@gpu
@pytest.mark.parametrize("lo,cols", [(2, 34), (2, 64), (1, 34), (4, 1030), (0, 90)])
def test_rows_that_allow_pairs(lo, cols):
    # even widths on even and odd offsets: pieces of eight, pairs, single elements
    big = torch.randn(60, 1040, device="cuda")
    ids = torch.randint(0, 60, (500,), device="cuda")
    for dtype in (F32, BF16):
        w = big.to(dtype)[:, lo:lo + cols]
        assert torch.equal(binding.mvue_embedding(ids, w), w[ids])
        wide = torch.randn(500, 1040, device="cuda").to(dtype)
        out = torch.full((60, 1040), 5.0, device="cuda")
        binding.mvue_embedding_grad(ids, wide[:, lo:lo + cols], 60, out=out[:, lo:lo + cols])
        check_grad(out[:, lo:lo + cols], ids, wide[:, lo:lo + cols], 60, 1.0)
        assert bool((out[:, :lo] == 5).all()) and bool((out[:, lo + cols:] == 5).all())


def sums64(ids, dy, vocab, scale, padding):
    """(sum, sum of magnitudes, count) for each id, in 64 bits."""
    keep = (ids >= 0) & (ids < vocab) & (ids != padding)
    ids, dy = ids[keep].long(), dy[keep].double()
    out = [torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device=dy.device).index_add_(0, ids, x) for x in (dy, dy.abs())]
    return out[0] * scale, out[1] * abs(scale), torch.bincount(ids, minlength=vocab).double()


def check_grad(got, ids, dy, vocab, scale, padding=-1, old=None):
    total, mags, count = sums64(ids, dy, vocab, scale, padding)
    # additions in a run of 32 tokens, additions of runs (a token's run may be cut at both ends), the product
    bound = mags * ((torch.minimum(count, torch.tensor(32.0, device=count.device)) + torch.ceil(count / 32) + 3) * U)[:, None]
    if old is not None:
        total = total + old.double()
        bound = bound + U * total.abs() * (count > 0)[:, None]
    lo, hi = total - bound, total + bound
    if got.dtype == BF16:                                   # rounding is monotone
        lo, hi = lo.float().to(BF16), hi.float().to(BF16)
    assert bool(((lo.double() <= got.double()) & (got.double() <= hi.double())).all())


@gpu
@pytest.mark.parametrize("dtype,dw_dtype", [(BF16, F32), (F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("kind", ["one", "hot", "sorted", "spread"])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (2, 5, 8), (31, 300, 40), (33, 511, 33), (64, 512, 264), (1000, 1000, 96),
                                               (4097, 40, 24), (9000, 70000, 64), (50001, 262145, 8)])
def test_gradient(tokens, vocab, cols, kind, dtype, dw_dtype):
    gen = torch.Generator().manual_seed(tokens)
    ids = id_list(kind, tokens, vocab, gen, torch.int32 if tokens % 2 else torch.int64)
    dy = torch.randn(tokens, cols, generator=gen).to(dtype).cuda()
    got = binding.mvue_embedding_grad(ids, dy, vocab, scale=0.5, out_dtype=dw_dtype, out=torch.full((vocab, cols), float("nan"), device="cuda", dtype=dw_dtype))
    check_grad(got, ids, dy, vocab, 0.5)
    again = binding.mvue_embedding_grad(ids, dy, vocab, scale=0.5, out_dtype=dw_dtype)
    assert torch.equal(got, again)                          # bit for bit, whatever the schedule
    whole = torch.randint(-8, 9, (tokens, cols), generator=gen).to(dtype).cuda()
    if dw_dtype == F32:                                     # whole numbers add without rounding: equality
        want, _, _ = sums64(ids, whole, vocab, 1.0, -1)
        assert torch.equal(binding.mvue_embedding_grad(ids, whole, vocab).double(), want)


@gpu
@pytest.mark.parametrize("tokens", [0, 1, 700])
def test_gradient_accumulates_skips_padding_and_unknown_ids(tokens):
    gen = torch.Generator().manual_seed(5)
    vocab, cols = 90, 72
    ids = torch.randint(-5, 95, (tokens,), generator=gen).cuda()
    dy = torch.randn(tokens, cols, generator=gen).to(BF16).cuda()
    old = torch.randn(vocab, cols, generator=gen).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = binding.mvue_embedding_grad(ids, dy, vocab, scale=2.0, padding_idx=7, out=old.clone(), accumulate=True, dev_status=status)
    check_grad(got, ids, dy, vocab, 2.0, 7, old)
    assert torch.equal(got[7], old[7])
    fresh = binding.mvue_embedding_grad(ids, dy, vocab, scale=2.0, padding_idx=7)
    check_grad(fresh, ids, dy, vocab, 2.0, 7)
    assert float(fresh[7].abs().max()) == 0
    if tokens == 700:
        assert int(status) == -13


@gpu
def test_gradient_strides_workspace_stream_and_graph():
    gen = torch.Generator().manual_seed(6)
    tokens, vocab, cols = 5000, 3000, 48
    ids = id_list("hot", tokens, vocab, gen)
    wide = torch.randn(tokens, 80, generator=gen).cuda()
    for dy in (wide[:, :48], wide[:, 5:53]):
        out = torch.full((vocab, 64), 3.0, device="cuda")
        for view in (out[:, 8:56], out[:, 1:49]):
            out.fill_(3.0)
            binding.mvue_embedding_grad(ids, dy, vocab, out=view)
            check_grad(view, ids, dy, vocab, 1.0)
            assert int((out == 3.0).sum()) >= vocab * 16    # beside the view nothing is written
    dy = wide[:, :48].contiguous()
    ws = torch.empty(binding.mvue_embedding_grad_workspace_bytes(tokens, cols), dtype=torch.uint8, device="cuda")
    out = torch.empty(vocab, cols, device="cuda")
    want = binding.mvue_embedding_grad(ids, dy, vocab)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        binding.mvue_embedding_grad(ids, dy, vocab, out=out, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mvue_embedding_grad(ids, dy, vocab, out=out, workspace=ws)
    dy.mul_(2.0)
    graph.replay()
    assert torch.equal(out, want * 2)


@gpu
def test_gradient_is_the_lookups():
    # <dy, d out> against differences of <dy, out> in the direction of a random dW, in 64 bits of the tables' fp32 results:
    # the lookup is linear, so a difference over 1 is exact but for fp32 roundings
    gen = torch.Generator().manual_seed(7)
    ids = id_list("hot", 300, 50, gen)
    w, v = (torch.randn(50, 20, generator=gen).cuda() for _ in range(2))
    dy = torch.randn(300, 20, generator=gen).cuda()
    diff = ((binding.mvue_embedding(ids, w + v, scale=3.0) - binding.mvue_embedding(ids, w, scale=3.0)).double() * dy).sum()
    grad = binding.mvue_embedding_grad(ids, dy, 50, scale=3.0).double()
    size = (w.double().abs() + v.double().abs())
    slack = 8 * U * 3.0 * (size[ids] * dy.abs()).sum() + 400 * U * (grad.abs() * v.abs()).sum()
    assert abs(float(diff - (grad * v).sum())) <= float(slack)


def test_refusals_before_any_launch():
    L = binding.lib()
    p = ctypes.c_void_p

    def look(ids=4096, id_bits=64, tokens=4, w=8192, w_dtype=1, vocab=10, cols=8, ldw=8, out=16384, out_dtype=1, ldo=8):
        return L.mvue_embedding(p(ids), id_bits, tokens, p(w), w_dtype, vocab, cols, ldw, 1.0, p(out), out_dtype, ldo, None, None)

    assert look(ids=None) == -1 and look(w=None) == -1 and look(out=None) == -1
    assert look(tokens=-1) == -3 and look(vocab=0) == -3 and look(cols=0) == -3 and look(ldw=7) == -3 and look(ldo=7) == -3
    assert look(id_bits=16) == -5 and look(w_dtype=2) == -5 and look(out_dtype=-1) == -5
    assert look(ids=4100) == -4 and look(w=8193) == -4 and look(out=16386, out_dtype=0) == -4
    assert look(tokens=0, ids=None) == 0

    def grad(ids=4096, id_bits=64, tokens=4, dy=8192, dy_dtype=1, cols=8, ldy=8, dw=16384, dw_dtype=0, vocab=10, ldw=8, acc=0, ws=32768, nws=1 << 20):
        return L.mvue_embedding_grad(p(ids), id_bits, tokens, p(dy), dy_dtype, cols, ldy, 1.0, -1, p(dw), dw_dtype, vocab, ldw, acc, p(ws), nws, None, None)

    assert grad(ids=None) == -1 and grad(dy=None) == -1 and grad(dw=None) == -1
    assert grad(tokens=-1) == -3 and grad(vocab=0) == -3 and grad(ldy=7) == -3 and grad(ldw=7) == -3
    assert grad(dy_dtype=3) == -5 and grad(dw_dtype=1, acc=1) == -5 and grad(id_bits=8) == -5
    assert grad(dw=16386) == -4 and grad(dy=8193) == -4 and grad(ids=4098, id_bits=32) == -4
    assert grad(ws=None) == -7 and grad(nws=16) == -7 and grad(ws=32776) == -7
    assert grad(tokens=0, acc=1, ids=None, dy=None, ws=None) == 0
    assert binding.mvue_embedding_grad_workspace_bytes(0, 5) == 0
    with pytest.raises(binding.MvueError):
        binding.mvue_embedding_grad_workspace_bytes(-1, 5)
