"""Newton-Schulz orthogonalisation of long rows: a tensor core's sum cuts off what lies below its last place, so one accumulator takes
2^17 terms at most.  2^13 additions (of sixteen terms) that lose half of 2^-23 of the sum each: A is off by 2^-11, a step by as much at most, less
than what the roundings of the operands do in five steps.  Rows longer than eight such sums are refused.  Sums of pair tiles
go through a rounding of A to binary16 for each 2^17 terms: 2^-12 of A, eight times at most, as the one that there is anyway."""
import ctypes

import pytest
import torch

from paper_2203_10991_b200 import binding

A, B, C = 3.4445, -4.7750, 2.0315
CHUNK = 1 << 20


def polynomial(x, steps):
    """The matrix P with x' = P x in 64 bits, for one matrix x [few, many], through X X^T."""
    rows = x.shape[0]
    eye = torch.eye(rows, dtype=torch.float64, device=x.device)
    gram = torch.zeros_like(eye)
    for c in x.split(CHUNK, 1):
        gram += c.double() @ c.double().T
    norm = gram.diagonal().sum().sqrt() + 1e-7
    gram /= norm * norm
    p = eye
    for _ in range(steps):
        s = p @ gram @ p.T
        p = (A * eye + B * s + C * (s @ s)) @ p
    return p / norm


def off(got, x, steps):
    p = polynomial(x, steps)
    wrong = whole = 0.0
    for g, c in zip(got.split(CHUNK, 1), x.split(CHUNK, 1)):
        want = p @ c.double()
        wrong += float((g.double() - want).square().sum())
        whole += float(want.square().sum())
    return (wrong / whole) ** 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 2, 2**20), (1, 16, 2**20 - 7), (24, 16, 2**20), (40, 2, 2**19 + 1), (1, 1030, 2**20), (3, 300, 2**18 + 8), (1, 700, 2**19),
                                             (1, 128, 2**18), (64, 2, 2**18),
                                             (1, 1800, 2**17 + 8), (1, 2000, 2**19), (1, 1793, 2**18 - 1)])
def test_long_rows(batch, rows, cols):
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.empty(batch, rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    # and a direction that all rows share, three times as strong
    x += 3 * torch.randn(batch, rows, 1, generator=gen, device="cuda").to(x.dtype) * torch.randn(batch, 1, cols, generator=gen, device="cuda").to(x.dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for steps in (1, 5):
        got = binding.mvue_orthogonalize(x, steps=steps, out_dtype=torch.float32, dev_status=status)
        for i in {0, batch - 1}:
            # (five steps: the bound of other extents; one: 2^-11 and the roundings of three operands)
            assert off(got[i], x[i], steps) < (3e-3 if steps == 1 else 6e-3)
        del got
    if rows == 2 and batch == 1:                                             # long columns
        got = binding.mvue_orthogonalize(x[0].T.contiguous(), out_dtype=torch.float32, dev_status=status)
        assert off(got.T.contiguous(), x[0], 5) < 6e-3
    assert int(status) == 0
    torch.cuda.empty_cache()


def test_longer_rows_are_refused():
    L, size = binding.lib(), ctypes.c_size_t()
    for rows, cols, status in ((2, 2**20, 0), (2**20, 2, 0), (2**17, 2**20, 0), (2, 2**20 + 1, -3), (2, 2**21, -3), (2**29, 2, -3), (2, 2**31 - 256, -3), (2**17 + 1, 2**17 + 1, -3),
                               (2**40, 1, -3)):
        assert L.mvue_orthogonalize_workspace_bytes(1, rows, cols, ctypes.byref(size)) == status, (rows, cols)
        entry = (binding.MuonTensor * 1)(binding.MuonTensor(param=4096, grad=4096, momentum=4096, rows=rows, cols=cols))
        assert L.mvue_muon_workspace_bytes(entry, 1, ctypes.byref(size)) == status, (rows, cols)
        if status:
            fake = ctypes.c_void_p(4096)
            assert L.mvue_orthogonalize(fake, 0, 1, rows, cols, cols, rows * cols, 5, fake, 0, cols, rows * cols, fake, 1 << 60, None, None) == status
            config = binding.MuonConfig(lr=0.1, momentum=0.9, grad_scale=1.0, ns_steps=5)
            assert L.mvue_muon_step(entry, 1, config, fake, 1 << 60, None, None) == status
