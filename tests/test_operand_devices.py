"""Operands that are not on the current CUDA device are refused by the Python calls before anything is launched (the library
would read a host address on the GPU).  Nothing here launches a kernel; where both kinds of tensors are needed, the call
raises on the host."""
import pytest
import torch

from paper_2203_10991_b200 import binding


class On:
    """A tensor as far as the check looks at it."""
    dtype = torch.int32

    def __init__(self, device, contiguous=True, numel=1):
        self.device, self.contiguous, self.count = device, contiguous, numel

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def numel(self):
        return self.count


def test_the_check_itself(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    a, b, host, other = On(0), On(0), On(-1), On(1)
    binding._operands(a, b, None, workspace=b, dev_status=b)
    for args, kw in (((host, host), {}), ((a, host), {}), ((a, b, None, other), {}), ((other, other), {}), ((a,), {"workspace": host}),
                     ((a,), {"dev_status": host}), ((a,), {"workspace": On(0, contiguous=False)}), ((a,), {"dev_status": On(0, numel=0)})):
        with pytest.raises(ValueError):
            binding._operands(*args, **kw)
    wide = On(0)
    wide.dtype = torch.int64
    with pytest.raises(ValueError):
        binding._operands(a, dev_status=wide)


def test_calls_refuse_host_tensors():
    ids, w, dy = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8), torch.zeros(3, 8)
    x, stat = torch.zeros(2, 4, 8), torch.zeros(2, 2)
    for call in (lambda: binding.mvue_embedding(ids, w), lambda: binding.mvue_embedding_grad(ids, dy, 5),
                 lambda: binding.mvue_group_norm_act(x, 2), lambda: binding.mvue_group_norm_act_backward(x, x, stat, stat, 2)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_calls_refuse_one_host_tensor_among_device_ones():
    def variants(**tensors):
        """Every operand in turn on the host."""
        for name in tensors:
            yield {k: t.cpu() if k == name else t for k, t in tensors.items()}

    ids, w, dy = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    x, stat, c = torch.zeros(2, 4, 8, device="cuda"), torch.zeros(2, 2, device="cuda"), torch.zeros(8, device="cuda")
    status, ws = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    calls = [
        (binding.mvue_embedding, {}, dict(ids=ids, W=w, out=dy, dev_status=status)),
        (binding.mvue_embedding_grad, {"vocab": 5}, dict(ids=ids, dy=dy, out=w, workspace=ws, dev_status=status)),
        (binding.mvue_group_norm_act, {"groups": 2}, dict(x=x, weight=c, bias=c, out=x, workspace=ws, dev_status=status)),
        (binding.mvue_group_norm_act_backward, {"groups": 2}, dict(dy=x, x=x, mean=stat, rstd=stat, weight=c, bias=c, out=x, workspace=ws,
                                                                   dev_status=status)),
    ]
    for call, fixed, tensors in calls:
        for args in variants(**tensors):
            with pytest.raises(ValueError):
                call(**fixed, **args)
        call(**fixed, **tensors)                             # and with all of them in place it runs
    torch.cuda.synchronize()
    assert int(status) == 0
