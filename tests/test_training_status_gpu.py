"""The training step hands its status word to every call that takes one, and the command looks at it."""
import inspect

import pytest
import torch

from paper_2203_10991_b200 import binding, training

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm,products,optimizer", [("group", "bf16", "adamw"), ("layer", "e4m3", "muon")])
def test_every_call_has_it(norm, products, optimizer, monkeypatch):
    net = training.PrunedNet(200, [128, 256, 128], norm=norm, products=products, optimizer=optimizer)
    seen = set()

    def watched(owner, name):
        call = getattr(owner, name)
        if "dev_status" not in inspect.signature(call).parameters:
            return

        def with_status(*args, **kw):
            assert kw.get("dev_status") is net.dev_status, name
            seen.add(name)
            return call(*args, **kw)
        monkeypatch.setattr(owner, name, with_status)

    for name in dir(binding):
        if name.startswith("mvue_") and name != "mvue_muon_step":            # (the plan hands it on)
            watched(binding, name)
    if net.muon is not None:
        watched(net.muon, "step")
    ids = torch.randint(0, 200, (2, 128), device="cuda")
    loss = net.step(ids, torch.zeros(2, 128, 128, device="cuda"))
    assert bool(loss.isfinite()) and len(seen) == 6, seen
    net.check()


def test_check_raises():
    net = training.PrunedNet(50, [128, 128])
    ids = torch.zeros(1, 128, dtype=torch.int64, device="cuda")
    ids[0, 3] = 50                                                           # outside the vocabulary
    net.step(ids, torch.zeros(1, 128, 128, device="cuda"))
    with pytest.raises(binding.MvueError) as e:
        net.check()
    assert e.value.status == -13
    net.dev_status.fill_(-10)
    with pytest.raises(binding.MvueError) as e:
        net.check()
    assert e.value.status == -10


def test_the_command_raises(monkeypatch):
    forward = training.PrunedNet.forward

    def lost(self, ids):
        self.dev_status.fill_(-10)
        return forward(self, ids)
    monkeypatch.setattr(training.PrunedNet, "forward", lost)
    with pytest.raises(binding.MvueError):
        training.main(["--steps", "1"])
