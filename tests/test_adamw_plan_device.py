"""The AdamW step goes to the device of its params, whichever is current: on the host, with the library call and the device
switch replaced."""
import contextlib

import pytest
import torch

from paper_2203_10991_b200 import binding, optim


@pytest.mark.parametrize("current,params", [(0, 0), (0, 1), (1, 0)])
def test_the_step_runs_on_the_params_device(monkeypatch, current, params):
    now, calls = [current], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], torch.device(d).index
        yield
        now[0] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(binding, "mvue_adamw_step", lambda tensors, count, config: calls.append(now[0]))
    plan = optim.AdamWPlan([], [], [])
    plan._device = torch.device("cuda", params)
    plan.step([], step=1, lr=1e-3)
    assert calls == [params] and now == [current]
