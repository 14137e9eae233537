"""The training step that strings the operators together: its gradients without pruning noise against autograd in 64
bits, determinism, and that it learns."""
import pytest
import torch

from paper_2203_10991_b200 import training

pytestmark = pytest.mark.gpu


def reference(net, ids, target):
    """Loss and gradients of the same net in 64 bits (autograd), the activations unrounded."""
    tensors = [net.embedding, *net.weights, *(t for pair in net.norms for t in pair)]
    p = [t.double().requires_grad_() for t in tensors]
    emb, weights, norms = p[0], p[1:1 + len(net.weights)], p[1 + len(net.weights):]
    h = emb[ids] * net.scale
    for i, w in enumerate(weights):
        z = h @ w.T
        if i + 1 < len(weights):
            z = torch.nn.functional.group_norm(z.transpose(1, 2), net.groups, norms[2 * i], norms[2 * i + 1]).transpose(1, 2)
            h = torch.nn.functional.silu(z)
    loss = 0.5 * (z - target).square().mean()
    return loss, torch.autograd.grad(loss * target.numel(), p)


def test_mean_gradient_is_the_dense_one():
    # the pruned gradients are unbiased: their mean over seeds approaches autograd's as 1 / sqrt(seeds), down to the bf16
    # roundings of activations and gradients
    net = training.PrunedNet(300, [128, 256, 128], groups=4, seed=3)
    gen = torch.Generator().manual_seed(5)
    ids = torch.randint(0, 300, (2, 128), generator=gen).cuda()
    target = torch.randn(2, 128, 128, generator=gen).cuda()
    loss, want = reference(net, ids, target.double())
    pred, kept = net.forward(ids)
    diff = pred.float() - target
    loss = float(loss.detach())
    assert abs(float(0.5 * diff.square().mean()) - loss) < 1e-2 * loss
    means, errors = None, {}
    for k in range(1, 65):
        grads = [g.double().clone() for g in net.backward(ids, diff.to(torch.bfloat16), kept, 1000 + k)]
        means = grads if means is None else [m + g for m, g in zip(means, grads)]
        if k in (1, 64):
            errors[k] = [float((m / k - w).norm() / w.norm()) for m, w in zip(means, want)]
    for one, many in zip(errors[1], errors[64]):
        assert many < 0.3 * one or many < 0.02              # 1/8 by the law of large numbers, or the bf16 floor


@pytest.mark.parametrize("state_bits", [8, 32])
def test_it_learns_and_repeats(state_bits):
    def run():
        net = training.PrunedNet(200, [128, 256, 128], groups=8, state_bits=state_bits, seed=1)
        gen = torch.Generator().manual_seed(2)
        table = torch.randn(200, 128, generator=gen).cuda()
        losses = []
        for _ in range(60):
            ids = torch.randint(0, 200, (4, 128), generator=gen).cuda()
            losses.append(net.step(ids, table[ids], lr=3e-3))
        return net, torch.stack(losses)

    net, a = run()
    again, b = run()
    assert torch.equal(a, b)                                # bit for bit: no atomics, the seeds fix every draw
    assert all(torch.equal(x, y) for x, y in zip(net.weights, again.weights)) and torch.equal(net.embedding, again.embedding)
    assert bool(torch.isfinite(a).all()) and float(a[-5:].mean()) < 0.5 * float(a[:5].mean())


def test_the_command_runs():
    assert training.main(["--steps", "40"]) < 0.6
