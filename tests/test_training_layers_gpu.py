"""The training step with layer norm, products of 8-bit codes and Muon: its gradients against autograd in 64 bits and against differences."""
import pytest
import torch

from paper_2203_10991_b200 import training
from tests.helpers import layer_ref

pytestmark = pytest.mark.gpu


def loss_of(net, tensors, ids, target):
    emb, weights, norms = tensors[0], tensors[1:1 + len(net.weights)], tensors[1 + len(net.weights):]
    h = emb[ids] * net.scale
    for i, w in enumerate(weights):
        z = h @ w.T
        if i + 1 < len(weights):
            h = torch.relu(torch.nn.functional.layer_norm(z, z.shape[-1:], norms[2 * i], norms[2 * i + 1]))
    return 0.5 * (z - target).square().mean()


def setup(products, seed=3):
    net = training.PrunedNet(300, [128, 256, 128], seed=seed, norm="layer", products=products, optimizer="muon")
    gen = torch.Generator().manual_seed(5)
    ids = torch.randint(0, 300, (2, 128), generator=gen).cuda()
    target = torch.randn(2, 128, 128, generator=gen).cuda()
    return net, ids, target


def formulas(net, ids, g, kept):
    """The backward pass in 64 bits from what the forward pass kept: its activations, its products' weights (the codes' values), its
    statistics.  A gradient that went through other activations says little: e4m3 moves a unit in a hundred across ReLU's edge."""
    d_weights, d_norms = [], []
    g = g.double()
    for i in reversed(range(len(net.weights))):
        h, norm, codes = kept[i]
        w = net.weights[i].double() if codes is None else layer_ref.dequantize(*codes, 128)
        d_weights.insert(0, g.reshape(-1, g.shape[-1]).T @ h.double().reshape(-1, h.shape[-1]))
        dh = g @ w
        if i > 0:
            z, mean, rstd = kept[i - 1][1]
            (g, dw, db), _ = layer_ref.layer_norm_backward(dh * (h > 0), z, mean, rstd, net.norms[i - 1][0])
            g = g.reshape(z.shape)
            d_norms = [dw, db, *d_norms]
    d_embedding = torch.zeros(net.embedding.shape, dtype=torch.float64, device="cuda").index_add_(0, ids.reshape(-1), dh.reshape(-1, dh.shape[-1])) * net.scale
    return [d_embedding, *d_weights, *d_norms]


@pytest.mark.parametrize("products", ["bf16", "e4m3"])
def test_mean_gradient_is_the_dense_one(products):
    net, ids, target = setup(products)
    tensors = [t.double().requires_grad_() for t in (net.embedding, *net.weights, *(t for pair in net.norms for t in pair))]
    loss = loss_of(net, tensors, ids, target.double())
    true = torch.autograd.grad(loss * target.numel(), tensors)
    pred, kept = net.forward(ids)
    diff = pred.float() - target
    # e4m3: both operands of three products off by 2^-5 on average in each element, 4 % of each product's size
    assert abs(float(0.5 * diff.square().mean()) - float(loss.detach())) < (2e-2 if products == "bf16" else 0.1) * float(loss.detach())
    want = formulas(net, ids, diff.to(torch.bfloat16), kept)
    means, errors = None, {}
    for k in range(1, 65):
        grads = [g.double().clone() for g in net.backward(ids, diff.to(torch.bfloat16), kept, 1000 + k)]
        means = grads if means is None else [m + g for m, g in zip(means, grads)]
        if k in (1, 64):
            errors[k] = [float((m / k - w).norm() / w.norm()) for m, w in zip(means, want)]
    # 1/8 of a single one's error by the law of large numbers, or the bf16 roundings of the gradients between the layers
    for one, many in zip(errors[1], errors[64]):
        assert many < 0.3 * one or many < 0.02, (errors[1], errors[64])
    if products == "bf16":                                                   # and autograd's agrees with the formulas
        for t, g in zip(true, want):
            assert float((t - g).norm()) < 0.1 * float(t.norm())             # (the bf16 forward pass moves ReLU's edge a little, too)
    # autograd's gradient against differences in 64 bits
    for t, g in zip(tensors, true):
        direction = torch.randn_like(t)
        h = 1e-6
        with torch.no_grad():
            up, down = (loss_of(net, [v + s * h * direction if v is t else v for v in tensors], ids, target.double()) for s in (1, -1))
        assert abs(float((up - down) / (2 * h) * target.numel()) - float((g * direction).sum())) < 1e-4 * float(g.norm() * direction.norm())


@pytest.mark.parametrize("products,norm,optimizer", [("e4m3", "layer", "muon"), ("bf16", "group", "muon"), ("e4m3", "group", "adamw")])
def test_it_runs_and_repeats(products, norm, optimizer):
    def run():
        net = training.PrunedNet(200, [128, 256, 128], groups=8, seed=1, norm=norm, products=products, optimizer=optimizer)
        gen = torch.Generator().manual_seed(2)
        table = torch.randn(200, 128, generator=gen).cuda()
        losses = []
        for _ in range(10):
            ids = torch.randint(0, 200, (4, 128), generator=gen).cuda()
            losses.append(net.step(ids, table[ids], lr=3e-3))
        return net, torch.stack(losses)

    net, a = run()
    again, b = run()
    assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    assert all(torch.equal(x, y) for x, y in zip(net.weights, again.weights)) and torch.equal(net.embedding, again.embedding)


def test_the_command_runs():
    assert training.main(["--steps", "5", "--norm", "layer", "--products", "e4m3", "--optimizer", "muon"]) > 0


def test_unknown_variants_are_refused():
    for kw in ({"norm": "batch"}, {"products": "fp4"}, {"optimizer": "sgd"}):
        with pytest.raises(ValueError):
            training.PrunedNet(10, [128, 128], **kw)
