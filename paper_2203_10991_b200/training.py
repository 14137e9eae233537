"""A training step in which every neural gradient is MVUE-pruned, from token ids to updated weights.

    python -m paper_2203_10991_b200.training [--steps 200] [--state-bits 8]

The net: scaled embedding, blocks of linear layer -> group norm + SiLU over the tokens of a sequence (channels last), a
linear read-out, mean squared error.  One step calls, in order,
    forward   mvue_embedding; per block a dense bf16 product (cuBLAS) and mvue_group_norm_act
    backward  per linear layer, top down: mvue_prune + mvue_sparse_update_gemm (dW), mvue_prune + mvue_sparse_backward_gemm
              (dh), mvue_group_norm_act_backward (the gradient that the layer below prunes); mvue_embedding_grad
    update    one AdamW call over all tensors (optim.AdamWPlan)
The demonstration learns a fixed random map of the tokens.
"""
from __future__ import annotations

import argparse

import torch

from . import binding, optim
from .chain import TC, layer_seeds


class PrunedNet:
    """Weights, optimiser and one step.  widths: channels of the embedding, the blocks and the read-out (multiples of 128);
    tokens of a batch a multiple of 128.  bf16 weights with fp32 copies; norm weights fp32; states in state_bits bits."""

    def __init__(self, vocab: int, widths, groups: int = 8, state_bits: int = 32, seed: int = 0, joint: int | None = None):
        gen = torch.Generator().manual_seed(seed)
        self.vocab, self.widths, self.groups, self.joint, self.seed = vocab, list(widths), groups, joint, seed
        self.scale = float(widths[0]) ** 0.5
        normal = lambda *shape, std: (std * torch.randn(shape, generator=gen)).to(torch.bfloat16).cuda()  # noqa: E731
        self.embedding = normal(vocab, widths[0], std=widths[0] ** -0.5)
        self.weights = [normal(o, i, std=i ** -0.5) for i, o in zip(widths[:-1], widths[1:])]
        self.norms = [(torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")) for c in widths[1:-1]]
        self.d_embedding = torch.empty(vocab, widths[0], device="cuda")
        self.d_weights = [torch.empty_like(w, dtype=torch.float32) for w in self.weights]
        params = [self.embedding, *self.weights, *(t for pair in self.norms for t in pair)]
        self.plan = optim.AdamWPlan.zeros(params, state_bits=state_bits, master=True)
        self.steps = 0

    def forward(self, ids: torch.Tensor):
        """(prediction, what the backward pass needs) for ids [n, s]."""
        h = binding.mvue_embedding(ids, self.embedding, scale=self.scale)
        kept = []
        for i, w in enumerate(self.weights):
            z = h @ w.T
            if i + 1 == len(self.weights):
                kept.append((h, None))
                return z, kept
            y, mean, rstd = binding.mvue_group_norm_act(z, self.groups, *self.norms[i], act="silu")
            kept.append((h, (z, mean, rstd)))
            h = y

    def backward(self, ids: torch.Tensor, g: torch.Tensor, kept, base_seed: int):
        """Gradients of all tensors, in the order of the plan, for the neural gradient g of the prediction."""
        n, s = ids.shape
        norm_grads = []
        for i in reversed(range(len(self.weights))):
            flat, s_upd_bwd = g.reshape(n * s, -1), layer_seeds(base_seed, i)
            values, meta = binding.mvue_prune(flat, 2, 4, 0, s_upd_bwd[0], layout=TC, joint=self.joint)
            binding.mvue_sparse_update_gemm(values, meta, kept[i][0].reshape(n * s, -1), out=self.d_weights[i])
            values, meta = binding.mvue_prune(flat, 2, 4, 1, s_upd_bwd[1], layout=TC, joint=self.joint)
            dh = binding.mvue_sparse_backward_gemm(values, meta, self.weights[i]).reshape(n, s, -1)
            if i > 0:
                z, mean, rstd = kept[i - 1][1]
                g, dweight, dbias = binding.mvue_group_norm_act_backward(dh, z, mean, rstd, self.groups, *self.norms[i - 1], act="silu")
                norm_grads = [dweight, dbias] + norm_grads
        binding.mvue_embedding_grad(ids, dh, self.vocab, scale=self.scale, out=self.d_embedding)
        return [self.d_embedding, *self.d_weights, *norm_grads]

    def step(self, ids: torch.Tensor, target: torch.Tensor, lr: float = 1e-3) -> torch.Tensor:
        """One training step on ids [n, s] and target [n, s, widths[-1]]; the loss before it (a device scalar)."""
        pred, kept = self.forward(ids)
        diff = pred.float() - target
        # the gradient is handed down multiplied by its element count, which AdamW's scale takes back: bf16 keeps its digits
        grads = self.backward(ids, diff.to(torch.bfloat16), kept, self.seed + self.steps)
        self.steps += 1
        self.plan.step(grads, step=self.steps, lr=lr, weight_decay=0.01, grad_scale=1.0 / diff.numel(), seed=self.seed + self.steps)
        return 0.5 * diff.square().mean()


def main(argv=None) -> float:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args(argv)
    vocab, n, s = 1000, 8, 256
    net = PrunedNet(vocab, [256, 512, 512, 128], state_bits=a.state_bits)
    gen = torch.Generator().manual_seed(1)
    table = torch.randn(vocab, 128, generator=gen).cuda()
    loss = 0.0
    for i in range(a.steps):
        ids = torch.randint(0, vocab, (n, s), generator=gen).cuda()
        value = net.step(ids, table[ids], lr=2e-3)
        if i % 20 == 0 or i + 1 == a.steps:
            loss = float(value)
            print(f"step {i:4d}  loss {loss:.4f}")
    return loss


if __name__ == "__main__":
    main()
