"""The inner phase of a small mixture on one GPU, with 8-bit activations, followed by the outer
synchronisation (Algorithm 1: inner optimisation of every path on its own shard, then the outer loop).

Every module is a pre-norm feed-forward block, ``x + W2 gelu(W1 norm(x))``, whose parameters (gamma,
beta, W1, W2) lie flattened in the path copies that ``dipaco_outer_sync`` reads and writes.  Between a
block's forward and backward pass only packed matrices and the norm's statistics are kept: 10 bytes
per token and model width where bf16 activations would take 20.

Run ``python -m paper_2403_10616_b200.inner_phase`` for a 2x2 mixture on synthetic shards; it prints the
paths' mean loss before every round.
"""
from __future__ import annotations

import argparse
from typing import List, NamedTuple

import numpy as np
import torch

from . import binding as B
from . import inner, synth

WIDENING = 4  # hidden width over model width


class BlockWeights(NamedTuple):
    gamma: torch.Tensor   # [width]
    beta: torch.Tensor    # [width]
    up: torch.Tensor      # [4 width, width]
    down: torch.Tensor    # [width, 4 width]


class BlockSaved(NamedTuple):
    """What a block keeps for its backward pass."""
    x: inner.Packed       # the norm's input
    mean: torch.Tensor
    rstd: torch.Tensor
    normed: inner.Packed  # the norm's result, operand of W1 and of its gradient
    hidden: inner.Packed  # the GELU's input
    active: inner.Packed  # the GELU's result, operand of W2 and of its gradient
    up: inner.Packed
    down: inner.Packed


def block_numel(width: int) -> int:
    return 2 * width + 2 * WIDENING * width * width


def block_weights(flat: torch.Tensor, width: int) -> BlockWeights:
    """Views of a flattened module."""
    n = WIDENING * width * width
    gamma, beta, up, down = flat.split((width, width, n, n))
    return BlockWeights(gamma, beta, up.view(WIDENING * width, width), down.view(width, WIDENING * width))


def block_forward(x: torch.Tensor, w: BlockWeights):
    """(x + W2 gelu(W1 norm(x)), BlockSaved) for x [tokens, width] in bf16."""
    up, down = inner.pack(w.up), inner.pack(w.down)
    normed, kept, mean, rstd = inner.layer_norm_pack(x, w.gamma, w.beta)
    hidden = inner.packed_matmul(normed, up, transpose_b=True)
    active, hidden = inner.gelu_pack(hidden)
    out = inner.packed_matmul(active, down, transpose_b=True)
    return out.add_(x), BlockSaved(kept, mean, rstd, normed, hidden, active, up, down)


def block_backward(dz: torch.Tensor, w: BlockWeights, saved: BlockSaved):
    """(dx, gradients as BlockWeights in fp32) from the gradient of the block's result."""
    dz8 = inner.pack(dz)
    d_down = inner.packed_matmul(dz8, saved.active, transpose_a=True, out_dtype=torch.float32)
    d_hidden = inner.gelu_pack_backward(inner.packed_matmul(dz8, saved.down), saved.hidden)
    d_up = inner.packed_matmul(d_hidden, saved.normed, transpose_a=True, out_dtype=torch.float32)
    d_normed = inner.packed_matmul(d_hidden, saved.up)
    dx, d_gamma, d_beta = inner.layer_norm_backward(d_normed, saved.x, saved.mean, saved.rstd, w.gamma)
    return dx.add_(dz), BlockWeights(d_gamma, d_beta, d_up, d_down)


def path_loss(copy: torch.Tensor, levels: int, width: int, x: torch.Tensor, target: torch.Tensor, grads=None):
    """Mean squared error of a path (one block per level) on a batch; with ``grads`` (a list) the blocks'
    gradients, first level first, are appended to it."""
    blocks = [block_weights(f, width) for f in copy.view(levels, -1).unbind(0)]
    saved = []
    for w in blocks:
        x, s = block_forward(x, w)
        saved.append(s)
    error = x.float() - target.float()
    if grads is not None:
        dz = (error * (2.0 / error.numel())).to(torch.bfloat16)
        found = []
        for w, s in zip(reversed(blocks), reversed(saved)):
            dz, g = block_backward(dz, w, s)
            found.append(g)
        grads.extend(reversed(found))
    return error.square().mean()


def inner_steps(copy: torch.Tensor, levels: int, width: int, x: torch.Tensor, target: torch.Tensor, steps: int,
                lr: float, beta: float = 0.9) -> None:
    """Trains a path copy in place: `steps` of gradient descent with momentum, in fp32 between the steps."""
    master, momentum = copy.float(), torch.zeros(copy.shape, device=copy.device)
    for _ in range(steps):
        grads: List[BlockWeights] = []
        path_loss(copy, levels, width, x, target, grads)
        flat = torch.cat([t.reshape(-1) for g in grads for t in g])
        momentum.mul_(beta).add_(flat)
        master.sub_(momentum, alpha=lr)
        copy.copy_(master)


class Mixture:
    """A grid of feed-forward modules, one copy per path in bf16, and the context that synchronises them."""

    def __init__(self, modules_per_level=(2, 2), width: int = 256, device="cuda:0", seed: int = 0):
        self.levels, self.width = len(modules_per_level), width
        self.table = synth.path_table(modules_per_level)
        paths, numel = self.table.shape[0], block_numel(width)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.theta = torch.empty(sum(modules_per_level), numel, device=device)
        for module in self.theta:
            w = block_weights(module, width)
            w.gamma.fill_(1.0)
            w.beta.zero_()
            w.up.normal_(0.0, width ** -0.5, generator=gen)
            w.down.normal_(0.0, 0.5 * (WIDENING * width) ** -0.5, generator=gen)
        self.momentum = torch.zeros_like(self.theta)
        self.copies = torch.empty(paths, self.levels * numel, device=device, dtype=torch.bfloat16)
        first = np.concatenate([[0], np.cumsum(modules_per_level)])
        for i in range(paths):
            self.copies[i] = torch.cat([self.theta[first[l] + self.table[i, l]] for l in range(self.levels)])
        self.sync = B.OuterSync(modules_per_level, [numel] * self.levels, self.table, path_dtype="bf16",
                                device=self.theta.device.index)

    def round(self, shards, steps: int, lr: float) -> None:
        """One round: every path trains on its shard (x, target), then the modules are synchronised."""
        for copy, (x, target) in zip(self.copies, shards):
            inner_steps(copy, self.levels, self.width, x, target, steps, lr)
        self.sync.sync(self.theta, self.momentum, list(self.copies))

    def loss(self, shards) -> float:
        return sum(float(path_loss(c, self.levels, self.width, x, t)) for c, (x, t) in zip(self.copies, shards)) / len(shards)

    def close(self) -> None:
        self.sync.close()


def make_shards(paths: int, tokens: int, width: int, device="cuda:0", seed: int = 1):
    """A synthetic shard per path: inputs, and what one function of all shards and a path's own shift make of them."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    mix = torch.empty(width, width, device=device).normal_(0.0, width ** -0.5, generator=gen)
    shards = []
    for _ in range(paths):
        x = torch.empty(tokens, width, device=device).normal_(0.0, 1.0, generator=gen)
        shift = torch.empty(width, device=device).normal_(0.0, 0.3, generator=gen)
        shards.append((x.to(torch.bfloat16), (x + 0.5 * torch.tanh(x @ mix) + shift).to(torch.bfloat16)))
    return shards


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=2048, help="tokens of a path's shard")
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--steps", type=int, default=10, help="inner steps per round")
    ap.add_argument("--lr", type=float, default=0.2)
    args = ap.parse_args()
    mixture = Mixture(width=args.width)
    shards = make_shards(len(mixture.copies), args.tokens, args.width)
    for r in range(args.rounds):
        print("round %d: loss %.4f" % (r, mixture.loss(shards)))
        mixture.round(shards, args.steps, args.lr)
    print("after %d rounds: loss %.4f" % (args.rounds, mixture.loss(shards)))
    if inner.inner_status() != B.DIPACO_OK or mixture.sync.status() != B.DIPACO_OK:
        raise RuntimeError("a kernel reported a failure")
    mixture.close()


if __name__ == "__main__":
    main()
