"""The inner phase of a small mixture on one GPU, with 8-bit activations, followed by the outer
synchronisation (Algorithm 1: inner optimisation of every path on its own shard, then the outer loop).

Every module is a feed-forward block whose parameters lie flattened in the path copies that
``dipaco_outer_sync`` reads and writes, of one of three kinds:

    plain    x + W2 gelu(W1 norm(x)), one operator after another
    biased   x + W2 gelu(W1 norm(x) + b1) + b2, on linear layers that do the rest in their epilogue
    gated    s x + gate * norm(W2 gelu(W1 norm(x) + b1)): norms on both sides, a learned gate for every
             column, and the norm after one block done together with the one before the next

Between a block's forward and backward pass only packed matrices and the norms' statistics are kept: 10 bytes
per token and model width where bf16 activations would take 20 (gated: 11).

Run ``python -m paper_2403_10616_b200.inner_phase`` for a 2x2 mixture on synthetic shards; it prints the
paths' mean loss before every round.  ``--block`` picks the kind, ``--clip`` the most that the norm of a
path's gradients may be.
"""
from __future__ import annotations

import argparse
import math
from typing import List, NamedTuple, Optional

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


class BiasedWeights(NamedTuple):
    gamma: torch.Tensor
    beta: torch.Tensor
    up: torch.Tensor
    up_bias: torch.Tensor      # [4 width]
    down: torch.Tensor
    down_bias: torch.Tensor    # [width]


class GatedWeights(NamedTuple):
    gamma: torch.Tensor
    beta: torch.Tensor
    up: torch.Tensor
    up_bias: torch.Tensor
    down: torch.Tensor
    post_gamma: torch.Tensor   # [width], as the following
    post_beta: torch.Tensor
    gate: torch.Tensor


BLOCKS = {"plain": BlockWeights, "biased": BiasedWeights, "gated": GatedWeights}
RESIDUAL_SCALE = 0.9           # of gated blocks


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


def _shapes(width: int, kind: str):
    wide = WIDENING * width
    of = {"up": (wide, width), "up_bias": (wide,), "down": (width, wide)}
    return [of.get(name, (width,)) for name in BLOCKS[kind]._fields]


def block_numel(width: int, kind: str = "plain") -> int:
    return sum(math.prod(shape) for shape in _shapes(width, kind))


def block_weights(flat: torch.Tensor, width: int, kind: str = "plain"):
    """Views of a flattened module."""
    shapes = _shapes(width, kind)
    parts = flat.split([math.prod(shape) for shape in shapes])
    return BLOCKS[kind](*(part.view(shape) for part, shape in zip(parts, shapes)))


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


def biased_forward(x: torch.Tensor, w: BiasedWeights):
    """(x + W2 gelu(W1 norm(x) + b1) + b2, BlockSaved) for x [tokens, width] in bf16."""
    up, down = inner.pack(w.up), inner.pack(w.down)
    normed, kept, mean, rstd = inner.layer_norm_pack(x, w.gamma, w.beta)
    active, hidden = inner.packed_linear_pack(normed, up, w.up_bias, "gelu")
    out = inner.packed_linear(active, down, w.down_bias, None, x)
    return out, BlockSaved(kept, mean, rstd, normed, hidden, active, up, down)


def _feed_forward_backward(df: torch.Tensor, saved):
    """(gradient of the norm's result, of up, of up_bias, of down) of W2 gelu(W1 n + b1)."""
    df8 = inner.pack(df)
    d_down = inner.packed_matmul(df8, saved.active, transpose_a=True, out_dtype=torch.float32)
    d_hidden, d_up_bias = inner.packed_linear_pack_backward(df8, saved.down, saved.hidden, "gelu")
    d_up = inner.packed_matmul(d_hidden, saved.normed, transpose_a=True, out_dtype=torch.float32)
    return inner.packed_matmul(d_hidden, saved.up), d_up, d_up_bias, d_down


def biased_backward(dz: torch.Tensor, w: BiasedWeights, saved: BlockSaved):
    """(dx, gradients as BiasedWeights in fp32)."""
    d_normed, d_up, d_up_bias, d_down = _feed_forward_backward(dz, saved)
    dx, d_gamma, d_beta = inner.layer_norm_backward(d_normed, saved.x, saved.mean, saved.rstd, w.gamma)
    return dx.add_(dz), BiasedWeights(d_gamma, d_beta, d_up, d_up_bias, d_down, dz.sum(0, dtype=torch.float32))


class GatedSaved(NamedTuple):
    """What a gated block keeps; its stream is kept by the norm before the next block."""
    normed: inner.Packed
    hidden: inner.Packed
    active: inner.Packed
    up: inner.Packed
    down: inner.Packed
    f: inner.Packed                  # the feed-forward part's result, which the norm after it reads
    stream: Optional[inner.Packed]   # what the norm before the next block reads
    stats: torch.Tensor              # of both


def gated_forward(x: torch.Tensor, blocks: List[GatedWeights]):
    """(the last block's stream, what the backward pass needs) of x [tokens, width] in bf16 through gated blocks."""
    first = blocks[0]
    normed, kept, mean, rstd = inner.layer_norm_pack(x, first.gamma, first.beta)
    start, saved = (kept, mean, rstd), []
    for w, then in zip(blocks, blocks[1:] + [None]):
        up, down = inner.pack(w.up), inner.pack(w.down)
        active, hidden = inner.packed_linear_pack(normed, up, w.up_bias, "gelu")
        f = inner.packed_linear(active, down)
        after = (w.post_gamma, w.post_beta, w.gate, RESIDUAL_SCALE)
        own, stream = normed, None
        if then is None:
            x, _, stats = inner.residual_norm(x, f, None, None, *after, norm=False)
        else:
            x, normed, stream, stats = inner.residual_norm_pack(x, f, then.gamma, then.beta, *after)
        saved.append(GatedSaved(own, hidden, active, up, down, inner.pack(f), stream, stats))
    return x, (start, saved)


def gated_backward(dz: torch.Tensor, blocks: List[GatedWeights], kept):
    """(dx, gradients as GatedWeights in fp32, first block first)."""
    (x, mean, rstd), saved = kept
    found, dn, gamma = [], None, None
    for w, s in zip(reversed(blocks), reversed(saved)):
        g = inner.residual_norm_backward(dn, dz, s.f, s.stream, s.stats, gamma, w.post_gamma, w.post_beta, w.gate,
                                         RESIDUAL_SCALE)
        if found:  # those of the norm before the block after this one
            found[-1] = found[-1]._replace(gamma=g.gamma, beta=g.beta)
        dz, gamma = g.x, w.gamma
        dn, d_up, d_up_bias, d_down = _feed_forward_backward(g.f, s)
        found.append(GatedWeights(None, None, d_up, d_up_bias, d_down, g.post_gamma, g.post_beta, g.gate))
    dx, d_gamma, d_beta = inner.layer_norm_backward(dn, x, mean, rstd, gamma)
    found[-1] = found[-1]._replace(gamma=d_gamma, beta=d_beta)
    return dx.add_(dz), found[::-1]


def path_loss(copy: torch.Tensor, levels: int, width: int, x: torch.Tensor, target: torch.Tensor, grads=None,
              kind: str = "plain"):
    """Mean squared error of a path (one block per level) on a batch; with ``grads`` (a list) the blocks'
    gradients, first level first, are appended to it."""
    blocks = [block_weights(f, width, kind) for f in copy.view(levels, -1).unbind(0)]
    if kind == "gated":
        x, kept = gated_forward(x, blocks)
    else:
        forward, backward = (block_forward, block_backward) if kind == "plain" else (biased_forward, biased_backward)
        saved = []
        for w in blocks:
            x, s = forward(x, w)
            saved.append(s)
    error = x.float() - target.float()
    if grads is not None:
        dz = (error * (2.0 / error.numel())).to(torch.bfloat16)
        if kind == "gated":
            grads.extend(gated_backward(dz, blocks, kept)[1])
        else:
            found = []
            for w, s in zip(reversed(blocks), reversed(saved)):
                dz, g = backward(dz, w, s)
                found.append(g)
            grads.extend(reversed(found))
    return error.square().mean()


def inner_steps(copy: torch.Tensor, levels: int, width: int, x: torch.Tensor, target: torch.Tensor, steps: int,
                lr: float, beta: float = 0.9, kind: str = "plain", clip: Optional[float] = None) -> None:
    """Trains a path copy in place: `steps` of gradient descent with momentum, in fp32 between the steps, on gradients
    whose common norm is clipped to `clip`."""
    master, momentum = copy.float(), torch.zeros(copy.shape, device=copy.device)
    for _ in range(steps):
        grads: list = []
        path_loss(copy, levels, width, x, target, grads, kind)
        flat, _ = inner.gather_gradients([t for g in grads for t in g], clip, norm=False)
        momentum.mul_(beta).add_(flat)
        master.sub_(momentum, alpha=lr)
        copy.copy_(master)


class Mixture:
    """A grid of feed-forward modules, one copy per path in bf16, and the context that synchronises them."""

    def __init__(self, modules_per_level=(2, 2), width: int = 256, device="cuda:0", seed: int = 0, block: str = "plain"):
        self.levels, self.width, self.block = len(modules_per_level), width, block
        self.table = synth.path_table(modules_per_level)
        paths, numel = self.table.shape[0], block_numel(width, block)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.theta = torch.empty(sum(modules_per_level), numel, device=device)
        for module in self.theta:
            w = block_weights(module, width, block)
            module.zero_()
            w.gamma.fill_(1.0)
            if block == "gated":
                w.post_gamma.fill_(1.0)
                w.gate.fill_(0.3)
            w.up.normal_(0.0, width ** -0.5, generator=gen)
            w.down.normal_(0.0, 0.5 * (WIDENING * width) ** -0.5, generator=gen)
        self.momentum = torch.zeros_like(self.theta)
        self.copies = torch.empty(paths, self.levels * numel, device=device, dtype=torch.bfloat16)
        first = np.concatenate([[0], np.cumsum(modules_per_level)])
        for i in range(paths):
            self.copies[i] = torch.cat([self.theta[first[l] + self.table[i, l]] for l in range(self.levels)])
        self.sync = B.OuterSync(modules_per_level, [numel] * self.levels, self.table, path_dtype="bf16",
                                device=self.theta.device.index)

    def round(self, shards, steps: int, lr: float, clip: Optional[float] = None) -> None:
        """One round: every path trains on its shard (x, target), then the modules are synchronised."""
        for copy, (x, target) in zip(self.copies, shards):
            inner_steps(copy, self.levels, self.width, x, target, steps, lr, kind=self.block, clip=clip)
        self.sync.sync(self.theta, self.momentum, list(self.copies))

    def loss(self, shards) -> float:
        return sum(float(path_loss(c, self.levels, self.width, x, t, kind=self.block))
                   for c, (x, t) in zip(self.copies, shards)) / len(shards)

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
    ap.add_argument("--block", choices=sorted(BLOCKS), default="plain")
    ap.add_argument("--clip", type=float, default=None, help="the most that the norm of a path's gradients may be")
    args = ap.parse_args()
    mixture = Mixture(width=args.width, block=args.block)
    shards = make_shards(len(mixture.copies), args.tokens, args.width)
    for r in range(args.rounds):
        print("round %d: loss %.4f" % (r, mixture.loss(shards)))
        mixture.round(shards, args.steps, args.lr, args.clip)
    print("after %d rounds: loss %.4f" % (args.rounds, mixture.loss(shards)))
    if inner.inner_status() != B.DIPACO_OK or mixture.sync.status() != B.DIPACO_OK:
        raise RuntimeError("a kernel reported a failure")
    mixture.close()


if __name__ == "__main__":
    main()
