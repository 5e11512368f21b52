"""Blocks on linear layers with their epilogues and on the norms around a block, and paths of them, against their
formulas in 64 bits; steps of a path with clipped gradients."""
from __future__ import annotations

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner, inner_phase
from tests import inner_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def norm(v, gamma, beta):
    mean = v.mean(1, keepdim=True)
    return (v - mean) * torch.rsqrt((v - mean).square().mean(1, keepdim=True) + 1e-5) * gamma + beta


def exact_path(x, blocks, kind):
    for w in blocks:
        f = ref.gelu(norm(x, w.gamma, w.beta) @ w.up.t() + w.up_bias) @ w.down.t()
        if kind == "biased":
            x = x + f + w.down_bias
        else:
            x = inner_phase.RESIDUAL_SCALE * x + w.gate * norm(f, w.post_gamma, w.post_beta)
    return x


def random_blocks(levels, width, kind, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    flat = torch.empty(levels, inner_phase.block_numel(width, kind), device=DEV)
    for row in flat:
        row.normal_(0.0, 0.2, generator=gen)
        w = inner_phase.block_weights(row, width, kind)
        w.gamma.add_(1.0)
        w.up.normal_(0.0, width ** -0.5, generator=gen)
        w.down.normal_(0.0, (4 * width) ** -0.5, generator=gen)
        if kind == "gated":
            w.post_gamma.add_(1.0)
            w.gate.add_(0.5)
    return flat.to(torch.bfloat16), gen


@pytest.mark.parametrize("kind", ["biased", "gated"])
@pytest.mark.parametrize("levels,tokens,width", [(1, 300, 256), (2, 130, 96), (2, 500, 200), (3, 5, 64)])
def test_a_path_and_its_gradients_against_64_bits(kind, levels, tokens, width):
    """A value rounded to e4m3 is off by at most 2^-4 of itself, 2.6 % in the mean square.  A block's result passes through
    four roundings of operands that are independent of one another, a gradient through eight, and through as many in
    every further block: 0.026 * sqrt(8 levels) of the norm, 13 % for three blocks.  A half more is allowed."""
    flat, gen = random_blocks(levels, width, kind, 5)
    blocks = [inner_phase.block_weights(f, width, kind) for f in flat]
    x = torch.empty(tokens, width, device=DEV).normal_(0.0, 1.0, generator=gen).to(torch.bfloat16)
    target = torch.empty(tokens, width, device=DEV).normal_(0.0, 1.0, generator=gen).to(torch.bfloat16)
    grads = []
    loss = inner_phase.path_loss(flat.view(-1), levels, width, x, target, grads, kind)
    assert inner.inner_status() == B.DIPACO_OK
    exact = [type(w)(*(t.double().requires_grad_() for t in w)) for w in blocks]
    out = exact_path(x.double(), exact, kind)
    want = (out - target.double()).square().mean()
    want.backward()
    most = 1.5 * 0.026 * (8 * levels) ** 0.5
    assert abs(float(loss) - float(want.detach())) <= most * float(want.detach())
    assert len(grads) == levels
    for level, (g, w) in enumerate(zip(grads, exact)):
        for name, got, leaf in zip(g._fields, g, w):
            assert got.dtype == torch.float32 and got.shape == leaf.shape
            off = float((got.double() - leaf.grad).norm() / leaf.grad.norm())
            assert off <= most, (kind, level, name, off)


def test_a_step_takes_the_clipped_gradients():
    """The step is lr times the gradients, scaled to the norm that was asked for where theirs is larger."""
    width, levels = 96, 2
    flat, gen = random_blocks(levels, width, "gated", 7)
    x, target = (torch.empty(200, width, device=DEV).normal_(0.0, 1.0, generator=gen).to(torch.bfloat16) for _ in range(2))
    grads = []
    inner_phase.path_loss(flat.view(-1), levels, width, x, target, grads, "gated")
    flat_grad = torch.cat([t.reshape(-1) for g in grads for t in g]).double()
    norm_of_all = float(flat_grad.norm())
    for clip in (None, 2.0 * norm_of_all, 0.25 * norm_of_all):
        copy, lr = flat.view(-1).clone(), 0.5
        inner_phase.inner_steps(copy, levels, width, x, target, 1, lr, kind="gated", clip=clip)
        by = 1.0 if clip is None or clip > norm_of_all else 0.25
        want = flat.view(-1).double() - lr * by * flat_grad
        # rounded to bf16; the step itself in fp32 on gradients scaled in fp32
        assert bool(((copy.double() - want).abs() <= want.abs() * 2.0 ** -8 + 1e-6 * flat_grad.abs() + 1e-30).all())


@pytest.mark.parametrize("kind", ["biased", "gated"])
def test_a_mixture_of_such_blocks_trains_and_synchronises(kind):
    mixture = inner_phase.Mixture((1, 2), width=128, block=kind)
    shards = inner_phase.make_shards(2, 512, 128)
    for _ in range(2):
        mixture.round(shards, steps=3, lr=0.1, clip=1.0)
        shared = mixture.copies.view(2, 2, -1)[:, 0]
        assert torch.equal(shared[0], shared[1])
        assert torch.equal(shared[0], mixture.theta[0].to(torch.bfloat16))
        assert bool(torch.isfinite(mixture.copies).all())
    assert inner.inner_status() == B.DIPACO_OK and mixture.sync.status() == B.DIPACO_OK
    mixture.close()


def test_a_path_captured_and_replayed_follows_its_inputs():
    width, levels = 128, 2
    flat, gen = random_blocks(levels, width, "gated", 9)
    x, target = (torch.empty(256, width, device=DEV).normal_(0.0, 1.0, generator=gen).to(torch.bfloat16) for _ in range(2))

    def step():
        grads = []
        loss = inner_phase.path_loss(flat.view(-1), levels, width, x, target, grads, "gated")
        return (loss, *inner.gather_gradients([t for g in grads for t in g], 0.01))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (1, 2):
        x.normal_(0.0, 1.0, generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step()):
            assert torch.equal(a, b)
    assert inner.inner_status() == B.DIPACO_OK
