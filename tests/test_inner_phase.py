"""The feed-forward block of the inner phase, on packed activations, against its formula in 64 bits, and a
small mixture that trains and synchronises."""
from __future__ import annotations

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner, inner_phase
from tests import inner_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def exact_block(x, w):
    """The block in 64 bits, differentiable."""
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + 1e-5)
    n = (x - mean) * rstd * w.gamma + w.beta
    return x + ref.gelu(n @ w.up.t()) @ w.down.t()


@pytest.mark.parametrize("tokens,width", [(300, 256), (128, 96), (1000, 200)])
def test_block_and_its_gradient_against_64_bits(tokens, width):
    """A value rounded to e4m3 is off by at most 2^-4 of itself, 2.6 % in the mean square.  A result here
    passes through at most eight roundings of operands that are independent of one another, which adds up to
    0.026 * sqrt(8) = 7.4 % of its norm; 12 % is allowed."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    flat = torch.empty(inner_phase.block_numel(width), device=DEV)
    w = inner_phase.block_weights(flat, width)
    w.gamma.normal_(1.0, 0.2, generator=gen)
    w.beta.normal_(0.0, 0.2, generator=gen)
    w.up.normal_(0.0, width ** -0.5, generator=gen)
    w.down.normal_(0.0, (4 * width) ** -0.5, generator=gen)
    w = inner_phase.block_weights(flat.to(torch.bfloat16), width)
    x = torch.empty(tokens, width, device=DEV).normal_(0.0, 1.0, generator=gen).to(torch.bfloat16)
    dz = torch.empty(tokens, width, device=DEV).normal_(0.0, 1e-3, generator=gen).to(torch.bfloat16)
    z, saved = inner_phase.block_forward(x, w)
    dx, grads = inner_phase.block_backward(dz, w, saved)
    assert inner.inner_status() == B.DIPACO_OK

    exact = [t.double().requires_grad_() for t in (x, *w)]
    want = exact_block(exact[0], inner_phase.BlockWeights(*exact[1:]))
    want.backward(dz.double())
    # the residual stream itself is exact: what is compared is what the block adds to it
    assert_near(z.double() - x.double(), (want - exact[0]).detach(), "result")
    assert_near(dx.double() - dz.double(), exact[0].grad - dz.double(), "dx")
    for name, got, leaf in zip(grads._fields, grads, exact[1:]):
        assert got.dtype == torch.float32 and got.shape == leaf.shape
        assert_near(got.double(), leaf.grad, name)


def assert_near(got, want, what):
    off = float((got - want).norm() / want.norm())
    assert off <= 0.12, (what, off)


def test_a_mixture_trains_and_synchronises():
    mixture = inner_phase.Mixture((1, 2), width=128)
    shards = inner_phase.make_shards(2, 512, 128)
    first = mixture.loss(shards)
    for _ in range(3):
        mixture.round(shards, steps=6, lr=0.1)
        # both copies hold the same shared module again, and the module itself in bf16
        shared = mixture.copies.view(2, 2, -1)[:, 0]
        assert torch.equal(shared[0], shared[1])
        assert torch.equal(shared[0], mixture.theta[0].to(torch.bfloat16))
    assert inner.inner_status() == B.DIPACO_OK and mixture.sync.status() == B.DIPACO_OK
    assert mixture.loss(shards) < 0.9 * first
    mixture.close()
