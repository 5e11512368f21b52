"""The operators of the inner phase in 64 bits on the CPU, from their definitions (test infrastructure)."""
from __future__ import annotations

import math

import torch

BLOCK = 128
U = 2.0 ** -24  # unit round-off of fp32
ROOT = math.sqrt(2.0 / math.pi)
CUBIC = 0.044715


def e4m3_spacing(v):
    """Distance of neighbouring e4m3 values around v (three bits after the leading one, least 2^-9)."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)


def spread(per_block, rows, cols):
    return per_block.repeat_interleave(BLOCK, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def block_scales(x):
    """[ceil(R/128), ceil(C/128)] powers of two: the least 2^e >= 2^-126 with max|finite x| <= 448 * 2^e."""
    rows, cols = x.shape
    out = torch.ones(-(-rows // BLOCK), -(-cols // BLOCK), dtype=torch.float64)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            block = x[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            block = block[torch.isfinite(block)].abs()
            top = float(block.max()) if block.numel() else 0.0
            if top > 0:
                e = -126
                while top > math.ldexp(448.0, e):
                    e += 1
                out[i, j] = math.ldexp(1.0, e)
    return out


def pack(x):
    """(codes, scales) in float64; codes of infinities and NaN are NaN."""
    x = x.double()
    scales = block_scales(x)
    v = x / spread(scales, *x.shape)
    s = e4m3_spacing(torch.where(torch.isfinite(v), v, torch.zeros_like(v)))
    codes = torch.round(v / s) * s
    return torch.where(torch.isfinite(x), codes, torch.full_like(codes, math.nan)), scales


def values(codes, scales):
    """float64 values of codes and scales held in their 8-bit types."""
    return codes.cpu().double() * spread(scales.cpu().double(), *codes.shape)


def layer_norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt((x - mean[:, None]).square().mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    y = y if gamma is None else y * gamma.double()
    return (y if beta is None else y + beta.double()), mean, rstd


def layer_norm_backward(dy, x, mean, rstd, gamma):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x - mean) * rstd
    g = dy if gamma is None else dy * gamma.double()
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def gelu(a):
    a = a.double()
    return a / (1.0 + torch.exp(-2.0 * ROOT * (a + CUBIC * a ** 3)))


def gelu_slope(a):
    a = a.double()
    s = 1.0 / (1.0 + torch.exp(-2.0 * ROOT * (a + CUBIC * a ** 3)))
    return s + a * s * (1.0 - s) * 2.0 * ROOT * (1.0 + 3.0 * CUBIC * a ** 2)


def assert_packed_close(codes, scales, want, slack, what=""):
    """codes * scales is `want` rounded to e4m3: within half a spacing and `slack` (the fp32 error of
    the value before rounding, same shape), with the scale of the largest magnitude.  A block whose
    largest magnitude lies within that error of 448 * 2^e may take either scale."""
    got_scales, exact = scales.cpu().double(), block_scales(want)
    ratio = got_scales / exact
    for i, j in torch.nonzero(ratio != 1.0).tolist():
        at = (slice(i * BLOCK, (i + 1) * BLOCK), slice(j * BLOCK, (j + 1) * BLOCK))
        top, off = float(want[at].abs().max()), float(slack[at].max())
        edge = 448.0 * min(float(got_scales[i, j]), float(exact[i, j]))
        assert ratio[i, j] in (0.5, 2.0) and abs(top - edge) <= off, (what, i, j, float(ratio[i, j]))
    scale = spread(got_scales, *want.shape)
    got = codes.cpu().double() * scale
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), what
    half = 0.5 * e4m3_spacing(torch.where(fine, want, torch.zeros_like(want)) / scale) * scale
    err = (got - want).abs()
    bad = fine & (err > half * (1 + 1e-12) + slack)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[0].tolist(), float(err[bad].max()))
