"""The operators of the inner phase against plain 64-bit implementations, through the public calls.

Tolerances are bounds of the kernels' own rounding errors, with u = 2^-24 the unit round-off of fp32:
a sum that a kernel takes as chains of at most n additions, joined, is off by at most (n + 16) u times
the sum of magnitudes; chains are shorter than 96 at the sizes used here unless a test says otherwise.
A result in bf16 adds half a unit of its last place, a packed one half the spacing of its code.
"""
from __future__ import annotations

import concurrent.futures
import ctypes
import itertools
import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import build as libbuild
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref

DEV = "cuda:0"
U = ref.U
CHAIN = 112 * U          # chains of fewer than 96 additions, joined
F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def matrix(seed, rows, cols, dtype=F32, std=1.0, pad=0, offset=0):
    """A CPU matrix and its copy on the device inside a wider buffer, its first element `offset`
    elements from the start of an allocation, the rest of the buffer NaN."""
    x = torch.empty(rows, cols).normal_(0.0, std, generator=gen(seed)).to(dtype)
    return x, place(x, pad, offset)


def place(x, pad=0, offset=0):
    rows, cols = x.shape
    hold = torch.full((offset + rows * (cols + pad) + 16,), math.nan, dtype=x.dtype, device=DEV)
    view = hold[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def half(dtype, v):
    """Half a unit in the last place of `dtype` (8 or 24 significant bits) at magnitude v."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -126))) - (8 if dtype == BF16 else 24))


def assert_within(got, want, tol, what="", dtype=None):
    """|got - want| <= tol, and half a unit of dtype more where the result was rounded to it."""
    got = got.cpu().double()
    if dtype is not None:
        tol = tol + half(dtype, want.abs() + tol)
    err = (got - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[0].tolist(), float(err.max()))


SIZES = [(1, 1), (1, 896), (3, 8), (2, 16), (5, 17), (7, 100), (130, 64), (129, 127), (128, 128), (131, 129),
         (64, 257), (33, 896), (20, 1023), (9, 2048), (6, 2047), (4, 5000), (3, 8192), (2, 16384), (2, 20001), (1, 40000)]


# ------------------------------------------------------------------ packing

def packed_cases():
    for (rows, cols), dtype in itertools.product([(1, 1), (1, 896), (5, 17), (128, 128), (129, 257), (300, 391), (64, 2048)],
                                                 (F32, BF16)):
        yield rows, cols, dtype, 0, 0
    yield 200, 300, BF16, 4, 3
    yield 200, 300, BF16, 1, 1
    yield 200, 301, F32, 2, 1
    yield 130, 131, F32, 0, 3


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,pad,offset", list(packed_cases()))
def test_pack_rounds_every_value_and_picks_the_least_scale(rows, cols, dtype, pad, offset):
    size = torch.exp(3 * torch.randn(-(-rows // 128), -(-cols // 128), generator=gen(5)))
    x = (torch.randn(rows, cols, generator=gen(6)) * ref.spread(size, rows, cols)).to(dtype)
    p = inner.pack(place(x, pad, offset))
    codes, scales = ref.pack(x)
    assert torch.equal(p.scales.cpu().double(), scales)
    assert torch.equal(p.codes.cpu().double(), codes)
    # and back: a code times its scale is exact in either type
    for back in (F32, BF16):
        assert torch.equal(inner.unpack(p, back).cpu().double(), codes * ref.spread(scales, rows, cols))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pack_of_zeros_infinities_nan_and_extreme_magnitudes(dtype):
    x = torch.zeros(384, 640, dtype=dtype)
    x[:128, 128:256] = torch.randn(128, 128, generator=gen(1)).to(dtype)
    x[3, 130], x[4, 131], x[5, 132] = math.inf, -math.inf, math.nan
    x[:128, 256:384] = math.nan                                    # nothing finite
    x[:128, 384:512] = math.inf
    x[128:256, :128] = torch.finfo(dtype).max
    x[128:256, 128:256] = -torch.finfo(dtype).max
    x[128:256, 256:384] = 2.0 ** -133 if dtype == BF16 else 1e-45  # subnormal
    x[128:256, 384:512] = 448.0
    x[128:256, 512:] = torch.tensor(448.0) * (1 + 2.0 ** -7)       # just over
    x[256:, :128] = torch.logspace(-30, 30, 128, base=2.0).to(dtype)
    x[256:, 128:256] = -0.0
    p = inner.pack(place(x))
    codes, scales = ref.pack(x)
    assert torch.equal(p.scales.cpu().double(), scales)
    got = p.codes.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(codes))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(codes))


@pytest.mark.gpu
def test_every_code_and_scale_unpacks_to_its_value():
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).view(torch.float8_e4m3fn)
    for first in (0, 1, 120, 253):
        scales = torch.tensor([[first, first + 1], [first + 2, 127]], dtype=torch.uint8).view(torch.float8_e8m0fnu)
        want = (codes.double() * ref.spread(scales.double(), 256, 256))
        got = inner.unpack(inner.Packed(codes.to(DEV), scales.to(DEV)), F32).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got, posinf=-1.0), torch.nan_to_num(want.float(), posinf=-1.0))


@pytest.mark.gpu
def test_writers_stay_inside_a_slice_of_a_wider_packed_buffer():
    hold = torch.full((200, 320), 0x55, dtype=torch.uint8, device=DEV)
    codes = hold.view(torch.float8_e4m3fn)[:, 16:117]
    x, xd = matrix(3, 200, 101, BF16)
    p = inner.Packed(codes, torch.empty(2, 1, dtype=torch.float8_e8m0fnu, device=DEV))
    B.dipaco_pack(xd.data_ptr(), xd.stride(0), B.DIPACO_BF16, p.struct, 0, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(p.codes.cpu().double(), ref.pack(x)[0])
    assert bool((hold[:, :16] == 0x55).all()) and bool((hold[:, 117:] == 0x55).all())


# ------------------------------------------------------------------ layer norm

def norm_slack(x, gamma, beta, mean, rstd):
    """Bound of the fp32 error of y: mean and variance are off by CHAIN times the row's magnitudes."""
    big = x.double().abs().amax(1, keepdim=True) * rstd[:, None]
    g = 1.0 if gamma is None else gamma.double().abs()
    b = 0.0 if beta is None else beta.double().abs()
    hat = ((x.double() - mean[:, None]) * rstd[:, None]).abs()
    return CHAIN * ((hat + big) * g + b)


def norm_params(cols, dtype, which, seed=11):
    if which == "none":
        return None, None
    gamma = torch.empty(cols).normal_(1.0, 0.3, generator=gen(seed)).to(dtype)
    beta = torch.empty(cols).normal_(0.0, 0.3, generator=gen(seed + 1)).to(dtype)
    return gamma, (None if which == "gamma" else beta)


def on_device(t, offset=0):
    if t is None:
        return None
    hold = torch.empty(t.numel() + offset, dtype=t.dtype, device=DEV)
    hold[offset:].copy_(t)
    return hold[offset:]


def norm_cases():
    for i, (rows, cols) in enumerate(SIZES):
        for dtype in (F32, BF16):
            yield rows, cols, dtype, (F32, BF16)[i % 2], ("both", "gamma", "none")[i % 3], 0, 0
    yield 33, 896, BF16, BF16, "both", 8, 0
    yield 33, 896, BF16, F32, "both", 1, 1
    yield 33, 897, BF16, BF16, "both", 7, 8
    yield 17, 2047, F32, F32, "both", 1, 0
    yield 17, 2047, F32, BF16, "both", 2, 3
    yield 5000, 24, BF16, BF16, "both", 0, 0


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,pdtype,which,pad,offset", list(norm_cases()))
def test_layer_norm_and_its_gradient(rows, cols, dtype, pdtype, which, pad, offset):
    x, xd = matrix(rows * 7 + cols, rows, cols, dtype, 1.3, pad, offset)
    gamma, beta = norm_params(cols, pdtype, which)
    y, mean, rstd = inner.layer_norm(xd, on_device(gamma, offset), on_device(beta, offset), 1e-5, stats=True)
    wy, wmean, wrstd = ref.layer_norm(x, gamma, beta, 1e-5)
    assert_within(mean, wmean, CHAIN * x.double().abs().amax(1), "mean")
    if cols > 1:
        assert_within(rstd, wrstd, CHAIN * wrstd * (1 + wrstd * x.double().abs().amax(1)), "rstd")
        assert_within(y, wy, norm_slack(x, gamma, beta, wmean, wrstd), "y", dtype)
    assert torch.equal(y, inner.layer_norm(xd, on_device(gamma, offset), on_device(beta, offset), 1e-5))

    dy, dyd = matrix(rows + cols * 5, rows, cols, dtype, 1e-2, pad, offset)
    dx, dgamma, dbeta = inner.layer_norm_backward(dyd, xd, mean, rstd, on_device(gamma, offset))
    check_gradient(dx, dgamma, dbeta, dy, x, mean.cpu(), rstd.cpu(), gamma)
    # the same from the packed checkpoint of x
    p = inner.pack(xd)
    dx, dgamma, dbeta = inner.layer_norm_backward(dyd, p, mean, rstd, on_device(gamma, offset))
    check_gradient(dx, dgamma, dbeta, dy, ref.values(p.codes, p.scales), mean.cpu(), rstd.cpu(), gamma)


def check_gradient(dx, dgamma, dbeta, dy, x, mean, rstd, gamma):
    wx, wg, wb = ref.layer_norm_backward(dy, x, mean, rstd, gamma)
    r = rstd.double()[:, None]
    h = ((x.double() - mean.double()[:, None]) * r).abs()
    big = h + mean.double().abs()[:, None] * r       # h itself is off by a few u of its terms
    g = dy.double().abs() * (1.0 if gamma is None else gamma.double().abs())
    slack = CHAIN * r * (g + g.mean(1, keepdim=True) + big * (g * big).mean(1, keepdim=True))
    assert_within(dx, wx, slack, "dx", dx.dtype)
    rows = dy.shape[0]
    n = (rows + 112) * U if rows < 4096 else CHAIN * 2  # blocks share the rows: short chains, joined
    assert_within(dgamma, wg, n * (dy.double().abs() * big).sum(0), "dgamma")
    assert_within(dbeta, wb, n * dy.double().abs().sum(0), "dbeta")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_of_rows_with_a_large_mean_and_of_constant_rows(dtype):
    x = torch.randn(6, 1000, generator=gen(2))
    x[0] += 1000.0
    x[1] = 3.0
    x[2] = 0.0
    x[3] *= 1e-6
    x[4] *= 1e15
    x = x.to(dtype)
    y, mean, rstd = inner.layer_norm(place(x), eps=1e-5, stats=True)
    wy, wmean, wrstd = ref.layer_norm(x, None, None, 1e-5)
    assert_within(mean, wmean, CHAIN * x.double().abs().amax(1))
    # the centred values are off by the error of the mean: beside 1000 +- 1 that is CHAIN * 1000
    assert_within(y, wy, norm_slack(x, None, None, wmean, wrstd), "y", dtype)
    assert bool((y[1:3] == 0).all())


@pytest.mark.gpu
def test_a_bad_row_of_the_norm_harms_no_other():
    x, _ = matrix(1, 40, 896, BF16)
    clean = inner.layer_norm(place(x), stats=True)
    x[7, 3], x[9, 800], x[11] = math.nan, math.inf, -math.inf
    got = inner.layer_norm(place(x), stats=True)
    keep = [i for i in range(40) if i not in (7, 9, 11)]
    for a, b in zip(got, clean):
        assert torch.equal(a[keep], b[keep])
        assert bool(torch.isnan(got[0][[7, 9, 11]]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,which,pad,offset,keep", [
    (1, 896, BF16, "both", 0, 0, True), (129, 896, BF16, "both", 0, 0, True), (300, 130, F32, "gamma", 0, 0, True),
    (257, 2047, BF16, "both", 1, 3, True), (140, 257, F32, "none", 2, 1, False), (128, 2048, BF16, "both", 0, 0, False),
    (200, 1, F32, "both", 0, 0, True), (130, 20000, BF16, "both", 0, 0, True), (260, 5000, F32, "both", 0, 0, True)])
def test_layer_norm_packs_its_result_and_its_input(rows, cols, dtype, which, pad, offset, keep):
    x, xd = matrix(rows + cols, rows, cols, dtype, 2.0, pad, offset)
    gamma, beta = norm_params(cols, dtype, which)
    y, kept, mean, rstd = inner.layer_norm_pack(xd, on_device(gamma), on_device(beta), 1e-5, keep=keep)
    wy, wmean, wrstd = ref.layer_norm(x, gamma, beta, 1e-5)
    assert_within(mean, wmean, CHAIN * x.double().abs().amax(1))
    assert_within(rstd, wrstd, CHAIN * wrstd * (1 + wrstd * x.double().abs().amax(1)))
    ref.assert_packed_close(y.codes, y.scales, wy, norm_slack(x, gamma, beta, wmean, wrstd), "y")
    assert (kept is not None) == keep
    if keep:
        codes, scales = ref.pack(x)
        assert torch.equal(kept.scales.cpu().double(), scales)
        assert torch.equal(kept.codes.cpu().double(), codes)


@pytest.mark.gpu
def test_packed_norm_with_infinities_and_nan():
    x, _ = matrix(5, 256, 256, BF16)
    x[3, 7], x[200, 9] = math.inf, math.nan
    y, kept, mean, rstd = inner.layer_norm_pack(place(x))
    assert bool(torch.isnan(y.codes[3].float()).all()) and bool(torch.isnan(y.codes[200].float()).all())
    keep = [i for i in range(256) if i not in (3, 200)]
    wy = ref.layer_norm(x[keep], None, None, 1e-5)[0]
    got = (y.codes.cpu().double() * ref.spread(y.scales.cpu().double(), 256, 256))[keep]
    assert bool((got - wy).abs().max() <= 2.0 ** -4 * wy.abs().max())
    assert int(torch.isnan(kept.codes.float()).sum()) == 2
    assert torch.equal(kept.scales.cpu().double(), ref.block_scales(x.double()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [200, 128])
def test_packed_norm_scales_an_edge_with_infinities_by_what_is_inside(rows, dtype):
    # rows far from zero: a row of zeros beyond the last, normed like it, would be thousands
    x = (1000 + 4 * torch.randn(rows, 200, generator=gen(31))).to(dtype)
    gamma = torch.ones(200)
    gamma[3] = gamma[150] = math.inf
    y, _, mean, rstd = inner.layer_norm_pack(place(x), gamma.to(DEV))
    want = ref.layer_norm(x, gamma, None, 1e-5)[0]
    largest = torch.where(torch.isfinite(want), want, torch.zeros_like(want)).abs()
    blocks = torch.stack([torch.stack([largest[i:i + 128, j:j + 128].max() for j in (0, 128)]) for i in range(0, rows, 128)])
    # the largest finite value needs at least half of the codes' range, and fits in it up to its own rounding
    scales = y.scales.cpu().double()
    assert bool((blocks <= 448 * scales * (1 + 2.0 ** -10)).all()) and bool((blocks > 224 * scales * (1 - 2.0 ** -10)).all())


@pytest.mark.gpu
def test_norm_of_rows_without_values():
    x = torch.empty(5, 0, device=DEV)
    empty = torch.ones(1 << 12, device=DEV)  # what uninitialised statistics would be
    del empty
    for _, mean, rstd in (inner.layer_norm(x, stats=True), inner.layer_norm_pack(x)[1:]):
        assert bool(torch.isnan(mean).all()) and bool(torch.isnan(rstd).all())


@pytest.mark.gpu
def test_norm_gradient_against_differences():
    """<dx, v> and <dgamma, w> against central differences of the kernel's own forward pass in fp32."""
    rows, cols, eps = 12, 300, 1e-2
    x, xd = matrix(1, rows, cols, F32)
    gamma, beta = norm_params(cols, F32, "both")
    weight = torch.randn(rows, cols, generator=gen(4), dtype=torch.float64)
    v = torch.randn(rows, cols, generator=gen(5))
    w = torch.randn(cols, generator=gen(6))

    def loss(x, gamma, beta):
        return float((inner.layer_norm(x.to(DEV), gamma.to(DEV), beta.to(DEV)).cpu().double() * weight).sum())

    _, mean, rstd = inner.layer_norm(xd, gamma.to(DEV), beta.to(DEV), stats=True)
    dx, dgamma, dbeta = inner.layer_norm_backward(weight.float().to(DEV), xd, mean, rstd, gamma.to(DEV))
    # a central difference is off by eps^2/6 of the third derivative (here about 1 for each of
    # rows * cols terms of random sign) and by the forward pass's rounding over eps
    tol = (rows * cols) ** 0.5 * (eps ** 2 * 5 + 8 * U * 4 / eps)
    d = (loss(x + eps * v, gamma, beta) - loss(x - eps * v, gamma, beta)) / (2 * eps)
    assert abs(d - float((dx.cpu().double() * v.double()).sum())) <= tol
    d = (loss(x, gamma + eps * w, beta) - loss(x, gamma - eps * w, beta)) / (2 * eps)
    assert abs(d - float((dgamma.cpu().double() * w.double()).sum())) <= tol
    d = (loss(x, gamma, beta + eps * w) - loss(x, gamma, beta - eps * w)) / (2 * eps)
    assert abs(d - float((dbeta.cpu().double() * w.double()).sum())) <= tol


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [896, 20000])
def test_norm_gradient_of_no_rows_and_of_parts(cols):
    empty = torch.empty(0, cols, device=DEV)
    none = torch.empty(0, device=DEV)
    dx, dgamma, dbeta = inner.layer_norm_backward(empty, empty, none, none)
    assert dx.shape == (0, cols) and not bool(dgamma.any()) and not bool(dbeta.any())
    x, xd = matrix(2, 37, cols)
    _, mean, rstd = inner.layer_norm(xd, stats=True)
    dy, dyd = matrix(3, 37, cols)
    dx, dgamma, dbeta = inner.layer_norm_backward(dyd, xd, mean, rstd)
    need = B.dipaco_layer_norm_workspace(37, cols)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    for part in range(3):  # each output alone
        out = [torch.full_like(t, 7.0) if i == part else None for i, t in enumerate((dx, dgamma, dbeta))]
        ptr = [None if t is None else t.data_ptr() for t in out]
        B.dipaco_layer_norm_backward(dyd.data_ptr(), cols, xd.data_ptr(), cols, None, mean.data_ptr(),
                                     rstd.data_ptr(), None, ptr[0], cols, ptr[1], ptr[2], 37, cols, B.DIPACO_F32,
                                     B.DIPACO_F32, work.data_ptr(), need, 0, stream)
        assert torch.equal(out[part], (dx, dgamma, dbeta)[part])


# ------------------------------------------------------------------ GELU

def gelu_cases():
    for rows, cols in [(1, 1), (1, 896), (5, 17), (128, 128), (129, 257), (300, 391), (64, 2048)]:
        for dtype in (F32, BF16):
            yield rows, cols, dtype, 0, 0
    yield 200, 300, BF16, 4, 3
    yield 200, 301, F32, 2, 1


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,pad,offset", list(gelu_cases()))
def test_gelu_packs_its_result_and_its_gradient(rows, cols, dtype, pad, offset):
    x, xd = matrix(rows + cols, rows, cols, dtype, 2.5, pad, offset)
    y, kept = inner.gelu_pack(xd)
    want = ref.gelu(x)
    # s is off by a few u, and by the error of 2u times s (1 - s): |2u| (1 - s) s <= 0.3 s
    slack = 16 * U * want.abs() + 8 * U * x.double().abs() * (2.0 * x.double() ** 2 + 4).clamp(max=64.0) * \
        torch.exp(-x.double().abs())
    ref.assert_packed_close(y.codes, y.scales, want, slack, "gelu")
    codes, scales = ref.pack(x)
    assert torch.equal(kept.codes.cpu().double(), codes) and torch.equal(kept.scales.cpu().double(), scales)
    again, nothing = inner.gelu_pack(xd, keep=False)
    assert nothing is None and torch.equal(again.codes.float(), y.codes.float())

    dy, dyd = matrix(rows * 3 + cols, rows, cols, dtype, 1e-3, pad, offset)
    got = inner.gelu_pack_backward(dyd, kept)
    a = ref.values(kept.codes, kept.scales)
    want = dy.double() * ref.gelu_slope(a)
    slack = dy.double().abs() * U * (32 + 8 * (2 * a * a + 4).clamp(max=64.0) ** 2 * torch.exp(-a.abs()))
    ref.assert_packed_close(got.codes, got.scales, want, slack, "gradient")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gelu_of_extreme_values(dtype):
    top = float(torch.finfo(dtype).max)
    x = torch.tensor([[0.0, -0.0, 50.0, -50.0, 1e4, -1e4, 1e20, -1e20, top, -top, math.nan, math.inf, -math.inf, 1e-30]],
                     dtype=dtype)
    for i in range(x.shape[1]):  # each in a block of its own: the scale is that of the value
        y, kept = inner.gelu_pack(place(x[:, i:i + 1].contiguous()))
        v, got = float(x[0, i]), float(ref.values(y.codes, y.scales))
        if not math.isfinite(v):
            assert math.isnan(got) and math.isnan(float(ref.values(kept.codes, kept.scales)))
        elif v >= 50.0:
            assert abs(got - v) <= 2.0 ** -4 * v
        elif v <= -50.0 or v == 0.0:
            assert got == 0.0
        dy = torch.full((1, 1), 2.0, dtype=dtype, device=DEV)
        slope = float(ref.values(*(lambda p: (p.codes, p.scales))(inner.gelu_pack_backward(dy, kept))))
        if not math.isfinite(v):
            assert math.isnan(slope)
        else:
            want = 2.0 if v >= 50.0 else 0.0 if v <= -50.0 else 1.0
            assert slope == want


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gelu_of_values_far_below_zero_beside_others(dtype):
    """Large negative values, infinities and NaN share pairs, warps and blocks with ordinary ones."""
    x = torch.randn(256, 256, generator=gen(4)) * 2
    x[5, 10:20] = torch.tensor([-7.0, -8.0, -9.0, -9.9, -10.5, -20.0, -1e4, -1e30, -7.6, -7.7])
    x[130:140] = -9.0 - torch.rand(10, 256, generator=gen(5))
    x[200, ::2] = -30.0
    x = x.to(dtype)
    y, _ = inner.gelu_pack(place(x))
    want = ref.gelu(x)
    ref.assert_packed_close(y.codes, y.scales, want, 16 * U * want.abs() + 8 * U * x.double().abs() *
                            (2.0 * x.double() ** 2 + 4).clamp(max=64.0) * torch.exp(-x.double().abs()))
    clean = ref.values(y.codes, y.scales)
    x[5, 11], x[60, 3], x[61, 7] = math.nan, math.inf, -math.inf
    y, _ = inner.gelu_pack(place(x))
    got = ref.values(y.codes, y.scales)
    assert int(torch.isnan(got).sum()) == 3
    assert torch.equal(torch.nan_to_num(got)[~torch.isnan(got)], clean[~torch.isnan(got)])


@pytest.mark.gpu
def test_gelu_gradient_against_differences():
    """dy * gelu' from the checkpoint against central differences of the 64-bit GELU at its values."""
    x, xd = matrix(8, 256, 128, F32, 2.0)
    kept = inner.gelu_pack(xd)[1]
    dy = torch.ones(256, 128, device=DEV)
    got = inner.gelu_pack_backward(dy, kept)
    a, eps = ref.values(kept.codes, kept.scales), 1e-5
    want = (ref.gelu(a + eps) - ref.gelu(a - eps)) / (2 * eps)   # off by eps^2/6 * gelu''' < 1e-10
    ref.assert_packed_close(got.codes, got.scales, want, torch.full_like(want, 64 * U + 1e-9))


# ------------------------------------------------------------------ products

FORMS = {"forward": (False, True), "input": (False, False), "weight": (True, False), "both": (True, True)}


def packed_operand(seed, rows, cols, std=1.0):
    """Packed values whose blocks differ in size; returns (Packed, float64 values)."""
    size = torch.exp(torch.randn(-(-rows // 128), -(-cols // 128), generator=gen(seed + 1)))
    x = torch.randn(rows, cols, generator=gen(seed)) * std * ref.spread(size, rows, cols)
    codes, scales = ref.pack(x)
    hold = torch.full((rows, -(-cols // 16) * 16 + 16), 0x7F, dtype=torch.uint8, device=DEV)  # NaN around it
    hold = hold.view(torch.float8_e4m3fn)[:, :cols]
    hold.copy_(codes.to(torch.float8_e4m3fn))
    p = inner.Packed(hold, scales.to(torch.float8_e8m0fnu).to(DEV))
    return p, codes * ref.spread(scales, rows, cols)


def product_tolerance(a, b, k):
    """The tensor cores add 32 products at a time to an fp32 sum and may truncate: each of k/32 + 2
    additions is off by at most 2^-22 of the magnitudes summed so far."""
    return (k / 32 + 2) * 2.0 ** -22 * (a.abs() @ b.abs())


PRODUCT_SIZES = [(1, 1, 1), (1, 896, 896), (1, 130, 4000), (2, 300, 65), (5, 64, 31), (16, 257, 300), (17, 128, 129),
                 (33, 500, 1000), (128, 128, 128), (129, 127, 257), (200, 300, 400), (255, 513, 96), (384, 640, 1024),
                 (1000, 130, 2100)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("m,n,k", PRODUCT_SIZES)
def test_product_of_packed_matrices(m, n, k, form):
    ta, tb = FORMS[form]
    a, av = packed_operand(m + 3 * n, *((k, m) if ta else (m, k)))
    b, bv = packed_operand(n + 7 * k, *((n, k) if tb else (k, n)), std=0.02)
    av, bv = (av.t() if ta else av), (bv.t() if tb else bv)
    want = av @ bv
    for dtype in (F32, BF16):
        got = inner.packed_matmul(a, b, ta, tb, dtype)
        assert inner.inner_status() == B.DIPACO_OK
        assert_within(got, want, product_tolerance(av, bv, k), str(dtype), dtype)
        # into a slice of a wider buffer at odd offsets, and added to what is there
        hold = torch.full((m, n + 5), 3.0, dtype=dtype, device=DEV)
        out = hold[:, 3:3 + n]
        inner.packed_matmul(a, b, ta, tb, out=out)
        assert torch.equal(out, got)
        before = torch.randn(m, n, generator=gen(9)).to(dtype)
        out.copy_(before)
        inner.packed_matmul(a, b, ta, tb, out=out, accumulate=True)
        total = want + before.double()
        assert_within(out, total, product_tolerance(av, bv, k) + U * total.abs(), "accumulated", dtype)
        assert bool((hold[:, :3] == 3.0).all()) and bool((hold[:, 3 + n:] == 3.0).all())


def random_packed_on_device(seed, rows, cols, std=1.0):
    """(Packed, float64 values on the device) of normal values whose blocks differ in size."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    size = torch.empty(-(-rows // 128), -(-cols // 128), device=DEV).normal_(0.0, 1.0, generator=g).exp()
    x = torch.empty(rows, cols, device=DEV).normal_(0.0, std, generator=g) * ref.spread(size, rows, cols)
    p = inner.pack(x)
    return p, p.codes.double() * ref.spread(p.scales.double(), rows, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("m,n,k", [(2000, 1792, 900), (4100, 2048, 512), (600, 1000, 9000), (3000, 5000, 700),
                                   (300, 70, 20000), (70, 9000, 1500), (65, 4096, 4096), (20000, 900, 128),
                                   (10000, 2300, 3584), (64, 5000, 4100), (8000, 20, 2500)])
def test_product_of_larger_packed_matrices(m, n, k, form):
    """Several tiles per block, ragged last tiles, contractions shared between blocks."""
    ta, tb = FORMS[form]
    a, av = random_packed_on_device(m + n, *((k, m) if ta else (m, k)))
    b, bv = random_packed_on_device(n + k, *((n, k) if tb else (k, n)), std=0.02)
    av, bv = (av.t() if ta else av), (bv.t() if tb else bv)
    want = av @ bv
    for dtype in (F32, BF16):
        got = inner.packed_matmul(a, b, ta, tb, dtype)
        assert inner.inner_status() == B.DIPACO_OK
        tol = product_tolerance(av, bv, k)
        err, tol = (got.double() - want).abs(), tol + half(dtype, want.abs() + tol)
        assert bool((err <= tol).all()), (dtype, float((err / tol).max()))
        assert torch.equal(got, inner.packed_matmul(a, b, ta, tb, dtype))
        out = torch.full((m, n + 3), 1.0, dtype=dtype, device=DEV)[:, 1:n + 1]
        inner.packed_matmul(a, b, ta, tb, out=out, accumulate=True)
        total = want + 1.0
        err = (out.double() - total).abs()
        tol = product_tolerance(av, bv, k) + U * total.abs()
        assert bool((err <= tol + half(dtype, total.abs() + tol)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(300, 400), (40, 50)])
def test_long_sums_in_fp32_do_not_drift(m, n):
    """2048 values at a time on the tensor cores, 64 additions each off by at most 2^-24 of the sum on
    average over truncation, the parts added in fp32: the norm of the error stays under
    (64 + parts) * 2^-24 of the result's."""
    k = 40000
    a, av = random_packed_on_device(1, k, m)
    b, bv = random_packed_on_device(2, k, n)
    want = av.t() @ bv
    got = inner.packed_matmul(a, b, transpose_a=True, out_dtype=F32)
    assert float((got.double() - want).norm() / want.norm()) <= (64 + k / 2048) * U


@pytest.mark.gpu
@pytest.mark.parametrize("form", sorted(FORMS))
def test_products_are_exact_for_small_whole_numbers(form):
    """Whole codes and scales of one: sums below 2^24 have no rounding at all."""
    ta, tb = FORMS[form]
    m, n, k = 300, 270, 520
    a = torch.randint(-8, 9, (k, m) if ta else (m, k), generator=gen(1)).double()
    b = torch.randint(-8, 9, (n, k) if tb else (k, n), generator=gen(2)).double()

    def hold(x):
        scales = torch.ones(-(-x.shape[0] // 128), -(-x.shape[1] // 128)).to(torch.float8_e8m0fnu)
        wide = torch.zeros(x.shape[0], -(-x.shape[1] // 16) * 16, device=DEV, dtype=torch.float8_e4m3fn)
        wide[:, :x.shape[1]].copy_(x.to(torch.float8_e4m3fn))
        return inner.Packed(wide[:, :x.shape[1]], scales.to(DEV))

    got = inner.packed_matmul(hold(a), hold(b), ta, tb, F32)
    assert torch.equal(got.cpu().double(), (a.t() if ta else a) @ (b.t() if tb else b))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 40, 200])
def test_product_passes_nan_to_its_rows_and_columns_alone(m):
    n, k = 300, 260
    a, av = packed_operand(1, m, k)
    b, bv = packed_operand(2, n, k)
    a.codes.view(torch.uint8)[m - 1, 255] = 0x7F
    b.codes.view(torch.uint8)[131, 3] = 0xFF
    got = inner.packed_matmul(a, b, transpose_b=True, out_dtype=F32).cpu()
    bad = torch.zeros(m, n, dtype=torch.bool)
    bad[m - 1], bad[:, 131] = True, True
    assert torch.equal(torch.isnan(got), bad)
    want = av @ bv.t()
    tol = product_tolerance(av, bv.t(), k)
    assert bool(((got.double() - want).abs() <= tol)[~bad].all())


@pytest.mark.gpu
def test_product_of_extreme_scales():
    """Scales near both ends of their range meet: their product stays a normal number."""
    a, av = packed_operand(1, 130, 140)
    b, bv = packed_operand(2, 150, 140)
    for shift in (100, -100):
        sa = a.scales.float() * 2.0 ** shift
        sb = b.scales.float() * 2.0 ** -shift
        pa = inner.Packed(a.codes, sa.to(torch.float8_e8m0fnu))
        pb = inner.Packed(b.codes, sb.to(torch.float8_e8m0fnu))
        got = inner.packed_matmul(pa, pb, transpose_b=True, out_dtype=F32)
        want = av @ bv.t()
        assert_within(got, want, product_tolerance(av, bv.t(), 140))


@pytest.mark.gpu
def test_products_over_nothing():
    dev = torch.device(DEV)
    a, b = inner.Packed.empty(5, 0, dev), inner.Packed.empty(7, 0, dev)
    out = torch.full((5, 7), 2.0, device=DEV)
    inner.packed_matmul(a, b, transpose_b=True, out=out, accumulate=True)
    assert bool((out == 2.0).all())
    inner.packed_matmul(a, b, transpose_b=True, out=out)
    assert not bool(out.any())
    assert inner.packed_matmul(inner.Packed.empty(0, 9, dev), inner.Packed.empty(9, 4, dev)).shape == (0, 4)
    for fn in (inner.pack, inner.layer_norm, lambda x: inner.gelu_pack(x)[0]):
        for shape in ((0, 5), (5, 0)):
            assert tuple(fn(torch.empty(shape, device=DEV)).shape) == shape


# ------------------------------------------------------------------ streams, repeats, graphs

@pytest.mark.gpu
def test_threads_that_launch_different_sizes_do_not_disturb_one_another():
    # sizes that need different amounts of shared memory of one kernel
    def work(i, cols):
        rows = torch.ones(2, cols, device=DEV)
        tokens, weight = inner.pack(rows), inner.pack(torch.ones(4, cols, device=DEV))
        stat = torch.zeros(2, device=DEV)
        for _ in range(300):
            results[i].append((inner.layer_norm(rows), inner.packed_matmul(tokens, weight, transpose_b=True, out_dtype=F32),
                               inner.layer_norm_backward(rows, rows, stat, stat)[2]))
        torch.cuda.synchronize()

    sizes, results = [7000, 16000, 8000, 15000], [[], [], [], []]
    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        for done in [pool.submit(work, i, cols) for i, cols in enumerate(sizes)]:
            done.result()
    for cols, got in zip(sizes, results):
        for y, product, dbeta in got[::30]:
            assert bool((y == 0).all()) and bool((product == cols).all()) and bool((dbeta == 2).all())


@pytest.mark.gpu
def test_operators_follow_the_current_stream_and_repeat_bitwise():
    x, xd = matrix(1, 500, 896, BF16)
    gamma, beta = (t.to(DEV) for t in norm_params(896, BF16, "both"))
    w = inner.pack(torch.randn(640, 896, generator=gen(3)).to(DEV))

    def step():
        n, kept, mean, rstd = inner.layer_norm_pack(xd, gamma, beta)
        a = inner.packed_matmul(n, w, transpose_b=True)
        h, akept = inner.gelu_pack(a)
        da = inner.gelu_pack_backward(a, akept)
        dn = inner.packed_matmul(da, w)
        dw = inner.packed_matmul(da, n, transpose_a=True, out_dtype=F32)
        return (dw, h.codes.float(), *inner.layer_norm_backward(dn, kept, mean, rstd, gamma))

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(first, other):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(first, captured):
        assert torch.equal(p, q)


# ------------------------------------------------------------------ refusals (no GPU needed)

@pytest.fixture(scope="module")
def library():
    libbuild.build()
    return B.load()


def refused(status, fn, *args):
    with pytest.raises(B.DipacoError) as e:
        fn(*args)
    assert e.value.status == status


def struct(rows=4, cols=4, stride=16, codes=4096, scales=4096):
    return B.PackedStruct(codes, scales, rows, cols, stride)


NORM = dict(x=4096, x_stride=8, gamma=4096, beta=4096, y=8192, y_stride=8, mean=4096, rstd=4096, rows=4, cols=8,
            eps=1e-5, dtype=0, param_dtype=0, device=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), B.DIPACO_EINVAL), (dict(x=4098), B.DIPACO_EINVAL), (dict(x_stride=7), B.DIPACO_EINVAL),
    (dict(y=None, mean=None, rstd=None), B.DIPACO_EINVAL), (dict(y=8193), B.DIPACO_EINVAL),
    (dict(y_stride=-8), B.DIPACO_EINVAL), (dict(gamma=4097), B.DIPACO_EINVAL), (dict(beta=4098), B.DIPACO_EINVAL),
    (dict(mean=4097), B.DIPACO_EINVAL), (dict(rows=-1), B.DIPACO_EINVAL), (dict(cols=-1), B.DIPACO_EINVAL),
    (dict(eps=-1.0), B.DIPACO_EINVAL), (dict(eps=math.nan), B.DIPACO_EINVAL), (dict(eps=math.inf), B.DIPACO_EINVAL),
    (dict(dtype=2), B.DIPACO_EINVAL), (dict(param_dtype=-1), B.DIPACO_EINVAL), (dict(device=-1), B.DIPACO_EINVAL),
    (dict(rows=2 ** 31), B.DIPACO_ELIMIT), (dict(cols=2 ** 40, x_stride=2 ** 41, y_stride=2 ** 41), B.DIPACO_ELIMIT)])
def test_layer_norm_refuses(library, change, status):
    refused(status, B.dipaco_layer_norm, *{**NORM, **change}.values())


BACK = dict(dy=4096, dy_stride=8, x=4096, x_stride=8, x_packed=None, mean=4096, rstd=4096, gamma=None, dx=8192,
            dx_stride=8, dgamma=4096, dbeta=4096, rows=4, cols=8, dtype=0, param_dtype=0, workspace=4096,
            workspace_bytes=1 << 20, device=0, stream=None)


@pytest.mark.parametrize("change", [
    dict(dy=None), dict(dy=4097), dict(x=None), dict(x_packed=struct(4, 8)), dict(x=None, x_packed=struct(4, 9)),
    dict(x=None, x_packed=struct(4, 8, 15)), dict(x=None, x_packed=struct(4, 8, 16, 4100)),
    dict(x=None, x_packed=struct(4, 8, 16, 4096, 0)), dict(mean=None), dict(rstd=None), dict(mean=4098),
    dict(dx=None, dgamma=None, dbeta=None), dict(dgamma=4097), dict(dbeta=2), dict(gamma=4098), dict(dx_stride=3),
    dict(dtype=7), dict(param_dtype=7), dict(device=-2), dict(rows=-4), dict(rows=5000, workspace=None),
    dict(rows=5000, workspace_bytes=64), dict(rows=5000, workspace=4100)])
def test_layer_norm_backward_refuses(library, change):
    refused(B.DIPACO_EINVAL, B.dipaco_layer_norm_backward, *{**BACK, **change}.values())


@pytest.mark.parametrize("change", [
    dict(a=None), dict(b=None), dict(b=struct(8, 5)), dict(a=struct(4, 4, 24)), dict(a=struct(4, 4, 16, 0)),
    dict(b=struct(8, 4, 16, 4104)), dict(b=struct(8, 4, 16, 4096, 0)), dict(c=None), dict(c=4098), dict(c_stride=7),
    dict(dtype=3), dict(device=-1), dict(transpose_b=0)])
def test_packed_matmul_refuses(library, change):
    good = dict(a=struct(4, 4), b=struct(8, 4), transpose_a=0, transpose_b=1, c=4096, c_stride=8, dtype=0,
                accumulate=0, workspace=None, workspace_bytes=0, device=0, stream=None)
    refused(B.DIPACO_EINVAL, B.dipaco_packed_matmul, *{**good, **change}.values())


def test_packing_entry_points_refuse(library):
    for bad in (struct(-1), struct(4, 4, 8), struct(codes=4097), struct(scales=0), None):
        refused(B.DIPACO_EINVAL, B.dipaco_pack, 4096, 4, 0, bad, 0, None)
        refused(B.DIPACO_EINVAL, B.dipaco_unpack, bad, 4096, 4, 0, 0, None)
        refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack, 4096, 4, 0, bad, None, 0, None)
        refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack_backward, 4096, 4, 0, bad, struct(), 0, None)
        refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack_backward, 4096, 4, 0, struct(), bad, 0, None)
        refused(B.DIPACO_EINVAL, B.dipaco_layer_norm_pack, 4096, 4, None, None, bad, None, 4096, 4096, 1e-5, 0, 0, 0, None)
    for x, stride, dtype, device in ((None, 4, 0, 0), (4097, 4, 1, 0), (4096, 3, 0, 0), (4096, 4, 2, 0), (4096, 4, 0, -1)):
        refused(B.DIPACO_EINVAL, B.dipaco_pack, x, stride, dtype, struct(), device, None)
        refused(B.DIPACO_EINVAL, B.dipaco_unpack, struct(), x, stride, dtype, device, None)
        refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack, x, stride, dtype, struct(), None, device, None)
        refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack_backward, x, stride, dtype, struct(), struct(), device, None)
    refused(B.DIPACO_EINVAL, B.dipaco_gelu_pack, 4096, 4, 0, struct(), struct(5), 0, None)
    refused(B.DIPACO_EINVAL, B.dipaco_layer_norm_pack, 4096, 4, None, None, struct(), None, None, 4096, 1e-5, 0, 0, 0, None)
    refused(B.DIPACO_ELIMIT, B.dipaco_pack, 4096, 2 ** 33, 0, struct(4, 2 ** 32, 2 ** 33), 0, None)


def test_workspace_queries(library):
    assert B.dipaco_layer_norm_workspace(0, 896) == 0 and B.dipaco_layer_norm_workspace(1, 896) == 0
    assert B.dipaco_layer_norm_workspace(50000, 896) >= 2 * 896 * 4
    assert B.dipaco_packed_matmul_workspace(1, 1, 0) >= 0
    refused(B.DIPACO_EINVAL, B.dipaco_layer_norm_workspace, -1, 4)
    refused(B.DIPACO_EINVAL, B.dipaco_packed_matmul_workspace, 4, 4, -1)
    refused(B.DIPACO_ELIMIT, B.dipaco_packed_matmul_workspace, 2 ** 32, 4, 4)


def test_tensor_level_calls_refuse_cpu_tensors_and_wrong_types(library):
    x = torch.zeros(4, 8)
    for fn in (inner.pack, inner.layer_norm, inner.layer_norm_pack, inner.gelu_pack):
        with pytest.raises(ValueError):
            fn(x)
    with pytest.raises(ValueError):
        inner.Packed(torch.zeros(4, 16), torch.ones(1, 1))
    with pytest.raises(ValueError):
        inner.Packed(x.to(torch.float8_e4m3fn), torch.ones(2, 1).to(torch.float8_e8m0fnu))


@pytest.mark.gpu
def test_tensor_level_calls_refuse_shapes_that_do_not_fit():
    x = torch.zeros(4, 8, device=DEV)
    p, q = inner.pack(x), inner.pack(torch.zeros(8, 4, device=DEV))
    stat = torch.zeros(4, device=DEV)
    for fn in (lambda: inner.layer_norm(x.half()), lambda: inner.layer_norm(x.t()), lambda: inner.layer_norm(x[0]),
               lambda: inner.layer_norm(x, stat), lambda: inner.layer_norm(x, torch.ones(8, device=DEV), torch.ones(8, device=DEV).bfloat16()),
               lambda: inner.layer_norm_backward(x, q, stat, stat), lambda: inner.layer_norm_backward(x, p, stat[:3], stat),
               lambda: inner.layer_norm_backward(x, x.bfloat16(), stat, stat), lambda: inner.gelu_pack_backward(x, q),
               lambda: inner.packed_matmul(p, p), lambda: inner.packed_matmul(p, q, out_dtype=torch.float16),
               lambda: inner.packed_matmul(p, q, accumulate=True), lambda: inner.packed_matmul(p, q, out=x),
               lambda: inner.unpack(p, torch.float16)):
        with pytest.raises(ValueError):
            fn()
