"""The loops of the inner phase's operators: enough rows that every block of threads goes round several
times (rings and buffers are filled again and their barriers change phase), rows that end inside a
16-byte unit with padding between them, and products of a few tokens over many outputs.

Everything is compared with 64-bit sums, at tolerances that follow from the kernels' roundings as in
test_inner_ops; what lies between the rows is NaN on the way in and has to be untouched on the way out.
"""
from __future__ import annotations

import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref
from tests.test_inner_ops import BF16, CHAIN, DEV, F32, U, half, product_tolerance

pytestmark = pytest.mark.gpu

CODE = {F32: B.DIPACO_F32, BF16: B.DIPACO_BF16}


def held(rows, cols, dtype, mode, fill=math.nan):
    """A matrix inside a buffer of `fill`: rows of whole 16-byte units ("units"), rows that end inside one
    but start on 16 bytes ("ragged"), or rows at any element ("single").  (view, buffer)"""
    per = 16 // dtype.itemsize
    stride = -(-cols // per) * per + (1 if mode == "single" else 0)
    buffer = torch.full((rows, stride), fill, dtype=dtype, device=DEV)
    assert mode == "single" or buffer.data_ptr() % 16 == 0
    return buffer[:, :cols], buffer


def filled(seed, rows, cols, dtype, mode, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    view, _ = held(rows, cols, dtype, mode)
    view.normal_(0.0, std, generator=g)
    return view


def width(cols, dtype, mode):
    """`cols`, made a whole number of 16-byte units for "units"."""
    per = 16 // dtype.itemsize
    assert cols % per
    return -(-cols // per) * per if mode == "units" else cols


def near(got, want, tol, what, dtype=None):
    tol = tol + (half(dtype, want.abs() + tol) if dtype is not None else 0.0)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[0].tolist())


def stream():
    return torch.cuda.current_stream().cuda_stream


# Rows at more than two passes of the grid: 148 SMs, up to eight blocks of threads on each.
NORM_ROWS = {BF16: [(60, 45000), (100, 20000), (250, 10000), (601, 10000), (897, 10000), (1505, 6000), (2047, 6000),
                    (4093, 2200), (8189, 1400), (16381, 400)],
             F32: [(30, 45000), (61, 20000), (126, 10000), (382, 10000), (1021, 6000), (2045, 2200), (4093, 1400),
                   (8189, 400), (16381, 400)]}


@pytest.mark.parametrize("mode", ["units", "ragged", "single"])
@pytest.mark.parametrize("dtype,cols,rows", [(t, c, r) for t in NORM_ROWS for c, r in NORM_ROWS[t]])
def test_norm_goes_over_its_rows_again(dtype, cols, rows, mode):
    cols = width(cols, dtype, mode)
    x = filled(cols, rows, cols, dtype, mode, 1.3)
    gamma, beta = torch.randn(cols, device=DEV) * 0.3 + 1, torch.randn(cols, device=DEV) * 0.3
    wy, wmean, wrstd = ref.layer_norm(x, gamma, beta, 1e-5)
    big = x.double().abs().amax(1)
    hat = ((x.double() - wmean[:, None]) * wrstd[:, None]).abs()
    slack = CHAIN * ((hat + (big * wrstd)[:, None]) * gamma.double().abs() + beta.double().abs())
    for with_y in (True, False):
        y, whole = held(rows, cols, dtype, mode, 7.0)
        mean, rstd = torch.full((2, rows), math.nan, device=DEV).unbind(0)
        B.dipaco_layer_norm(x.data_ptr(), x.stride(0), gamma.data_ptr(), beta.data_ptr(),
                            y.data_ptr() if with_y else None, y.stride(0), mean.data_ptr(), rstd.data_ptr(), rows, cols,
                            1e-5, CODE[dtype], B.DIPACO_F32, 0, stream())
        near(mean, wmean, CHAIN * big, "mean")
        near(rstd, wrstd, CHAIN * wrstd * (1 + wrstd * big), "rstd")
        if with_y:
            near(y, wy, slack, "y", dtype)
            assert bool((whole[:, cols:] == 7.0).all())
        else:
            assert bool((whole == 7.0).all())


# Rows at more than five passes of 148 blocks: more than the ring of rows on their way is deep.
BACK_ROWS = [(8, 115000), (16, 58000), (32, 29000), (64, 14600), (128, 7300), (256, 3700), (512, 1000), (1024, 1000)]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("mode", ["units", "ragged", "single"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("threads,rows", BACK_ROWS)  # threads for a row, 32 bytes each
def test_norm_gradient_refills_its_ring(threads, rows, dtype, mode, packed):
    cols = width(threads * 32 // dtype.itemsize - 3, dtype, mode)
    x = filled(threads, rows, cols, dtype, mode, 1.3)
    dy = filled(threads + 1, rows, cols, dtype, mode, 1e-2)
    gamma = torch.randn(cols, device=DEV) * 0.3 + 1
    _, mean, rstd = ref.layer_norm(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    kept = None
    if packed:
        kept = inner.pack(x)
        x64 = kept.codes.double() * ref.spread(kept.scales.double(), rows, cols)
    else:
        x64 = x.double()
    dx, whole = held(rows, cols, dtype, mode, 7.0)
    dgamma, dbeta = torch.full((2, cols), math.nan, device=DEV).unbind(0)
    need = B.dipaco_layer_norm_workspace(rows, cols)
    work = torch.empty(need, dtype=torch.uint8, device=DEV)
    B.dipaco_layer_norm_backward(dy.data_ptr(), dy.stride(0), None if packed else x.data_ptr(), x.stride(0),
                                 kept.struct if packed else None, mean.data_ptr(), rstd.data_ptr(), gamma.data_ptr(),
                                 dx.data_ptr(), dx.stride(0), dgamma.data_ptr(), dbeta.data_ptr(), rows, cols, CODE[dtype],
                                 B.DIPACO_F32, work.data_ptr(), need, 0, stream())
    assert inner.inner_status() == B.DIPACO_OK
    wx, wg, wb = ref.layer_norm_backward(dy, x64, mean, rstd, gamma)
    r = rstd.double()[:, None]
    big = ((x64 - mean.double()[:, None]) * r).abs() + mean.double().abs()[:, None] * r
    g = dy.double().abs() * gamma.double().abs()
    near(dx, wx, CHAIN * r * (g + g.mean(1, keepdim=True) + big * (g * big).mean(1, keepdim=True)), "dx", dtype)
    assert bool((whole[:, cols:] == 7.0).all())
    # a thread adds up at most 14 rows, 64 groups of a block are joined one by one, then the blocks' sums
    near(dgamma, wg, 192 * U * (dy.double().abs() * big).sum(0), "dgamma")
    near(dbeta, wb, 192 * U * dy.double().abs().sum(0), "dbeta")


# More than five blocks of 128 x 128 for each of 296 blocks of threads; few and many columns of blocks.
STREAMED = [(190000, 24, "units"), (190000, 21, "ragged"), (97000, 140, "ragged"), (5200, 5000, "units")]


@pytest.mark.parametrize("rows,cols,mode", STREAMED)
def test_streamed_blocks_refill_their_buffers(rows, cols, mode):
    x = filled(rows, rows, cols, BF16, mode, 2.0)
    x.mul_(torch.exp(2 * torch.rand(rows // 128 + 1, 1, device=DEV)).repeat_interleave(128, 0)[:rows].to(BF16))
    dy = filled(cols, rows, cols, BF16, mode, 1e-3)
    codes, scales = ref.pack(x.cpu())
    p = inner.pack(x)
    y, kept = inner.gelu_pack(x)
    dx = inner.gelu_pack_backward(dy, kept)
    gamma, beta = torch.randn(cols, device=DEV) * 0.3 + 1, torch.randn(cols, device=DEV) * 0.3
    normed, kept_too, mean, rstd = inner.layer_norm_pack(x, gamma, beta)
    assert inner.inner_status() == B.DIPACO_OK
    for q in (p, kept, kept_too):
        assert torch.equal(q.scales.cpu().double(), scales) and torch.equal(q.codes.cpu().double(), codes)

    a = x.cpu().double()
    want = ref.gelu(a)
    slack = 16 * U * want.abs() + 8 * U * a.abs() * (2.0 * a ** 2 + 4).clamp(max=64.0) * torch.exp(-a.abs())
    ref.assert_packed_close(y.codes, y.scales, want, slack, "gelu")
    a, d = codes * ref.spread(scales, rows, cols), dy.cpu().double()
    slack = d.abs() * U * (32 + 8 * (2 * a * a + 4).clamp(max=64.0) ** 2 * torch.exp(-a.abs()))
    ref.assert_packed_close(dx.codes, dx.scales, d * ref.gelu_slope(a), slack, "gradient")
    wy, wmean, wrstd = ref.layer_norm(x.cpu(), gamma.cpu(), beta.cpu(), 1e-5)
    big = x.cpu().double().abs().amax(1)
    near(mean.cpu(), wmean, CHAIN * big, "mean")
    near(rstd.cpu(), wrstd, CHAIN * wrstd * (1 + wrstd * big), "rstd")
    hat = ((x.cpu().double() - wmean[:, None]) * wrstd[:, None]).abs()
    slack = CHAIN * ((hat + (big * wrstd)[:, None]) * gamma.cpu().double().abs() + beta.cpu().double().abs())
    ref.assert_packed_close(normed.codes, normed.scales, wy, slack, "norm")


# As many tokens as are multiplied in registers, on either side, and outputs beyond one pass (4736).
@pytest.mark.parametrize("m,n,k", [(3, 130, 100), (4, 900, 515), (3, 5000, 700), (4, 9600, 257), (1, 9601, 700), (2, 9500, 31),
                                   (130, 3, 100), (900, 4, 515), (9600, 4, 257), (9601, 1, 700), (9500, 2, 1030), (4, 3, 5000),
                                   (3, 4, 5000), (5000, 3, 16)])
def test_product_of_a_few_tokens(m, n, k):
    def operand(seed, rows, std):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        size = torch.empty(-(-rows // 128), -(-k // 128), device=DEV).normal_(0.0, 1.0, generator=g).exp()
        values = torch.empty(rows, k, device=DEV).normal_(0.0, std, generator=g) * ref.spread(size, rows, k)
        p = inner.pack(values)
        # rows of codes are padded with anything: here with NaN
        hold = torch.full((rows, -(-k // 16) * 16 + 16), 0x7F, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        hold[:, :k].copy_(p.codes)
        return inner.Packed(hold[:, :k], p.scales), p.codes.double() * ref.spread(p.scales.double(), rows, k)

    (a, av), (b, bv) = operand(m, m, 1.0), operand(n + 1, n, 0.02)
    want, tol = av @ bv.t(), product_tolerance(av, bv.t(), k)
    for dtype in (F32, BF16):
        got = inner.packed_matmul(a, b, transpose_b=True, out_dtype=dtype)
        near(got, want, tol, str(dtype), dtype)
        whole = torch.full((m, n + 3), 2.0, dtype=dtype, device=DEV)
        inner.packed_matmul(a, b, transpose_b=True, out=whole[:, 1:n + 1], accumulate=True)
        near(whole[:, 1:n + 1], want + 2.0, tol + U * (want + 2.0).abs(), "accumulated", dtype)
        assert bool((whole[:, :1] == 2.0).all()) and bool((whole[:, n + 1:] == 2.0).all())
