"""Where the inner phase's operators have gone wrong, or lost something without a word."""
from __future__ import annotations

import copy
import pickle

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import build as libbuild
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref
from tests.test_inner_ops import BF16, CHAIN, DEV, F32, U, gen, half, place

# ------------------------------------------------------------------ norm of rows that hardly vary


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,pad", [(40, 7, 0), (40, 100, 0), (40, 896, 0), (40, 1000, 0), (40, 1021, 3), (40, 1024, 0),
                                           (40, 2047, 0), (40, 2045, 3), (33, 5000, 0), (20, 8190, 2), (7, 16381, 3),
                                           (5, 20001, 0)])
def test_norm_of_rows_of_one_fp32_value_is_zero(rows, cols, pad):
    """The mean of equal values is that value, whatever the roundings of their sum: a mean that is off by
    d = (n + 16) u of the value (n additions in a chain), left as it is, gives y = d / sqrt(eps).  Corrected by
    the mean of x - mean, whose own error is that much of d again, the mean rounds to the value itself."""
    value = torch.cat([torch.tensor([1000.1, 0.1, -3.3e4, 1e-3]), 1000 * torch.randn(rows - 4, generator=gen(cols))])
    x = value[:, None].expand(rows, cols)
    y, mean, rstd = inner.layer_norm(place(x, pad), stats=True)
    big = value.double().abs()
    twice = CHAIN * CHAIN * big + 4 * U * CHAIN * big    # of the mean of x - mean, and of y's own products
    assert torch.equal(mean.cpu(), value)
    assert bool((y.cpu().double().abs() <= 2 * (twice / 1e-5 ** 0.5)[:, None]).all())
    assert bool(((rstd.cpu().double() * 1e-5 ** 0.5 - 1).abs() <= 4 * U + CHAIN * (CHAIN * big) ** 2 / 1e-5).all())
    packed, _, mean, _ = inner.layer_norm_pack(place(x, pad))
    assert torch.equal(mean.cpu(), value) and not bool(packed.codes.float().any())
    dy = torch.randn(rows, cols, generator=gen(1))
    dx, dgamma, _ = inner.layer_norm_backward(place(dy, pad), place(x, pad), mean, rstd)
    assert not bool(dgamma.any())


@pytest.mark.gpu
@pytest.mark.parametrize("cols,pad", [(100, 0), (896, 0), (2047, 1), (5000, 0), (20001, 0)])
def test_norm_of_fp32_rows_whose_spread_is_small_beside_their_mean(cols, pad):
    x = 1000.0 + 1e-3 * torch.randn(50, cols, generator=gen(cols))
    y, mean, rstd = inner.layer_norm(place(x, pad), eps=1e-7, stats=True)
    wy, wmean, wrstd = ref.layer_norm(x, None, None, 1e-7)
    # the values less their mean: exact but for the mean's second error; then y's roundings and those of the variance
    slack = 4 * CHAIN * wy.abs() + wrstd[:, None] * 1001 * (CHAIN * CHAIN + 4 * U * CHAIN)
    assert bool(((y.cpu().double() - wy).abs() <= slack).all())
    assert bool(((mean.cpu().double() - wmean).abs() <= 1001 * (U + CHAIN * CHAIN)).all())


# ------------------------------------------------------------------ products over many values


@pytest.mark.gpu
@pytest.mark.parametrize("k", [65536, 2 ** 20 + 40])
def test_long_sums_in_bf16_do_not_drift(k):
    """Positive products, added up by truncation on the tensor cores: 32 of them lose up to 2^-24 of the sum, 2^-13
    over the 65536 that are added there at most; the parts are joined in fp32.  74 row tiles of one column tile:
    no pair of SMs leaves its sum to others."""
    m, n = 74 * 256, 32
    g = torch.Generator(device=DEV)
    g.manual_seed(k)

    def operand(codes, rows):
        hold = torch.empty(rows, -(-k // 16) * 16, dtype=torch.float8_e4m3fn, device=DEV)[:, :k]
        hold.copy_(codes.expand(rows, k))
        return inner.Packed(hold, torch.ones(-(-rows // 128), -(-k // 128), device=DEV).to(torch.float8_e8m0fnu))

    a = (torch.randn(1, k, device=DEV, generator=g) * 20).abs().to(torch.float8_e4m3fn)
    b = (torch.randn(n, k, device=DEV, generator=g) * 20).abs().to(torch.float8_e4m3fn)
    want = a.double() @ b.double().t()
    got = inner.packed_matmul(operand(a, m), operand(b, n), transpose_b=True)
    assert inner.inner_status() == B.DIPACO_OK
    drift = 2.0 ** -13 + k / 65536 * U
    assert bool(((got.double() - want).abs() <= half(BF16, want * (1 + drift)) + drift * want).all())


# ------------------------------------------------------------------ waits that run out


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.gpu
@pytest.mark.parametrize("operators", [0, 1, 2])  # norms, packing, products: each has an error word of its own
def test_a_wait_that_ran_out_is_reported_once(operators):
    """The diagnostic entry point makes a wait of 1 ms run out on a barrier of its own.  The kernel ends by
    itself, the status says so once, and the operators work as before."""
    x = torch.randn(300, 256, device=DEV)
    w = inner.pack(torch.randn(200, 256, device=DEV))

    def step():
        y, kept, mean, rstd = inner.layer_norm_pack(x)
        return (inner.packed_matmul(y, w, transpose_b=True, out_dtype=F32), *inner.layer_norm_backward(x, kept, mean, rstd))

    want = step()
    assert inner.inner_status() == B.DIPACO_OK
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    B.dipaco_selftest_inner_wait_expiry(operators, 1_000_000, 0, stream())
    end.record()
    torch.cuda.synchronize()
    assert 0.9 <= start.elapsed_time(end) < 100.0
    assert inner.inner_status() == B.DIPACO_ETIMEOUT
    assert inner.inner_status() == B.DIPACO_OK
    for got, before in zip(step(), want):
        assert torch.equal(got, before)
    assert inner.inner_status() == B.DIPACO_OK


@pytest.mark.gpu
def test_no_stream_takes_the_news_of_a_time_out_from_another():
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()

    def status(of):
        with torch.cuda.stream(of):
            return inner.inner_status()

    for s in (mine, other):  # whatever happened before
        status(s)
        assert status(s) == B.DIPACO_OK
    with torch.cuda.stream(mine):
        B.dipaco_selftest_inner_wait_expiry(2, 1_000_000, 0, stream())
    torch.cuda.synchronize()
    assert status(other) == B.DIPACO_ETIMEOUT and status(mine) == B.DIPACO_ETIMEOUT
    assert status(other) == B.DIPACO_OK and status(mine) == B.DIPACO_OK
    assert inner.inner_status() == B.DIPACO_ETIMEOUT and inner.inner_status() == B.DIPACO_OK


def test_the_waits_diagnostic_refuses():
    libbuild.build()
    for bad in ((-1, 1000, 0), (3, 1000, 0), (0, 0, 0), (0, 2 * 10 ** 9, 0), (0, 1000, -1)):
        with pytest.raises(B.DipacoError) as e:
            B.dipaco_selftest_inner_wait_expiry(*bad, None)
        assert e.value.status == B.DIPACO_EINVAL


# ------------------------------------------------------------------ gradients that would not be recorded


@pytest.mark.gpu
def test_tensors_that_require_a_gradient_are_refused_while_it_is_recorded():
    x, g = torch.randn(32, 64, device=DEV), torch.ones(64, device=DEV)
    leaf, weight = x.clone().requires_grad_(), g.clone().requires_grad_()
    stat = torch.ones(32, device=DEV)
    p, q = inner.pack(x), inner.pack(x.t().contiguous())
    out = torch.zeros(32, 32, device=DEV, requires_grad=True)
    calls = [lambda: inner.pack(leaf), lambda: inner.pack(leaf * 2), lambda: inner.layer_norm(leaf), lambda: inner.layer_norm(x, weight),
             lambda: inner.layer_norm(x, g, weight, stats=True), lambda: inner.layer_norm_pack(leaf),
             lambda: inner.layer_norm_pack(x, weight, g), lambda: inner.layer_norm_backward(leaf, x, stat, stat),
             lambda: inner.layer_norm_backward(x, leaf, stat, stat), lambda: inner.layer_norm_backward(x, p, stat, stat, weight),
             lambda: inner.layer_norm_backward(x, p, stat.clone().requires_grad_(), stat), lambda: inner.gelu_pack(leaf),
             lambda: inner.gelu_pack_backward(leaf, p), lambda: inner.packed_matmul(p, q, out=out)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    with torch.inference_mode():
        inner.layer_norm(leaf, weight)
    assert torch.equal(inner.layer_norm(leaf.detach(), weight.detach()), inner.layer_norm(x, g))


@pytest.mark.gpu
def test_the_operators_serve_an_autograd_function():
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gamma, beta):
            y, mean, rstd = inner.layer_norm(x, gamma, beta, stats=True)
            ctx.save_for_backward(x, mean, rstd, gamma)
            return y

        @staticmethod
        def backward(ctx, dy):
            return inner.layer_norm_backward(dy.contiguous(), *ctx.saved_tensors)

    x = torch.randn(40, 100, generator=gen(1)).to(DEV).requires_grad_()
    gamma, beta = (torch.randn(100, generator=gen(i)).to(DEV).requires_grad_() for i in (2, 3))
    dy = torch.randn(40, 100, generator=gen(4)).to(DEV)
    Norm.apply(x, gamma, beta).backward(dy)
    with torch.no_grad():
        _, mean, rstd = inner.layer_norm(x, gamma, beta, stats=True)
        for got, want in zip((x.grad, gamma.grad, beta.grad), inner.layer_norm_backward(dy, x, mean, rstd, gamma)):
            assert torch.equal(got, want)


# ------------------------------------------------------------------ packed matrices as objects


@pytest.mark.gpu
def test_a_packed_matrix_keeps_its_tensors():
    """The kernels go by addresses taken when the object was made: other tensors would not reach them."""
    p, q = inner.pack(torch.ones(64, 100, device=DEV)), inner.pack(torch.zeros(64, 100, device=DEV))
    for name in ("codes", "scales", "struct"):
        with pytest.raises(AttributeError):
            setattr(p, name, getattr(q, name))
    p.codes.copy_(q.codes)  # in place: the same data
    assert not bool(inner.unpack(p).any())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(64, 100), (1, 100), (300, 256), (3, 0), (0, 3)])
def test_a_packed_matrix_can_be_copied(rows, cols):
    x = torch.randn(rows, cols, generator=gen(rows)).to(DEV)
    p = inner.pack(x)
    want = inner.unpack(p, F32)
    shared = copy.copy(p)
    deep, read = copy.deepcopy(p), pickle.loads(pickle.dumps(p))
    p.codes.view(torch.uint8).zero_()
    for other in (deep, read):
        assert other.shape == (rows, cols) and torch.equal(inner.unpack(other, F32), want)
        assert rows * cols == 0 or other.struct.codes not in (p.struct.codes, shared.struct.codes)
    assert not bool(inner.unpack(shared, F32).any())


# ------------------------------------------------------------------ products into a part of a buffer


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1, 27, 30), (1, 1, 5), (8, 3, 100), (8, 25, 2318), (60, 41, 64), (30, 1001, 870), (300, 300, 300),
                                   (257, 333, 129), (2000, 1795, 900), (4100, 1021, 260), (1000, 510, 9000)])
def test_product_writes_nothing_beside_its_result(m, n, k, dtype):
    """Rows on 16-byte boundaries that end inside 16 bytes, with another's data behind them."""
    a, b = inner.pack(torch.randn(k, m, device=DEV)), inner.pack(torch.randn(n, k, device=DEV))
    want = inner.packed_matmul(a, b, True, True, dtype)
    for stride in {-(-n // 8) * 8, -(-n // 8) * 8 + 8, n}:
        for start in (0, 8):
            buffer = torch.full((start + (m - 1) * stride + n + 40,), 3.0, dtype=dtype, device=DEV)
            view = buffer.as_strided((m, n), (stride, 1), start)
            for accumulate in (False, True):
                view.fill_(0.0 if accumulate else 7.0)
                inner.packed_matmul(a, b, True, True, out=view, accumulate=accumulate)
                assert torch.equal(view, want)
                view.fill_(3.0)
                assert bool((buffer == 3.0).all()), (stride, start, accumulate)
