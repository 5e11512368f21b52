"""The common norm of many gradients and their clipping against 64 bits.

Squares are added in fp32 in chains of at most 20 values, four of them joined, each addition off by u = 2^-24 of a sum
of positive terms, and in fp64 beyond: the sum is off by at most 23 u of itself, and the norm by half of that and its own
rounding, under 24 u.  The factor is rounded once more, and
so is each product: a result is off by 26 u of itself, and half a unit of bf16 where it is rounded to that.
"""
from __future__ import annotations

import concurrent.futures
import ctypes
import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner
from tests.test_inner_ops import BF16, DEV, F32, U, assert_within, gen

NORM_OFF, RESULT_OFF = 24 * U, 26 * U


def tensors(sizes, dtypes, seed=0, std=1.0, offsets=(0,)):
    """CPU gradients and the same on the device, each starting some values into an allocation of NaN."""
    host, device = [], []
    for i, n in enumerate(sizes):
        dtype = dtypes[i % len(dtypes)]
        t = (torch.randn(n, generator=gen(seed + i)) * std).to(dtype)
        at = offsets[i % len(offsets)]
        hold = torch.full((at + t.numel() + 9,), math.nan, dtype=dtype, device=DEV)
        view = hold[at:at + t.numel()].view(t.shape)
        view.copy_(t)
        host.append(t)
        device.append(view)
    return host, device


def exact_norm(host):
    return math.sqrt(sum(float(t.double().square().sum()) for t in host))


def factor(norm, most):
    return min(1.0, most / norm) if norm else 1.0


def check(host, device, share):
    norm = exact_norm(host)
    most = share * norm
    by = factor(norm, most)
    got = inner.gradient_norm(device)
    assert got.dtype == F32 and got.shape == () and abs(float(got) - norm) <= NORM_OFF * norm
    want = torch.cat([t.double().reshape(-1) for t in host]) * by
    for dtype in (F32, BF16):
        flat, got = inner.gather_gradients(device, most, dtype=dtype)
        assert abs(float(got) - norm) <= NORM_OFF * norm
        assert_within(flat, want, RESULT_OFF * want.abs(), "gathered", dtype)
        flat, _ = inner.gather_gradients(device, dtype=dtype)
        assert torch.equal(flat.cpu(), torch.cat([t.reshape(-1).to(dtype) for t in host]))
    for t, h in zip(device, host):
        assert torch.equal(t.cpu(), h)
    got = inner.clip_gradients(device, most)
    assert abs(float(got) - norm) <= NORM_OFF * norm
    for t, h in zip(device, host):
        assert_within(t, h.double() * by, RESULT_OFF * h.double().abs() * by, "in place", t.dtype)
        if share > 1:
            assert torch.equal(t.cpu(), h)
        hold = t._base if t._base is not None else t
        first = (t.data_ptr() - hold.data_ptr()) // t.element_size()
        around = torch.cat((hold.view(-1)[:first], hold.view(-1)[first + t.numel():]))
        assert bool(torch.isnan(around).all())  # nothing is written beside a gradient


@pytest.mark.gpu
@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F32, BF16)])
@pytest.mark.parametrize("sizes", [
    [1], [7], [8], [255, 1, 4096], [8192], [8193, 8191], [100000], [0, 3, 0], [(3, 5), (), (2, 1, 7)],
    [(1024, 256), (1024,), (256, 1024), (256,), (256,), (256,)], [3_000_001, 17, 500_000]])
@pytest.mark.parametrize("offsets", [(0,), (1, 3, 0, 2), (4, 5)])
def test_norm_and_clipping(sizes, dtypes, offsets):
    for share in (0.25, 3.0):
        host, device = tensors(sizes, dtypes, 1, 1.0, offsets)
        check(host, device, share)


@pytest.mark.gpu
def test_a_tensor_whose_offsets_pass_32_bits():
    """2^31 values and some, nearly all of them nothing: the others' squares are whole numbers."""
    count = (1 << 31) + 8197
    g = torch.zeros(count, dtype=BF16, device=DEV)
    marks = {0: 3.0, 8191: -4.0, (1 << 30) + 5: 12.0, (1 << 31) - 1: 2.0, 1 << 31: 6.0, (1 << 31) + 1: -2.0, count - 1: 84.0}
    for i, v in marks.items():
        g[i] = v
    norm = math.sqrt(sum(v * v for v in marks.values()))
    assert abs(float(inner.gradient_norm([g])) - norm) <= NORM_OFF * norm
    flat, got = inner.gather_gradients([torch.ones(1, dtype=BF16, device=DEV), g], dtype=BF16)  # at another place within 16 bytes
    assert abs(float(got) - math.sqrt(norm * norm + 1)) <= NORM_OFF * norm
    assert torch.equal(flat[1:], g)
    del flat
    inner.clip_gradients([g], norm / 2)  # halves, which bf16 holds; the factor is off by less than a quarter of its units
    assert all(float(g[i]) == v / 2 for i, v in marks.items()) and int(torch.count_nonzero(g)) == len(marks)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [64, 65, 640, 641, 1300])
def test_many_tensors(count):
    sizes = [1 + (i * 37) % 501 for i in range(count)]
    host, device = tensors(sizes, (F32, BF16), 2)
    check(host, device, 0.5)


@pytest.mark.gpu
def test_so_many_sums_that_they_are_joined_first():
    host, device = tensors([9000] * 3200, (F32,), 3)
    check(host, device, 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("std", [1e-30, 1e-22, 1e-15, 1e15, 1e22, 1e30])
def test_magnitudes_whose_squares_fp32_does_not_hold(std):
    for dtype in (F32, BF16):
        host, device = tensors([5000, 300], (dtype,), 4, std)
        check(host, device, 0.5)


@pytest.mark.gpu
def test_zeros_infinities_and_nan():
    zero = [torch.zeros(100, device=DEV), torch.zeros(3, device=DEV, dtype=BF16)]
    assert float(inner.gradient_norm(zero)) == 0.0
    for most in (0.0, 1.0):
        flat, norm = inner.gather_gradients(zero, most)
        assert float(norm) == 0.0 and bool((flat == 0).all())
    g = [torch.ones(100, device=DEV), torch.full((4,), 2.0, device=DEV)]
    flat, norm = inner.gather_gradients(g, 0.0)
    assert bool((flat == 0).all())
    g[0][5] = math.nan
    flat, norm = inner.gather_gradients(g, 1.0)
    assert math.isnan(float(norm)) and bool(torch.isnan(flat).all())
    g[0][5] = -math.inf
    flat, norm = inner.gather_gradients(g, 1.0)
    assert float(norm) == math.inf and math.isnan(float(flat[5])) and float(flat.nan_to_num().abs().sum()) == 0.0
    flat, norm = inner.gather_gradients(g)
    assert float(norm) == math.inf and float(flat[5]) == -math.inf and float(flat[0]) == 1.0


@pytest.mark.gpu
def test_tensors_in_other_orders():
    """The norm and clipping in place go by memory; gathering takes the values in their own order."""
    t = torch.randn(4, 6, 5, generator=gen(1)).to(DEV).permute(2, 0, 1)
    norm = float(t.double().norm())
    assert abs(float(inner.gradient_norm([t])) - norm) <= NORM_OFF * norm
    want = t.double() * 0.5
    inner.clip_gradients([t], 0.5 * norm)
    assert_within(t, want.cpu(), RESULT_OFF * want.abs().cpu(), "permuted")
    with pytest.raises(ValueError):
        inner.gather_gradients([t])


@pytest.mark.gpu
def test_a_captured_call_follows_its_inputs_and_streams_agree():
    host, device = tensors([100_000, 77, 3], (F32, BF16), 5)
    first = inner.gather_gradients(device, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = inner.gather_gradients(device, 1.0)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = inner.gather_gradients(device, 1.0)
    with torch.cuda.graph(other):
        fourth = inner.gradient_norm(device)
    for t in device:
        t.mul_(2)
    graph.replay()
    other.replay()
    torch.cuda.synchronize()
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    assert float(third[1]) == 2 * float(first[1]) == float(fourth)  # powers of two change no rounding
    assert torch.equal(third[0], first[0])


@pytest.mark.gpu
def test_calls_from_several_threads():
    made = [tensors([50_000 + i, 10 * i + 1], (F32,), 10 * i) for i in range(4)]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                flat, norm = inner.gather_gradients(made[i][1], 1.0)
            torch.cuda.current_stream().synchronize()
            return flat, float(norm)

    torch.cuda.synchronize()
    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        for i, (flat, norm) in enumerate(pool.map(work, range(4))):
            want = exact_norm(made[i][0])
            assert abs(norm - want) <= NORM_OFF * want
            assert abs(float(flat.double().norm()) - 1.0) <= 2 * RESULT_OFF


def test_bad_arguments_are_refused():
    """By the library, before any CUDA call."""
    lib = B.load()
    p = 1 << 20  # never read
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32

    def status(grads=(p,), out=(2 * p,), numel=(8,), dtypes=(0,), out_dtypes=(0,), most=1.0, norm=p, work=p, size=1 << 20,
               device=0, count=None):
        array = lambda t, v: None if v is None else (t * len(v))(*v)  # noqa: E731
        return lib.dipaco_clip_gradients(array(vp, grads), array(vp, out), array(i64, numel), array(i32, dtypes),
                                         array(i32, out_dtypes), len(numel or ()) if count is None else count, most, norm, work,
                                         size, device, None)

    two = dict(grads=(p, 4 * p), numel=(8, 8), dtypes=(0, 0), out_dtypes=(0, 0))
    for bad in (dict(most=-1.0), dict(most=math.nan), dict(count=-1), dict(grads=None), dict(dtypes=None), dict(out_dtypes=None),
                dict(numel=(-1,)), dict(dtypes=(2,)), dict(out_dtypes=(-1,)), dict(grads=(None,)), dict(out=(None,)), dict(grads=(p + 2,)),
                dict(out=(p + 3,)), dict(norm=p + 1), dict(device=-1),
                dict(out=(p + 4,)), dict(out=(p - 4,)), dict(out=(p,), out_dtypes=(1,)),   # over its own gradient, not in place
                dict(**two, out=(p, p)), dict(**two, out=(8 * p, 8 * p + 28)),              # over one another
                dict(**two, out=(8 * p, p)), dict(**two, out=(4 * p, p))):                  # over another's gradient
        assert status(**bad) == B.DIPACO_EINVAL, bad
    many = dict(out=(1 << 40,), numel=(1 << 21,))  # fewer values need no workspace
    for bad in (dict(work=None), dict(work=p + 8), dict(size=64)):
        assert status(**many, **bad) == B.DIPACO_EINVAL, bad
    assert status(numel=(1 << 45,)) == B.DIPACO_ELIMIT
    assert status(numel=(1 << 44,)) == B.DIPACO_ELIMIT  # more chunks than are counted
    size = ctypes.c_int64()
    assert lib.dipaco_clip_gradients_workspace(None, 1, size) == B.DIPACO_EINVAL
    assert lib.dipaco_clip_gradients_workspace((i64 * 1)(-1), 1, size) == B.DIPACO_EINVAL
    assert lib.dipaco_clip_gradients_workspace((i64 * 2)(0, 0), 2, size) == B.DIPACO_OK and size.value == 0


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    x = torch.ones(4, 8, device=DEV)
    for bad in ([], [x.cpu()], [x.double()], [x, x.cpu()], [x[:, :7]], [x[:, ::2]], [x.expand(2, 4, 8)]):
        with pytest.raises(ValueError):
            inner.gradient_norm(bad)
    with pytest.raises(ValueError):
        inner.clip_gradients([x], -1.0)
    with pytest.raises(ValueError):
        inner.gather_gradients([x], dtype=torch.float16)
    with pytest.raises(B.DipacoError):
        inner.clip_gradients([x, x], 1.0)  # the same tensor twice would be scaled twice
    assert bool((x == 1).all())
    assert abs(float(inner.gradient_norm([x, x])) - 8.0) <= NORM_OFF * 8
    w = torch.ones(4, device=DEV, requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        inner.gradient_norm([w])
    with torch.no_grad():
        assert float(inner.gradient_norm([w])) == 2.0
