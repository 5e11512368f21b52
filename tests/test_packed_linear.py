"""Linear layers on packed matrices with bias, activation and residual against 64 bits.

The sums are those of the products (``product_tolerance``).  An activation is evaluated with an exponent that is off
by a few u = 2^-24 of itself and two approximations good to two units in the last place: off by 64 u of its value and
as much of its argument, up to 1; slopes are at most 1.13, so that what a sum is off grows by no more.
"""
from __future__ import annotations

import itertools
import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref
from tests.test_inner_ops import (BF16, CHAIN, DEV, F32, U, gen, half, packed_operand, place, product_tolerance,
                                  random_packed_on_device)

ACTIVATIONS = (None, "relu", "silu", "gelu")


def act(a, name):
    if name == "relu":
        return a.clamp(min=0.0)
    if name == "silu":
        return a / (1.0 + torch.exp(-a))
    return ref.gelu(a) if name == "gelu" else a


def slope(a, name):
    """Central differences of the activation in 64 bits, off by eps^2/6 times its third derivative: under 1e-10."""
    if name == "relu":
        return (a > 0).double()
    eps = 1e-5
    return (act(a + eps, name) - act(a - eps, name)) / (2 * eps)


def act_tolerance(a, y, name):
    return 0.0 if name in (None, "relu") else 64 * U * (y.abs() + a.abs().clamp(max=1.0))


def assert_dense(got, want, tol, dtype, what):
    got, tol = got.double(), tol + half(dtype, want.abs() + tol)
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[0].tolist(), float(((got - want).abs() / tol).max()))


def vector(seed, n, dtype=F32, std=0.5, mean=0.0):
    return (torch.randn(n, generator=gen(seed)) * std + mean).to(dtype)


SIZES = [(1, 1, 1), (1, 896, 896), (1, 130, 4000), (2, 300, 65), (4, 3000, 200), (5, 64, 31), (16, 257, 300), (33, 500, 1000),
         (128, 128, 128), (129, 127, 257), (200, 300, 400), (255, 513, 96), (384, 640, 1024), (300, 3, 500), (1000, 130, 2100)]


def check_all(m, n, k, name, operand, on, bias_dtype):
    """Every form at one size; `on` brings the 64-bit values where the operands' are."""
    x, xv = operand(m + 3 * n, m, k)
    w, wv = operand(n + 7 * k, n, k, 0.1)
    bias = vector(5, n, bias_dtype)
    a = xv @ wv.t() + on(bias.double())
    tol_a = product_tolerance(xv, wv.t(), k) + U * (a.abs() + on(bias.double()).abs())
    y = act(a, name)
    tol_y = 1.13 * tol_a + act_tolerance(a, y, name)
    for dtype in (F32, BF16):
        residual = torch.randn(m, n, generator=gen(9)).to(dtype)
        got = inner.packed_linear(x, w, bias.to(DEV), name, place(residual), dtype)
        assert got.dtype == dtype
        want = y + on(residual.double())
        assert_dense(on(got), want, tol_y + U * want.abs(), dtype, ("residual", name, dtype))
        assert torch.equal(got, inner.packed_linear(x, w, bias.to(DEV), name, place(residual, 3, 1)))  # other strides
        got = inner.packed_linear(x, w, bias.to(DEV), name, out_dtype=dtype)
        assert_dense(on(got), y, tol_y, dtype, ("bias", name, dtype))
        got = inner.packed_linear(x, w, None, name, out_dtype=dtype)
        a0 = xv @ wv.t()
        tol_0 = product_tolerance(xv, wv.t(), k)
        assert_dense(on(got), act(a0, name), 1.13 * tol_0 + act_tolerance(a0, act(a0, name), name), dtype, ("no bias", name, dtype))
    for keep in (True, False):
        got, kept = inner.packed_linear_pack(x, w, bias.to(DEV), name, keep)
        assert (kept is not None) == (keep and name is not None)
        ref.assert_packed_close(got.codes, got.scales, y.cpu(), tol_y.cpu(), ("y", name))
        if kept is not None:
            ref.assert_packed_close(kept.codes, kept.scales, a.cpu(), tol_a.cpu(), ("a", name))
    # back: dy [m, k] through a weight [k, n], slopes of a [m, n]
    dy, dyv = operand(m + 11, m, k, 0.01)
    v, vv = operand(n + 13, k, n, 0.1)
    at, av = operand(n + 17, m, n, 1.0)
    da = dyv @ vv
    tol = product_tolerance(dyv, vv, k)
    if name is not None:
        s = slope(av, name)
        tol = 1.13 * tol + (64 * U + 1e-9) * da.abs()
        da = da * s
    got, dbias = inner.packed_linear_pack_backward(dy, v, None if name is None else at, name)
    ref.assert_packed_close(got.codes, got.scales, da.cpu(), tol.cpu(), ("da", name))
    off = (on(dbias.double()) - da.sum(0)).abs()
    allowed = tol.sum(0) + CHAIN * da.abs().sum(0)
    assert bool((off <= allowed).all()), ("dbias", name, float((off / allowed).max()))
    again, none = inner.packed_linear_pack_backward(dy, v, None if name is None else at, name, bias=False)
    assert none is None and torch.equal(again.codes.view(torch.uint8), got.codes.view(torch.uint8))
    assert inner.inner_status() == B.DIPACO_OK


@pytest.mark.gpu
@pytest.mark.parametrize("name", ACTIVATIONS)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(m, n, k, name):
    check_all(m, n, k, name, packed_operand, lambda t: t.cpu(), F32 if (m + n) % 2 else BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,name", [(2000, 1792, 900, "gelu"), (4100, 2048, 512, "silu"), (600, 1000, 9000, "gelu"),
                                        (3000, 5000, 300, "relu"), (70, 9000, 1500, "gelu"), (65, 2048, 4096, None),
                                        (20000, 900, 128, "gelu"), (9000, 2300, 600, "silu"), (8000, 20, 2500, "gelu")])
def test_larger_sizes(m, n, k, name):
    """Several tiles for a pair of SMs, both widths of a tile, contractions that the dense form deals out."""
    check_all(m, n, k, name, random_packed_on_device, lambda t: t.to(DEV), F32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sums_that_are_taken_out_of_the_tensor_cores(dtype):
    """Contractions over 2048 values in fp32, and over 65536 in bf16, are joined from parts."""
    for k in (2300, 70000):
        x, xv = random_packed_on_device(1, 130, k)
        w, wv = random_packed_on_device(2, 140, k, 0.01)
        bias, residual = vector(3, 140), torch.randn(130, 140, generator=gen(4)).to(dtype)
        a = xv @ wv.t() + bias.double().to(DEV)
        got = inner.packed_linear(x, w, bias.to(DEV), "silu", residual.to(DEV))
        want = act(a, "silu") + residual.double().to(DEV)
        assert_dense(got, want, 1.13 * product_tolerance(xv, wv.t(), k) + act_tolerance(a, act(a, "silu"), "silu") + U * want.abs(),
                     dtype, k)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ACTIVATIONS)
@pytest.mark.parametrize("shift", [-0.5, -3.0, -30.0, 30.0])
@pytest.mark.parametrize("m,n", [(3, 200), (300, 520)])
def test_arguments_far_to_one_side(name, shift, m, n):
    """Blocks in which no argument is large: their largest activation is not that of the largest argument."""
    x, xv = packed_operand(1, m, 100, 0.05)
    w, wv = packed_operand(2, n, 100, 0.05)
    bias = vector(3, n, std=0.01, mean=shift)
    a = xv @ wv.t() + bias.double()
    tol_a = product_tolerance(xv, wv.t(), 100) + U * (a.abs() + bias.double().abs())
    y = act(a, name)
    got, kept = inner.packed_linear_pack(x, w, bias.to(DEV), name)
    # far below zero an activation is as small as its share, which is off by 2^-24 |e| of itself, |e| under 900
    ref.assert_packed_close(got.codes, got.scales, y, (1.13 * tol_a if shift > -3 else (1 + a.abs()) ** 3 * y.abs() * tol_a) +
                            act_tolerance(a, y, name) * (1.0 if shift > -3 else y.abs() * 900), name)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ACTIVATIONS)
@pytest.mark.parametrize("m", [2, 150])
def test_infinities_and_nan_harm_no_neighbour(name, m):
    n, k = 300, 64
    x, xv = packed_operand(1, m, k)
    w, wv = packed_operand(2, n, k, 0.1)
    bias = vector(3, n)
    clean, clean_a = inner.packed_linear_pack(x, w, bias.to(DEV), name)
    bias[7], bias[200], bias[299] = math.inf, -math.inf, math.nan
    got, got_a = inner.packed_linear_pack(x, w, bias.to(DEV), name)
    for p, q, kind in ((got, clean, name),) + (((got_a, clean_a, None),) if name else ()):
        v, before = ref.values(p.codes, p.scales), ref.values(q.codes, q.scales)
        nan = [7, 299] if kind == "relu" else [7, 200, 299]
        others = [c for c in range(n) if c not in (7, 200, 299)]
        assert bool(torch.isnan(v[:, nan]).all())
        if kind == "relu":
            assert bool((v[:, 200] == 0).all())
        # a block may have lost its largest value with those columns, and then has a finer scale
        spacing = ref.e4m3_spacing(before[:, others] / ref.spread(q.scales.cpu().double(), m, n)[:, others]) * ref.spread(q.scales.cpu().double(), m, n)[:, others]
        assert bool(((v[:, others] - before[:, others]).abs() <= spacing).all())
    dense = inner.packed_linear(x, w, bias.to(DEV), name, out_dtype=F32).cpu()
    fine = torch.isfinite(dense)
    assert bool(fine[:, [c for c in range(n) if c not in (7, 200, 299)]].all()) and bool(torch.isnan(dense[:, 299]).all())


@pytest.mark.gpu
def test_gradients_pass_infinities_and_nan_to_their_columns_alone():
    m, n, k = 140, 300, 40
    dy, _ = packed_operand(1, m, k)
    w, _ = packed_operand(2, k, n)
    a, _ = packed_operand(3, m, n)
    clean, clean_b = inner.packed_linear_pack_backward(dy, w, a, "gelu")
    a.codes.view(torch.uint8)[130, 5] = 0x7F  # NaN
    got, b = inner.packed_linear_pack_backward(dy, w, a, "gelu")
    v, before = ref.values(got.codes, got.scales), ref.values(clean.codes, clean.scales)
    assert int(torch.isnan(v).sum()) == 1 and bool(torch.isnan(v[130, 5])) and torch.isnan(b.cpu()).nonzero().tolist() == [[5]]
    assert torch.equal(v[:128], before[:128]) and torch.equal(b.cpu()[6:], clean_b.cpu()[6:])
    # products beyond fp32: infinities, which have no code
    big = inner.Packed(dy.codes, torch.full_like(dy.scales.view(torch.uint8), 254).view(torch.float8_e8m0fnu))
    got, _ = inner.packed_linear_pack_backward(big, inner.Packed(w.codes, torch.full_like(w.scales.view(torch.uint8), 200).view(torch.float8_e8m0fnu)))
    v = ref.values(got.codes, got.scales)
    assert bool(torch.isnan(v).any()) and not bool(torch.isinf(v).any())


@pytest.mark.gpu
def test_small_whole_numbers_are_exact():
    m, n, k = 300, 270, 520
    x = torch.randint(-8, 9, (m, k), generator=gen(1)).double()
    w = torch.randint(-8, 9, (n, k), generator=gen(2)).double()
    bias, residual = torch.randint(-99, 99, (n,), generator=gen(3)).float(), torch.randint(-99, 99, (m, n), generator=gen(4)).float()

    def hold(v):
        scales = torch.ones(-(-v.shape[0] // 128), -(-v.shape[1] // 128)).to(torch.float8_e8m0fnu)
        wide = torch.zeros(v.shape[0], -(-v.shape[1] // 16) * 16, device=DEV, dtype=torch.float8_e4m3fn)
        wide[:, :v.shape[1]].copy_(v.to(torch.float8_e4m3fn))
        return inner.Packed(wide[:, :v.shape[1]], scales.to(DEV))

    a = x @ w.t() + bias.double()
    got = inner.packed_linear(hold(x), hold(w), bias.to(DEV), "relu", residual.to(DEV))
    assert torch.equal(got.cpu().double(), a.clamp(min=0) + residual.double())
    got, kept = inner.packed_linear_pack(hold(x), hold(w), bias.to(DEV), "relu")
    for p, v in ((got, a.clamp(min=0)), (kept, a)):
        codes, scales = ref.pack(v)
        assert torch.equal(p.codes.cpu().double(), codes) and torch.equal(p.scales.cpu().double(), scales)
    got, dbias = inner.packed_linear_pack_backward(hold(x), hold(w.t()), kept, "relu")
    da = (x @ w.t()) * (ref.values(kept.codes, kept.scales) > 0)
    codes, scales = ref.pack(da)
    assert torch.equal(got.codes.cpu().double(), codes) and torch.equal(got.scales.cpu().double(), scales)
    assert torch.equal(dbias.cpu().double(), da.sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [3, 40, 300])
@pytest.mark.parametrize("n,first,stride", [(101, 16, 320), (300, 32, 384), (64, 0, 64)])
def test_results_stay_inside_a_slice_of_a_wider_buffer(m, n, first, stride):
    x, _ = packed_operand(1, m, 60)
    w, _ = packed_operand(2, n, 60)
    a, _ = packed_operand(3, m, n)
    back, _ = packed_operand(4, 60, n)
    want, kept = inner.packed_linear_pack(x, w, None, "gelu")
    da, _ = inner.packed_linear_pack_backward(x, back, a, "gelu")
    holds = [torch.full((m + 2, stride), 0x55, dtype=torch.uint8, device=DEV) for _ in range(3)]
    outs = [inner.Packed(h.view(torch.float8_e4m3fn)[1:m + 1, first:first + n], torch.empty_like(want.scales)) for h in holds]
    need = B.dipaco_packed_linear_pack_workspace(m, n, 60)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    B.dipaco_packed_linear_pack(x.struct, w.struct, None, 0, B.DIPACO_ACTIVATION_GELU, outs[0].struct, outs[1].struct,
                                work.data_ptr(), need, 0, stream)
    B.dipaco_packed_linear_pack_backward(x.struct, back.struct, a.struct, B.DIPACO_ACTIVATION_GELU, outs[2].struct, None,
                                         None, 0, 0, stream)
    for hold, out, p in zip(holds, outs, (want, kept, da)):
        assert torch.equal(out.codes.view(torch.uint8), p.codes.view(torch.uint8))
        assert torch.equal(out.scales.view(torch.uint8), p.scales.view(torch.uint8))
        out.codes.view(torch.uint8).fill_(0x55)
        assert bool((hold == 0x55).all())


@pytest.mark.gpu
@pytest.mark.parametrize("m,stride", [(3, 1 << 31), (100, 1 << 26)])
def test_rows_whose_offsets_pass_32_bits(m, stride):
    """Operands, checkpoint and residual with rows far apart give what the same rows give side by side."""
    n, k = 320, 256
    x, w, back = (random_packed_on_device(i, *shape)[0] for i, shape in enumerate(((m, k), (n, k), (k, n))))
    a = random_packed_on_device(3, m, n)[0]
    residual = torch.randn(m, n, generator=gen(4)).to(BF16).to(DEV)
    bias = vector(5, n).to(DEV)

    def far(p):
        hold = torch.empty((m - 1) * stride + p.shape[1], dtype=torch.uint8, device=DEV)
        codes = hold.as_strided(p.shape, (stride, 1))
        codes.copy_(p.codes.view(torch.uint8))
        return inner.Packed(codes.view(torch.float8_e4m3fn), p.scales)

    def far_dense(t):
        hold = torch.empty((m - 1) * (stride // 2) + n, dtype=BF16, device=DEV)
        view = hold.as_strided(t.shape, (stride // 2, 1))
        return view.copy_(t)

    def everything(x, a, residual):
        dense = inner.packed_linear(x, w, bias, "gelu", residual)
        y, kept = inner.packed_linear_pack(x, w, bias, "silu")
        da, dbias = inner.packed_linear_pack_backward(x, back, a, "gelu")
        return [t.view(torch.uint8) if t.element_size() == 1 else t
                for t in (dense, y.codes, y.scales, kept.codes, kept.scales, da.codes, da.scales, dbias)]

    near = everything(x, a, residual)
    for got, want in zip(everything(far(x), far(a), far_dense(residual)), near):
        assert torch.equal(got, want)


@pytest.mark.gpu
def test_sums_over_nothing():
    dev = torch.device(DEV)
    bias = vector(1, 200)
    for m in (1, 5, 300):
        x, w = inner.Packed.empty(m, 0, dev), inner.Packed.empty(200, 0, dev)
        residual = torch.randn(m, 200, generator=gen(2))
        got = inner.packed_linear(x, w, bias.to(DEV), "relu", residual.to(DEV))
        assert torch.equal(got.cpu(), bias.clamp(min=0) + residual)
        y, a = inner.packed_linear_pack(x, w, bias.to(DEV), "gelu")
        want = bias.double().expand(m, 200)
        ref.assert_packed_close(a.codes, a.scales, want, 0 * want)
        ref.assert_packed_close(y.codes, y.scales, act(want, "gelu"), 128 * U + 0 * want)
        da, dbias = inner.packed_linear_pack_backward(inner.Packed.empty(m, 0, dev), inner.Packed.empty(0, 200, dev), a, "gelu")
        assert bool((ref.values(da.codes, da.scales) == 0).all()) and bool((dbias == 0).all())
    for m, n, k in ((0, 5, 9), (5, 0, 9), (0, 0, 0)):
        x, w = inner.Packed.empty(m, k, dev), inner.Packed.empty(n, k, dev)
        assert inner.packed_linear(x, w, torch.zeros(n, device=DEV), "silu").shape == (m, n)
        assert inner.packed_linear_pack(x, w)[0].shape == (m, n)
        da, dbias = inner.packed_linear_pack_backward(inner.Packed.empty(m, k, dev), inner.Packed.empty(k, n, dev))
        assert da.shape == (m, n) and bool((dbias == 0).all())


@pytest.mark.gpu
def test_streams_repeats_and_graphs_agree():
    x, _ = random_packed_on_device(1, 700, 300)
    w, _ = random_packed_on_device(2, 900, 300)
    w2, _ = random_packed_on_device(3, 300, 900)
    bias, bias2 = vector(4, 900).to(DEV), vector(5, 300, BF16).to(DEV)
    residual = torch.randn(700, 300, generator=gen(6)).to(BF16).to(DEV)

    def step():
        y, a = inner.packed_linear_pack(x, w, bias, "gelu")
        out = inner.packed_linear(y, w2, bias2, None, residual)
        dy = inner.pack(out)
        da, dbias = inner.packed_linear_pack_backward(dy, w2, a, "gelu")
        return [out, dbias] + [t.view(torch.uint8) for p in (y, a, da) for t in (p.codes, p.scales)]

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    made = []
    for g in graphs:
        with torch.cuda.graph(g):
            made.append(step())
    for t in made[0] + made[1]:
        t.zero_()
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for a, b, c, d in zip(first, second, *made):
        assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)
    assert inner.inner_status() == B.DIPACO_OK


# ------------------------------------------------------------------ refusals

def test_bad_arguments_are_refused():
    """By the library, before any CUDA call."""
    lib = B.load()
    p = 1 << 20  # never read
    S = B.PackedStruct
    x, w, y = S(p, p, 4, 8, 16), S(p, p, 6, 8, 16), S(p, p, 4, 6, 16)

    def dense(x=x, w=w, bias=p, bias_dtype=0, act=0, residual=p, rs=6, out=p, ys=6, dtype=0, device=0):
        return lib.dipaco_packed_linear(x, w, bias, bias_dtype, act, residual, rs, out, ys, dtype, None, 0, device, None)

    for bad in (dict(x=None), dict(w=None), dict(w=S(p, p, 6, 9, 16)), dict(x=S(p, p, 4, 8, 15)), dict(x=S(p + 8, p, 4, 8, 16)),
                dict(x=S(None, p, 4, 8, 16)), dict(bias=p + 2), dict(bias_dtype=2), dict(act=4), dict(act=-1), dict(residual=p + 1),
                dict(rs=5), dict(out=None), dict(ys=5), dict(dtype=3), dict(device=-1)):
        assert dense(**bad) == B.DIPACO_EINVAL, bad

    def pack(x=x, w=w, bias=p, bias_dtype=0, act=3, y=y, a=None, work=p, size=1 << 20, device=0):
        return lib.dipaco_packed_linear_pack(x, w, bias, bias_dtype, act, y, a, work, size, device, None)

    for bad in (dict(x=None), dict(y=None), dict(y=S(p, p, 4, 7, 16)), dict(a=S(p, p, 5, 6, 16)), dict(a=S(p, None, 4, 6, 16)),
                dict(act=5), dict(bias=p + 1), dict(bias_dtype=-1), dict(device=-1)):
        assert pack(**bad) == B.DIPACO_EINVAL, bad
    nothing = dict(x=S(p, p, 4, 0, 16), w=S(p, p, 6, 0, 16))  # sums over nothing alone need a workspace
    for bad in (dict(work=None), dict(work=p + 4), dict(size=16)):
        assert pack(**nothing, **bad) == B.DIPACO_EINVAL, bad
    k = 65537
    assert pack(x=S(p, p, 4, k, k + 15), w=S(p, p, 6, k, k + 15)) == B.DIPACO_ELIMIT
    assert pack(x=S(p, p, 1 << 31, 8, 16), y=S(p, p, 1 << 31, 6, 16)) == B.DIPACO_ELIMIT

    v = S(p, p, 8, 6, 16)

    def back(dy=x, w=v, a=y, act=3, da=y, dbias=p, work=p, size=1 << 20, device=0):
        return lib.dipaco_packed_linear_pack_backward(dy, w, a, act, da, dbias, work, size, device, None)

    for bad in (dict(dy=None), dict(w=w), dict(a=None), dict(a=x), dict(da=None), dict(da=x), dict(act=9), dict(dbias=p + 2), dict(work=None),
                dict(work=p + 8), dict(size=8), dict(device=-1)):
        assert back(**bad) == B.DIPACO_EINVAL, bad
    assert back(dy=S(p, p, 4, k, k + 15), w=S(p, p, k, 6, 16)) == B.DIPACO_ELIMIT


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    x, w = inner.pack(torch.zeros(4, 8, device=DEV)), inner.pack(torch.zeros(6, 8, device=DEV))
    r = torch.zeros(4, 6, device=DEV)
    for bad in (dict(w=inner.pack(torch.zeros(6, 9, device=DEV))), dict(bias=r[0, :5]), dict(bias=r[0].double()), dict(bias=r[0].cpu()),
                dict(bias=torch.zeros(12, device=DEV)[::2]), dict(activation="tanh"), dict(residual=r[:3]), dict(residual=r.t()),
                dict(residual=r, out_dtype=BF16), dict(out_dtype=torch.float16), dict(residual=r.clone().requires_grad_())):
        with pytest.raises(ValueError):
            inner.packed_linear(**{**dict(x=x, w=w), **bad})
    a, v = inner.pack(r), inner.pack(torch.zeros(8, 6, device=DEV))
    for bad in (dict(w=w), dict(a=None), dict(a=x), dict(activation=None), dict(activation="selu")):
        with pytest.raises(ValueError):
            inner.packed_linear_pack_backward(**{**dict(dy=x, w=v, a=a, activation="gelu"), **bad})
    b = torch.zeros(6, device=DEV, requires_grad=True)
    for call in (inner.packed_linear, inner.packed_linear_pack):
        with pytest.raises(ValueError, match="gradient"):
            call(x, w, b)
        with torch.no_grad():
            call(x, w, b)
