"""Edges of the operators around a block, the linear layers and clipping, against 64 bits.

Tolerances are those of the operators' own tests (``check_norm``, ``product_tolerance``) unless stated.
"""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref
from tests.test_inner_ops import BF16, CHAIN, DEV, F32, U, assert_within, gen, packed_operand, place, product_tolerance
from tests.test_packed_linear import act
from tests.test_residual_norm import NAMES, backward, check_norm, forward, inputs, or_one, or_zero, statistics

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ norms around a block

@pytest.mark.parametrize("cols", [264, 520, 640, 1280, 2560, 5000, 7176])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", [None, "cols", "rows", "full"])
def test_a_partly_filled_unit_adds_nothing_to_the_second_norm(cols, dtype, kind):
    """Units behind a row hold zeros, which the norm of f takes far away where its mean is large beside its spread."""
    rows, eps = 6, 1e-5
    f = torch.stack([100.0 + torch.randn(cols, generator=gen(1)), torch.full((cols,), 100.0), torch.full((cols,), 100.0),
                     torch.full((cols,), -3.0e4), 1000.0 + 10 * torch.randn(cols, generator=gen(2)),
                     torch.randn(cols, generator=gen(3))]).to(dtype)
    x = torch.stack([torch.randn(cols, generator=gen(4)), torch.randn(cols, generator=gen(5)), torch.full((cols,), 4.0),
                     torch.full((cols,), 1.5), 30.0 + torch.randn(cols, generator=gen(6)),
                     torch.randn(cols, generator=gen(7))]).to(dtype)
    gamma, beta = torch.randn(cols, generator=gen(8)) * 0.3 + 1.0, torch.randn(cols, generator=gen(9)) * 0.3
    post, shift = torch.randn(cols, generator=gen(10)) * 0.3 + 1.0, torch.zeros(cols)
    gate = None
    if kind:
        gate = (torch.rand({"cols": (cols,), "rows": (rows, 1), "full": (rows, cols)}[kind], generator=gen(11)) + 0.5).to(dtype)
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    given = (on(gamma), on(beta), on(post), on(shift), on(gate), 0.5)
    z, n, stats = inner.residual_norm(on(x), on(f), *given)
    st, held = stats.cpu(), z.cpu().double()
    what = str((cols, dtype, kind))
    check_norm(None, st[0], st[1], f.double(), None, None, eps, dtype, what + " f")
    check_norm(n, st[2], st[3], held, gamma, beta, eps, dtype, what + " n")
    z_too, n_too, kept, stats_too = inner.residual_norm_pack(on(x), on(f), *given)
    assert torch.equal(z, z_too) and torch.equal(stats, stats_too)
    mean, rstd = (s.double()[:, None] for s in st[2:])
    want = (held - mean) * rstd * gamma.double() + beta.double()
    ref.assert_packed_close(n_too.codes, n_too.scales, want,
                            8 * U * (want.abs() + 2 * (1 + (held * rstd).abs()) * gamma.double().abs()), what + " packed")


@pytest.mark.parametrize("cols", [40, 37, 896, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gate_of_columns_multiplies_the_shifted_norm(cols, dtype):
    """gate (LN(f) post_gamma + post_beta), of a gate that is infinite, or too large for its product with post_gamma."""
    f = torch.randn(3, cols, generator=gen(1)).to(dtype)
    f[1] = 0.0
    f[1, 0], f[1, 1] = 1.0, -1.0                       # the mean is zero, and so is the norm of the others
    post, shift, gate = torch.ones(cols), torch.zeros(cols), torch.ones(cols)
    gate[5], gate[6] = math.inf, -math.inf
    shift[6], post[7], gate[7], shift[7] = 1000.0, 1e25, 1e25, 2.0
    on = lambda t: t.to(DEV)  # noqa: E731
    z, _, stats = inner.residual_norm(torch.zeros_like(on(f)), on(f), None, None, on(post), on(shift), on(gate), norm=False)
    z, mean = z.cpu().float(), stats[0].cpu()
    for row in (0, 2):
        assert float(z[row, 5]) == math.inf * (1 if f[row, 5] > mean[row] else -1)
    assert bool((z[:, 6] == -math.inf).all())          # the shift is larger than any row's values
    assert abs(float(z[1, 7]) / 2e25 - 1.0) <= (2.0 ** -8 if dtype == BF16 else 4 * U)
    assert float(z[1, 8]) == 0.0 and bool(torch.isnan(z[1, 5]))  # an infinite gate times a norm of zero


@pytest.mark.parametrize("cols", [5, 33, 40, 264, 300, 2000, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_infinity_at_a_row_s_end_counts_once_in_the_gradient_of_its_gate(cols, dtype):
    """Without the norm after the block dgate = sum dz f, which is infinite where f is and dz is not zero."""
    f, dz = torch.randn(4, cols, generator=gen(1)).to(dtype), torch.randn(4, cols, generator=gen(2)).to(dtype)
    f[1, cols - 1], f[2, 0] = math.inf, -math.inf
    dz[1, cols - 1], dz[2, 0] = 2.0, 3.0
    stats = torch.stack([torch.zeros(4), torch.ones(4), torch.zeros(4), torch.ones(4)]).to(DEV)
    got = inner.residual_norm_backward(None, dz.to(DEV), f.to(DEV), None, stats, gate=torch.ones(4, 1, device=DEV),
                                       post_norm=False)
    gate = got.gate.cpu().view(-1)
    assert float(gate[1]) == math.inf and float(gate[2]) == -math.inf
    each = dz.double() * f.double()
    for row in (0, 3):
        assert abs(float(gate[row]) - float(each[row].sum())) <= CHAIN * float(each[row].abs().sum())
    assert torch.equal(got.f.cpu(), dz)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gate_of_every_value_in_rows_of_one(dtype):
    """It has the shape of a gate of rows, and is one where it lies like one."""
    x, f, dn = (torch.randn(5, 1, generator=gen(i)).to(dtype).to(DEV) for i in range(3))
    gate = (torch.rand(5, 1, generator=gen(3)) + 0.5).to(dtype)
    together, apart = gate.to(DEV), place(gate, 3, 1)
    results = []
    for g in (together, apart):
        z, n, stats = inner.residual_norm(x, f, gate=g, post_norm=False)
        results.append((z, n, stats, *(t for t in inner.residual_norm_backward(dn, dn, f, z, stats, gate=g, post_norm=False)
                                       if t is not None)))
    assert results[0][5].dtype == F32 and results[1][5].dtype == dtype
    for a, b in zip(*results):
        assert torch.equal(a.to(b.dtype), b)
    with pytest.raises(ValueError):
        inner.residual_norm(x.expand(5, 2).contiguous(), f.expand(5, 2).contiguous(), gate=apart)


MATRICES = ("x", "f", "dn", "dz", "gate", "z")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 128), (6, 896), (4, 2048), (3, 8192), (3, 8200)])
def test_matrices_of_one_call_at_different_alignments(rows, cols, dtype):
    """One matrix at a time off the 16-byte boundaries that the others keep to: the results are those of the formula."""
    host, dev = inputs(rows, cols, dtype, F32, "full")
    ps, scale, eps = {k: dev[k] for k in NAMES}, 0.8, 1e-5
    p = {k: host[k] for k in NAMES}
    base = inner.residual_norm(dev["x"], dev["f"], **ps, gate=dev["gate"], residual_scale=scale)
    held = base[0].cpu()
    for odd in MATRICES:
        at = {k: place(host[k] if k != "z" else held, 3, 1) if k == odd else (dev[k] if k != "z" else base[0]) for k in MATRICES}
        z, n, stats = inner.residual_norm(at["x"], at["f"], **ps, gate=at["gate"], residual_scale=scale)
        st, zv = stats.cpu(), z.cpu().double()
        check_norm(None, st[0], st[1], host["f"].double(), None, None, eps, dtype, odd + " f")
        check_norm(n, st[2], st[3], zv, p["gamma"], p["beta"], eps, dtype, odd + " n")
        want, _ = forward(host["x"].double(), host["f"].double(), p, host["gate"].double(), scale, eps, True, False)
        mean, rstd = statistics(host["f"].double(), eps)
        hat, top = (host["f"].double() - mean) * rstd, host["f"].double().abs().amax(1, keepdim=True)
        post, shift = or_one(p["post_gamma"], hat), or_zero(p["post_beta"], hat)
        off = rstd * 6 * U * top + (CHAIN + 8 * U * top * rstd) * (1 + hat.abs())
        tol = 4 * U * ((scale * host["x"].double()).abs() + (want - scale * host["x"].double()).abs())
        tol = tol + host["gate"].double() * (off * post.abs() + 4 * U * ((hat * post).abs() + shift.abs()))
        assert_within(z, want, tol, odd + " z", dtype)
        stats = base[2]
        got = inner.residual_norm_backward(at["dn"], at["dz"], at["f"], at["z"], stats, dev["gamma"], dev["post_gamma"],
                                           dev["post_beta"], at["gate"], scale)
        wanted = backward(host["dn"], host["dz"], host["f"].double(), held.double(), stats.cpu(), p, host["gate"], scale, True)
        for name in got._fields:
            v, tol = wanted[name]
            assert_within(getattr(got, name), v, tol, odd + " d" + name, getattr(got, name).dtype)


# ------------------------------------------------------------------ clipping

@pytest.mark.parametrize("sizes", [(100, 4), (300_000, 7, 500_000)])
def test_without_a_limit_a_nan_stays_where_it_is(sizes):
    g = [torch.randn(n, generator=gen(i)).to(BF16 if i == 1 else F32) for i, n in enumerate(sizes)]
    g[0][5], g[1][0] = math.nan, math.inf
    dev = [t.to(DEV) for t in g]
    want = torch.cat([t.float() for t in g])
    for call in (lambda: inner.gather_gradients(dev), lambda: inner.gather_gradients(dev, math.inf)):
        flat, norm = call()
        assert math.isnan(float(norm))
        assert torch.equal(torch.isnan(flat.cpu()).nonzero(), torch.tensor([[5]]))
        assert torch.equal(flat.cpu().nan_to_num(), want.nan_to_num())
    assert math.isnan(float(inner.clip_gradients(dev, math.inf)))
    for t, h in zip(dev, g):
        assert torch.equal(t.cpu().nan_to_num(), h.nan_to_num())


@pytest.mark.parametrize("sizes", [(0, 0), (7,), (100, 4, 0, 9000), (300_000, 7, 500_001), (9, 8200) * 700])
def test_gathering_without_a_limit_or_the_norm_copies(sizes):
    g = [torch.randn(n, generator=gen(i)).to(BF16 if i % 2 else F32) for i, n in enumerate(sizes)]
    for t in g[:1]:
        t[:1] = math.nan
    dev = [t.to(DEV) for t in g]
    for dtype in (F32, BF16):
        flat, norm = inner.gather_gradients(dev, dtype=dtype, norm=False)
        want = torch.cat([t.to(dtype) for t in g])
        assert norm is None and torch.equal(torch.isnan(flat.cpu()), torch.isnan(want))
        assert torch.equal(flat.cpu().nan_to_num(), want.nan_to_num())
    dev = [t.nan_to_num() for t in dev]
    with_norm, norm = inner.gather_gradients(dev, 0.5)
    without, none = inner.gather_gradients(dev, 0.5, norm=False)
    assert none is None and torch.equal(with_norm, without)


def test_copies_need_no_workspace():
    t = torch.randn(900_000, generator=gen(1)).to(DEV)
    out, norm = torch.zeros_like(t), torch.zeros((), device=DEV)
    longs, ints = ctypes.c_int64 * 1, ctypes.c_int32 * 1

    def call(most, norm_ptr):
        B.dipaco_clip_gradients(longs(t.data_ptr()), longs(out.data_ptr()), longs(t.numel()), ints(0), ints(0), 1, most,
                                norm_ptr, None, 0, 0, torch.cuda.current_stream().cuda_stream)

    call(math.inf, None)
    assert torch.equal(out, t)
    for most, norm_ptr in ((1.0, None), (math.inf, norm.data_ptr())):
        with pytest.raises(B.DipacoError):
            call(most, norm_ptr)


@pytest.mark.parametrize("sizes", [(99_999,), (100_000,), (100_001,), (60_000, 40_000, 1), (1600,) * 63, (526_080,)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_numbers_of_values_around_which_a_cluster_gives_way(sizes, dtype):
    g = [torch.randn(n, generator=gen(i)).to(dtype) for i, n in enumerate(sizes)]
    whole = torch.cat(g).double()
    total = float(whole.norm())
    flat, norm = inner.gather_gradients([t.to(DEV) for t in g], 0.25 * total)
    assert abs(float(norm) - total) <= 24 * U * total
    assert_within(flat, whole * 0.25, 26 * U * whole.abs() * 0.25, "gathered")
    # in one launch by one cluster, without a workspace, while that takes no longer than all SMs
    need = B.dipaco_clip_gradients_workspace((ctypes.c_int64 * len(sizes))(*sizes), len(sizes))
    assert (need == 0) == (sum(sizes) <= 100_000)


@pytest.mark.parametrize("n", [1000, 900_000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_factor_that_fp32_hardly_holds(n, dtype):
    """Gradients near the largest value, clipped to a norm whose share of theirs is subnormal in fp32."""
    t = (torch.randn(n, generator=gen(1)).clamp(-3, 3) * 1e38).to(dtype)
    total = float(t.double().square().sum().sqrt())
    for most in (1.0, 1e-2, 1e-4):
        want = t.double() * (most / total)
        off = 26 * U * want.abs() + 2.0 ** -149
        flat, norm = inner.gather_gradients([t.to(DEV)], most)
        assert float(norm) == math.inf or abs(float(norm) - total) <= 24 * U * total
        assert_within(flat, want, off, str(most))
        own = t.to(DEV)
        inner.clip_gradients([own], most)
        assert_within(own, want, off, str(most), dtype)


# ------------------------------------------------------------------ linear layers

@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("shift", [-0.5, -2.0, -3.0, -5.0, -12.0, -30.0])
@pytest.mark.parametrize("m", [3, 300])
def test_tails_of_the_activations(name, shift, m):
    """y = a s with s = 1 / (1 + 2^e): e is off by 4 u of itself, and with it 2^e by 4 u |e| ln 2 of itself; the power, the
    sum, the reciprocal and the product by 8 u more.  What a is off counts by the slope there, which is at most
    |y| (1 + k) for the exponent's slope k.  Powers over 2^126 leave nothing."""
    n = 200
    x, xv = packed_operand(1, m, 100, 0.02)
    w, wv = packed_operand(2, n, 100, 0.02)
    bias = torch.randn(n, generator=gen(3)) * 0.01 + shift
    a = xv @ wv.t() + bias.double()
    tol_a = product_tolerance(xv, wv.t(), 100) + 2 * U * (a.abs() + bias.double().abs())
    if name == "gelu":
        e, k = 2 * ref.ROOT * (a + ref.CUBIC * a ** 3), 2 * ref.ROOT * (1 + 3 * ref.CUBIC * a ** 2)
    else:
        e, k = a, torch.ones_like(a)
    y = act(a, name).float().double()  # packed from its fp32 value, which may be nothing
    over = y.abs() * (4 * U * e.abs() + 8 * U) + (y.abs() * (1 / a.abs() + 1.01 * k)) * tol_a + 40 * 2.0 ** -126
    got, kept = inner.packed_linear_pack(x, w, bias.to(DEV), name)
    ref.assert_packed_close(got.codes, got.scales, y, over, (name, shift))
    ref.assert_packed_close(kept.codes, kept.scales, a, tol_a, (name, shift, "a"))
    dense = inner.packed_linear(x, w, bias.to(DEV), name, out_dtype=F32)
    assert_within(dense, y, over, (name, shift, "dense"))


@pytest.mark.parametrize("name", [None, "relu", "gelu"])
@pytest.mark.parametrize("m,n,k", [(100, 130, 8200), (300, 520, 8192), (70, 40, 65536), (300, 300, 65500), (9000, 1300, 10300)])
def test_bias_gradients_over_long_sums_of_one_sign(m, n, k, name):
    """Sums over up to 8192 values are taken in one go, longer ones in parts of 2048.  Of a part the tensor cores lose at most
    2^-25 for each product and 2^-23 for every 32 of them; joining parts, u for each; the tokens' sums, under 100 additions
    one after another."""
    def positive(seed, rows, cols):
        x = torch.exp(1.5 * torch.randn(rows, cols, generator=gen(seed))).to(DEV)  # sums with bits to lose
        p = inner.pack(x)
        return p, p.codes.double() * ref.spread(p.scales.double(), rows, cols)

    dy, dyv = positive(1, m, k)
    w, wv = positive(2, k, n)
    a = inner.pack(torch.full((m, n), 30.0, device=DEV))  # slopes of one
    da, dbias = inner.packed_linear_pack_backward(dy, w, None if name is None else a, name)
    part, each = k if k <= 8192 else 2048, dyv @ wv
    lost = part * 2.0 ** -25 + part / 32 * 2.0 ** -23 + k / 2048 * U
    want = each.sum(0)
    off = ((dbias.double() - want) / want).abs()
    assert float(off.max()) <= lost + CHAIN, float(off.max())
    ref.assert_packed_close(da.codes, da.scales, each.cpu(), (lost + 2 * U) * each.cpu())
    again, _ = inner.packed_linear_pack_backward(dy, w, None if name is None else a, name, bias=False)
    assert torch.equal(again.codes.view(torch.uint8), da.codes.view(torch.uint8))
    assert inner.inner_status() == B.DIPACO_OK
