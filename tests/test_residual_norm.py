"""The norms around a block with its gate and residual against plain 64-bit implementations.

Tolerances follow the roundings of the kernels' fp32 arithmetic, u = 2^-24: a sum taken as chains of fewer than 96
additions, joined, is off by at most CHAIN = 112 u times the sum of magnitudes.  They are stated value by value
below; a result in bf16 adds half a unit of its last place.
"""
from __future__ import annotations

import itertools
import math

import pytest
import torch

from paper_2403_10616_b200 import binding as B
from paper_2403_10616_b200 import inner
from tests import inner_reference as ref
from tests.test_inner_ops import BF16, CHAIN, DEV, F32, U, assert_within, gen, half, place

NAMES = ("gamma", "beta", "post_gamma", "post_beta")


# ------------------------------------------------------------------ 64 bits

def statistics(v, eps):
    mean = v.mean(1, keepdim=True)
    return mean, 1.0 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + eps)


def or_one(t, v):
    return torch.ones_like(v) if t is None else t.double().expand_as(v)


def or_zero(t, v):
    return torch.zeros_like(v) if t is None else t.double().expand_as(v)


def forward(x, f, p, gate, scale, eps, post_norm, norm, held=lambda z: z):
    """(z, n), differentiable; held rounds z to its type."""
    y = f
    if post_norm:
        mean, rstd = statistics(f, eps)
        y = (f - mean) * rstd * or_one(p["post_gamma"], f) + or_zero(p["post_beta"], f)
    z = scale * x + or_one(gate, f) * y
    if not norm:
        return z, None
    z_held = held(z)
    mean, rstd = statistics(z_held, eps)
    return z, (z_held - mean) * rstd * or_one(p["gamma"], f) + or_zero(p["beta"], f)


def through_norm(u, h, rstd):
    return rstd * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))


def backward(dn, dz, f, z, stats, p, gate, scale, post_norm):
    """The formula's gradients with their tolerances: {name: (value, tolerance)}."""
    mean_f, rstd_f, mean_z, rstd_z = (s.double()[:, None] for s in stats)
    d, tol = (torch.zeros_like(f), torch.zeros_like(f)) if dz is None else (dz.double(), 2 * U * dz.double().abs())
    out = {}

    def average(v, off=0.0):  # of a row, and how far it may be off
        return v.mean(1, keepdim=True), (off + CHAIN * v.abs()).mean(1, keepdim=True)

    def norm_back(q, tol_q, h, rstd):
        mean, off = average(q, tol_q)
        along, off_along = average(q * h, tol_q * h.abs())
        value = rstd * (q - mean - h * along)
        return value, rstd * (tol_q + off + h.abs() * off_along + 8 * U * (q.abs() + mean.abs() + (h * along).abs()))

    def sum_rows(v, off):
        return v.sum(0), off.sum(0) + (CHAIN * v.abs()).sum(0)

    if dn is not None:
        dn = dn.double()
        h = (z - mean_z) * rstd_z
        u = dn * or_one(p["gamma"], f)
        value, off = norm_back(u, 2 * U * u.abs(), h, rstd_z)
        d, tol = d + value, tol + off + 2 * U * (d.abs() + value.abs())
        out["gamma"], out["beta"] = sum_rows(dn * h, 4 * U * (dn * h).abs()), sum_rows(dn, 0 * dn)
    g, post = or_one(gate, f), or_one(p["post_gamma"], f)
    h = (f - mean_f) * rstd_f if post_norm else f
    y = h * post + or_zero(p["post_beta"], f)
    q = d * g * post
    tol_q = tol * (g * post).abs() + 4 * U * q.abs()
    out["x"] = scale * d, abs(scale) * tol + 2 * U * (scale * d).abs()
    out["f"] = norm_back(q, tol_q, h, rstd_f) if post_norm else (q, tol_q)
    if gate is not None:
        # d p as a sum of products with post_gamma and post_beta taken out: the parts' magnitudes count
        parts = (d * h * post).abs() + (d * or_zero(p["post_beta"], f)).abs()
        each, off = d * y, tol * y.abs() + 8 * U * parts
        if gate.shape == f.shape and gate.shape[1] != 1:
            out["gate"] = each, off
        else:
            over = 0 if gate.dim() == 1 else 1
            v = each.sum(over, keepdim=over == 1)
            out["gate"] = v, off.sum(over, keepdim=over == 1) + (CHAIN * parts).sum(over, keepdim=over == 1)
    if post_norm:
        w = d * g
        out["post_gamma"] = sum_rows(w * h, tol * (g * h).abs() + 6 * U * (w * h).abs())
        out["post_beta"] = sum_rows(w, tol * g.abs() + 4 * U * w.abs())
    return out


def test_the_formula_is_the_derivative():
    """Of the forward pass, against central differences in 64 bits."""
    rows, cols, h = 3, 7, 1e-6
    for kind, post_norm, norm in itertools.product((None, "cols", "rows", "full"), (True, False), (True, False)):
        t = {"x": torch.randn(rows, cols, generator=gen(1)), "f": torch.randn(rows, cols, generator=gen(2))}
        t.update({n: torch.randn(cols, generator=gen(3 + i)) for i, n in enumerate(NAMES)
                  if (norm if n in ("gamma", "beta") else post_norm)})
        if kind:
            t["gate"] = torch.rand({"cols": (cols,), "rows": (rows, 1), "full": (rows, cols)}[kind], generator=gen(9))
        t = {k: v.double() for k, v in t.items()}
        dn = torch.randn(rows, cols, generator=gen(10)).double() if norm else None
        dz = torch.randn(rows, cols, generator=gen(11)).double()

        def value(t):
            z, n = forward(t["x"], t["f"], {k: t.get(k) for k in NAMES}, t.get("gate"), 0.7, 1e-5, post_norm, norm)
            return float((z * dz).sum()) + (float((n * dn).sum()) if norm else 0.0)

        z, _ = forward(t["x"], t["f"], {k: t.get(k) for k in NAMES}, t.get("gate"), 0.7, 1e-5, post_norm, norm)
        stats = [s[:, 0] for v in (t["f"], z) for s in statistics(v, 1e-5)]
        found = backward(dn, dz, t["f"], z, stats, {k: t.get(k) for k in NAMES}, t.get("gate"), 0.7, post_norm)
        assert set(found) == set(t)
        for name, leaf in t.items():
            for i in range(leaf.numel()):
                ends = []
                for step in (h, -h):
                    moved = leaf.clone()
                    moved.view(-1)[i] += step
                    ends.append(value({**t, name: moved}))
                slope = (ends[0] - ends[1]) / (2 * h)
                # third derivatives are of order 10: h^2 and the cancellation 1e-16 / h stay far below
                assert abs(slope - float(found[name][0].reshape(-1)[i])) <= 1e-7 * (1 + abs(slope)), (name, i)


# ------------------------------------------------------------------ the kernels

def inputs(rows, cols, dtype, params, kind, post_norm=True, norm=True, pad=0, offset=0, seed=0):
    """(CPU tensors, device tensors): x, f, dn, dz, parameters and gate."""
    host = {}
    for i, name in enumerate(("x", "f", "dn", "dz")):
        v = torch.randn(rows, cols, generator=gen(seed + i)) * (1.0 if i < 2 else 1e-2)
        host[name] = (v + 0.3 * i if i < 2 else v).to(dtype)
    for i, name in enumerate(NAMES):
        wanted = norm if name in ("gamma", "beta") else post_norm
        host[name] = (torch.randn(cols, generator=gen(seed + 5 + i)) * 0.3 + (i % 2 == 0)).to(params) if wanted and params else None
    host["gate"] = None
    if kind:
        shape = {"cols": (cols,), "rows": (rows, 1), "full": (rows, cols)}[kind]
        host["gate"] = (torch.rand(shape, generator=gen(seed + 9)) + 0.1).to(dtype if kind == "full" else params or F32)
    device = {}
    for name, t in host.items():
        if t is None:
            device[name] = None
        elif t.dim() == 2 and t.shape == (rows, cols) and name != "gate" or kind == "full" and name == "gate":
            device[name] = place(t, pad, offset)
        else:
            device[name] = t.to(DEV)
    return host, device


def check_norm(got, mean, rstd, v, gamma, beta, eps, dtype, what):
    """got = LN(v) gamma + beta.  v - mean is off by 4 u of the row's largest magnitude (the corrected mean and one
    rounding), rstd by CHAIN of itself."""
    want_mean, want_rstd = statistics(v, eps)
    top = v.abs().amax(1, keepdim=True)
    assert_within(mean[:, None], want_mean, 4 * U * top + CHAIN * (v - want_mean).abs().mean(1, keepdim=True), what + " mean")
    assert_within(rstd[:, None], want_rstd, (CHAIN + 8 * U * top * want_rstd) * want_rstd, what + " rstd")
    if got is None:
        return
    hat = (v - want_mean) * want_rstd
    off = want_rstd * 6 * U * top + (CHAIN + 8 * U * top * want_rstd) * (1 + hat.abs())
    g, b = or_one(gamma, v), or_zero(beta, v)
    assert_within(got, hat * g + b, off * g.abs() + 4 * U * ((hat * g).abs() + b.abs()), what, dtype)


def run_and_check(rows, cols, dtype, params, kind, post_norm=True, norm=True, pad=0, offset=0, scale=0.8, packed=False):
    host, dev = inputs(rows, cols, dtype, params, kind, post_norm, norm, pad, offset)
    ps = {k: dev[k] for k in NAMES}
    eps = 1e-5
    if packed:
        z, n, kept, stats = inner.residual_norm_pack(dev["x"], dev["f"], **ps, gate=dev["gate"], residual_scale=scale,
                                                     post_norm=post_norm, eps=eps)
    else:
        z, n, stats = inner.residual_norm(dev["x"], dev["f"], **ps, gate=dev["gate"], residual_scale=scale,
                                          post_norm=post_norm, norm=norm, eps=eps)
    what = str((rows, cols, dtype, kind, post_norm, norm))
    x, f, st = host["x"].double(), host["f"].double(), stats.cpu()
    p = {k: host[k] for k in NAMES}
    # z: LN(f) as above, times the gate, with the products' own roundings
    want, _ = forward(x, f, p, host["gate"], scale, eps, post_norm, False)
    g = or_one(host["gate"], f)
    tol = 4 * U * ((scale * x).abs() + (want - scale * x).abs())
    if post_norm:
        check_norm(None, st[0], st[1], f, None, None, eps, dtype, what + " f")
        mean, rstd = statistics(f, eps)
        top = f.abs().amax(1, keepdim=True)
        hat = (f - mean) * rstd
        post, shift = or_one(p["post_gamma"], f), or_zero(p["post_beta"], f)
        off = rstd * 6 * U * top + (CHAIN + 8 * U * top * rstd) * (1 + hat.abs())
        tol = tol + g.abs() * (off * post.abs() + 4 * U * ((hat * post).abs() + shift.abs()))
    else:
        assert bool((st[0] == 0).all()) and bool((st[1] == 1).all())
    assert_within(z, want, tol, what + " z", dtype)
    z_held = z.cpu().double()
    if norm:
        if packed:
            check_norm(None, st[2], st[3], z_held, None, None, eps, dtype, what + " z")
            mean, rstd = (s.double()[:, None] for s in st[2:])
            want_n = (z_held - mean) * rstd * or_one(p["gamma"], f) + or_zero(p["beta"], f)
            ref.assert_packed_close(n.codes, n.scales, want_n, 8 * U * (want_n.abs() + 2 * (1 + (z_held * rstd).abs()) *
                                    or_one(p["gamma"], f).abs()), what + " n")
            codes, scales = ref.pack(z_held)
            assert torch.equal(kept.codes.cpu().double(), codes) and torch.equal(kept.scales.cpu().double(), scales)
        else:
            check_norm(n, st[2], st[3], z_held, p["gamma"], p["beta"], eps, dtype, what + " n")
    else:
        assert n is None and bool((st[2] == 0).all()) and bool((st[3] == 1).all())

    # the gradients, from the forward pass's own results, or checkpoints of them
    fd, zd = dev["f"], place(z.cpu(), pad, offset)
    fv, zv = f, z_held
    if packed:
        fd, zd = inner.pack(dev["f"]), kept
        fv, zv = ref.values(fd.codes, fd.scales), ref.values(kept.codes, kept.scales)
    for with_dz in (True, False):
        if not with_dz and not norm:
            continue
        got = inner.residual_norm_backward(dev["dn"] if norm else None, dev["dz"] if with_dz else None, fd,
                                           zd if norm else None, stats, dev["gamma"], dev["post_gamma"], dev["post_beta"],
                                           dev["gate"], scale, post_norm)
        wanted = backward(host["dn"] if norm else None, host["dz"] if with_dz else None, fv, zv, st, p, host["gate"], scale,
                          post_norm)
        for name in got._fields:
            g = getattr(got, name)
            assert (g is None) == (name not in wanted), (what, name)
            if g is not None:
                v, tol = wanted[name]
                assert g.shape == v.shape and g.dtype == (dtype if name in ("x", "f") or g.shape == (rows, cols) and cols > 1 and name == "gate" and kind == "full" else F32)
                assert_within(g, v, tol, what + " d" + name, g.dtype)


SIZES = [(1, 1), (1, 896), (2, 3), (3, 8), (5, 17), (70, 33), (4, 255), (40, 256), (3, 257), (33, 896), (20, 1023), (9, 2048),
         (6, 2047), (7, 2500), (3, 4096), (4, 5000), (3, 8192), (2, 8193), (2, 16384), (2, 20001)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sizes(rows, cols, dtype):
    run_and_check(rows, cols, dtype, dtype, "cols")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [None, "cols", "rows", "full"])
@pytest.mark.parametrize("post_norm,norm", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("dtype,params", [(F32, F32), (BF16, F32), (BF16, BF16), (BF16, None)])
def test_gates_and_norms_left_out(kind, post_norm, norm, dtype, params):
    for rows, cols in ((5, 96), (12, 896), (3, 1001)):
        run_and_check(rows, cols, dtype, params, kind, post_norm, norm)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["cols", "full"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (3, 5), (16, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_inside_wider_buffers_at_any_alignment(pad, offset, dtype, kind):
    for rows, cols in ((6, 128), (5, 897), (4, 2048)):
        run_and_check(rows, cols, dtype, F32, kind, pad=pad, offset=offset)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 896), (130, 129), (300, 200), (128, 2048), (3, 5000), (40, 9000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_results_and_checkpoints(rows, cols, dtype):
    run_and_check(rows, cols, dtype, F32, "cols", packed=True)
    run_and_check(rows, cols, dtype, F32, "rows", post_norm=False, packed=True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype", [(5000, 64, F32), (3001, 896, BF16), (2000, 2048, BF16), (1500, 1001, F32)])
def test_many_rows(rows, cols, dtype):
    run_and_check(rows, cols, dtype, F32, "cols")
    run_and_check(rows, cols, dtype, F32, "rows")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_hardly_vary_and_rows_of_zeros(dtype):
    """A row of equal values has the result beta (within what the corrected mean is off), not noise times 1/sqrt(eps)."""
    f = torch.stack((torch.full((896,), 1000.1), torch.zeros(896), 1000.0 + 1e-3 * torch.randn(896, generator=gen(1)))).to(dtype)
    x = torch.zeros_like(f)
    z, n, stats = inner.residual_norm(x.to(DEV), f.to(DEV))
    v = f.double()
    mean, rstd = statistics(v, 1e-5)
    # the corrected mean is off by a rounding of itself, u * 1000, and so is every difference
    assert_within(z, (v - mean) * rstd, rstd * 2 * U * v.abs() + 1e-3 * ((v - mean) * rstd).abs() + CHAIN, "z", dtype)
    assert float(z[1].abs().max()) == 0.0 and bool(torch.isfinite(n).all())


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows():
    for dtype in (F32, BF16):
        x, f = torch.randn(6, 300, generator=gen(1)).to(dtype), torch.randn(6, 300, generator=gen(2)).to(dtype)
        f[1, 7], f[3, 299], x[4, 0] = math.nan, math.inf, -math.inf
        z, n, stats = inner.residual_norm(x.to(DEV), f.to(DEV))
        assert torch.isfinite(n.cpu()).all(1).tolist() == [True, False, True, False, False, True]
        dn = torch.ones_like(z)
        got = inner.residual_norm_backward(dn, None, f.to(DEV), z, stats)
        assert torch.isfinite(got.f.cpu()).all(1).tolist() == [True, False, True, False, False, True]
        assert torch.isfinite(got.x.cpu()).all(1).tolist() == [True, False, True, False, False, True]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,pad", [(17, 255, 0), (300, 264, 0), (161, 512, 1), (5, 4096, 0), (5, 4097, 0), (4, 4104, 1), (3, 6144, 0),
                                           (3, 6145, 0), (160, 6152, 0), (2, 8191, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_widths_around_which_threads_take_other_shares(rows, cols, pad, dtype):
    run_and_check(rows, cols, dtype, F32, "cols", pad=pad)
    run_and_check(rows, cols, dtype, F32, "full", pad=pad)


@pytest.mark.gpu
def test_an_infinite_gate_meets_no_zero_that_nobody_gave():
    for dtype in (F32, BF16):
        f = torch.randn(3, 40, generator=gen(3)).to(dtype).to(DEV)
        gate = torch.ones(40, device=DEV)
        gate[5] = math.inf
        z, _, _ = inner.residual_norm(torch.zeros_like(f), f, gate=gate, post_norm=False, norm=False)
        assert torch.equal(z.float(), gate * f.float())
        z, _, _ = inner.residual_norm(torch.zeros_like(f), f, post_gamma=torch.ones(40, device=DEV), gate=gate, norm=False)
        assert bool((z[:, 5] == math.inf * torch.sign(f[:, 5].float() - f.float().mean(1))).all())


@pytest.mark.gpu
@pytest.mark.parametrize("cols,stride,at", [(896, 1 << 30, 0), (1001, (1 << 30) + 1, 3), (9000, 1 << 30, 0)])
def test_rows_whose_offsets_pass_32_bits(cols, stride, at):
    """Three rows of bf16 over 4 GB apart have the results of the same rows, placed the same way within 16 bytes, side by side."""
    _, d = inputs(3, cols, BF16, F32, "full")

    def far(t):
        hold = torch.empty(2 * stride + at + cols, dtype=BF16, device=DEV)
        view = hold.as_strided((3, cols), (stride, 1), at)
        view.copy_(t)
        return view

    def near(t):
        return place(t.cpu(), stride % 8 + 8 - cols % 8, at)

    results = []
    for put in (near, far):
        x, f, gate = put(d["x"]), put(d["f"]), put(d["gate"])
        z, n, stats = inner.residual_norm(x, f, *(d[k] for k in NAMES), gate, 0.5)
        del x
        z_far, dn, dz = put(z), put(d["dn"]), put(d["dz"])
        back = inner.residual_norm_backward(dn, dz, f, z_far, stats, d["gamma"], d["post_gamma"], d["post_beta"], gate, 0.5)
        results.append((z, n, stats, *back))
        del f, gate, z_far, dn, dz
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_no_rows_and_no_columns():
    for dtype in (F32, BF16):
        for rows, cols in ((0, 5), (4, 0), (0, 0)):
            x = torch.empty(rows, cols, dtype=dtype, device=DEV)
            z, n, stats = inner.residual_norm(x, x, gate=torch.ones(rows, 1, device=DEV))
            assert z.shape == n.shape == (rows, cols) and (stats.numel() == 0 or bool(torch.isnan(stats).all()))
            got = inner.residual_norm_backward(x, x, x, x, stats, gate=torch.ones(rows, 1, device=DEV))
            assert got.gamma.shape == (cols,) and bool((got.gamma == 0).all()) and bool((got.post_beta == 0).all())
            assert bool((got.gate == 0).all())
            got = inner.residual_norm_backward(x, x, x, x, stats, gate=torch.ones(cols, device=DEV))
            assert bool((got.gate == 0).all())


@pytest.mark.gpu
def test_results_do_not_depend_on_the_stream_and_are_the_same_again():
    _, d = inputs(700, 896, BF16, BF16, "cols")
    call = lambda: inner.residual_norm(d["x"], d["f"], *(d[k] for k in NAMES), d["gate"], 0.5)  # noqa: E731
    z, n, stats = call()
    back = lambda: inner.residual_norm_backward(d["dn"], d["dz"], d["f"], z, stats, d["gamma"], d["post_gamma"],  # noqa: E731
                                                d["post_beta"], d["gate"], 0.5)
    first = [*call(), *back()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = [*call(), *back()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = [*call(), *back()]
    for t in third:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


# ------------------------------------------------------------------ refusals

def test_bad_arguments_are_refused():
    """By the library, before any CUDA call."""
    args = lambda **k: B.ResidualNormStruct(**{**dict(rows=4, cols=8, gate_kind=0, gate_dtype=0, dtype=0, param_dtype=0,  # noqa: E731
                                                      post_norm=1, norm=1, residual_scale=1.0, eps=1e-5), **k})
    lib = B.load()
    p = 1 << 20  # never read

    def forward_status(a, x=p, xs=8, f=p, z=p, n=p, stats=p, device=0):
        return lib.dipaco_residual_norm(a, x, xs, f, 8, z, 8, n, 8, None, None, stats, device, None)

    for bad in (dict(rows=-1), dict(dtype=2), dict(param_dtype=-1), dict(gate_dtype=7), dict(eps=math.nan), dict(eps=-1.0),
                dict(residual_scale=math.inf), dict(gate_kind=4), dict(gate_kind=-1), dict(gate_kind=1), dict(gate=p + 2, gate_kind=1),
                dict(gate=p, gate_kind=3, gate_stride=7), dict(gate=p, gate_kind=3, gate_stride=8, gate_dtype=1),
                dict(gamma=p + 1), dict(post_norm=0, post_beta=p), dict(norm=0, gamma=p), dict(norm=0)):
        assert forward_status(args(**bad)) == B.DIPACO_EINVAL, bad
    for bad in (dict(x=None), dict(xs=7), dict(f=p + 1), dict(z=None), dict(stats=None), dict(stats=p + 2), dict(device=-1)):
        assert forward_status(args(), **bad) == B.DIPACO_EINVAL, bad
    assert forward_status(args(rows=1 << 31)) == B.DIPACO_ELIMIT

    def back_status(a, dn=p, dz=p, f=p, z=p, stats=p, dgate=None, dgamma=p, dpost=p, work=p, size=1 << 20):
        return lib.dipaco_residual_norm_backward(a, dn, 8, dz, 8, f, 8, None, z, 8, None, stats, p, 8, p, 8, dgate, 8, dgamma,
                                                 None, dpost, None, work, size, 0, None)

    for bad in (dict(dn=None), dict(f=None), dict(z=None), dict(stats=None), dict(dgate=p), dict(work=None), dict(work=p + 8),
                dict(size=16), dict(dz=p + 2), dict(dgamma=p + 1)):
        assert back_status(args(), **bad) == B.DIPACO_EINVAL, bad
    assert back_status(args(norm=0)) == B.DIPACO_EINVAL              # dn without norm
    assert back_status(args(post_norm=0)) == B.DIPACO_EINVAL         # a gradient of nothing


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    x = torch.zeros(4, 8, device=DEV)
    stats = torch.zeros(4, 4, device=DEV)
    for bad in (dict(f=x[:, :7]), dict(f=x.to(BF16)), dict(f=x.cpu()), dict(f=x.t()), dict(gamma=x[0, :7]), dict(gamma=x[0].double()),
                dict(gamma=x[0], beta=x[0].to(BF16)), dict(gate=x[:3]), dict(gate=x.to(BF16)), dict(gate=x[:, 0]),
                dict(post_gamma=x[0], post_norm=False), dict(beta=x[0], norm=False)):
        with pytest.raises(ValueError):
            inner.residual_norm(**{**dict(x=x, f=x), **bad})
    for bad in (dict(dn=None, dz=None), dict(f=None), dict(z=None), dict(stats=stats[:3]), dict(stats=stats.t()), dict(dz=x[:3]),
                dict(f=inner.pack(x[:3])), dict(dn=x.to(torch.float16))):
        with pytest.raises(ValueError):
            inner.residual_norm_backward(**{**dict(dn=x, dz=x, f=x, z=x, stats=stats), **bad})
    w = torch.zeros(8, device=DEV, requires_grad=True)
    for bad in (dict(gamma=w), dict(gate=w), dict(x=x.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            inner.residual_norm(**{**dict(x=x, f=x), **bad})
        with torch.no_grad():
            inner.residual_norm(**{**dict(x=x, f=x), **bad})
