"""Further operators of a path's inner training phase, measured: linear layers on packed matrices with bias,
activation and residual in their epilogue, the norms after and before a block fused with its gate and its
scaled residual, and the clipping of a path's gradients by their common norm.

A path of the mixture is a transformer of 12 blocks of width 896 (150M parameters) or of 24 blocks of width
2048; its feed-forward part is four times as wide.  A training step of a path sees up to 65536 tokens, an
evaluation step a handful or one.

Linear layers (x [tokens, in], w [out, in], both packed):
  dense     act(x w^T + bias) + residual, in bf16 or fp32
  pack      a = x w^T + bias and act(a), both packed: the operand of the next layer and the checkpoint
  back      da = (dy w) act'(a) packed, from the packed dy [tokens, out] and a [tokens, in], and its column sums
Norms of the rows, LN(v) = (v - mean v) / sqrt(var v + eps):
  p = LN(f) post_gamma + post_beta,  z = scale x + gate p  (held in x's type),  n = LN(z) gamma + beta,
  and the gradients of x, f, gate and the parameters from those of z and n
Clipping: the norm of all gradients together, and all of them in one vector, times min(1, most / norm).

Packed matrices: e4m3 codes with one power-of-two scale (an e8m0 byte) for each block of 128 x 128 values,
the smallest that brings the block's largest finite magnitude to at most 448.

``run`` computes the plain form with torch's elementary operations in 32 bits, or, where ``own`` is set,
calls the library's operators.  ``exact`` states the same in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5

# work limits of a drawn case: those of the largest listed ones
MOST_VALUES = 32768 * 3584
MOST_ROW_VALUES = 16384 * 2048
MOST_PRODUCTS = 16384 * 2048 * 8192
MOST_GRADIENTS = 144_000_000


def listed():
    return [
        # one token goes through the widening layer of a block when a path answers: latency of one call
        {"name": "linear: one token", "op": "linear", "form": "pack", "m": 1, "n": 3584, "k": 896,
         "activation": "gelu", "bias": "bf16", "keep": False},
        # the widening layer of a training step, 32 sequences of 1024 tokens: operand and checkpoint
        {"name": "linear: widening", "op": "linear", "form": "pack", "m": 32768, "n": 3584, "k": 896,
         "activation": "gelu", "bias": "bf16", "keep": True},
        # the narrowing layer of the wide model, added to the residual stream
        {"name": "linear: narrowing", "op": "linear", "form": "dense", "m": 16384, "n": 2048, "k": 8192,
         "activation": None, "bias": "bf16", "residual": True, "out": "bf16"},
        # the backward pass through the narrowing layer and the activation before it
        {"name": "linear: activation gradient", "op": "linear", "form": "back", "m": 32768, "n": 3584, "k": 896,
         "activation": "gelu", "bias": "f32"},
        # a ragged batch through a layer of odd widths, in 32 bits
        {"name": "linear: odd sizes", "op": "linear", "form": "dense", "m": 4999, "n": 1001, "k": 2047,
         "activation": "silu", "bias": "f32", "residual": True, "out": "f32"},
        # one token between two blocks when a path answers
        {"name": "norms: one token", "op": "norms", "rows": 1, "cols": 896, "pad": 0, "dtype": "bf16",
         "params": "bf16", "gate": "cols", "packed": False},
        # between two blocks of the wide model, 16 sequences of 1024 tokens, kept in bf16
        {"name": "norms: wide model", "op": "norms", "rows": 16384, "cols": 2048, "pad": 0, "dtype": "bf16",
         "params": "bf16", "gate": "cols", "packed": False},
        # between two blocks of a training step that keeps 8-bit checkpoints
        {"name": "norms: 8-bit checkpoints", "op": "norms", "rows": 32768, "cols": 896, "pad": 0, "dtype": "bf16",
         "params": "bf16", "gate": "cols", "packed": True},
        # their gradient in the wide model
        {"name": "norms back: wide model", "op": "norms back", "rows": 16384, "cols": 2048, "pad": 0,
         "dtype": "bf16", "params": "bf16", "gate": "cols", "packed": False},
        # a ragged batch of an odd width, gated token by token, in 32 bits
        {"name": "norms back: odd sizes", "op": "norms back", "rows": 4999, "cols": 2047, "pad": 0, "dtype": "f32",
         "params": "f32", "gate": "rows", "packed": False},
        # the six gradients of one feed-forward block of a small mixture
        {"name": "clip: one block", "op": "clip", "width": 256, "blocks": 1, "vocabulary": 0, "odd": 0,
         "dtype": "f32", "share": 0.5},
        # all gradients of a path: 12 blocks and the embedding
        {"name": "clip: a path", "op": "clip", "width": 896, "blocks": 12, "vocabulary": 32000, "odd": 0,
         "dtype": "f32", "share": 0.1},
    ]


def _size(rng, low, high):
    """A whole number of [low, high], spread over the logarithm; half of them multiples of 64 or 8."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    unit = rng.choice((1, 1, 8, 64))
    return max(low, min(high, n // unit * unit))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear", "norms", "norms back", "norms back", "clip"))
    if op == "linear":
        form = rng.choice(("dense", "pack", "back"))
        m, n, k = _size(rng, 1, 65536), _size(rng, 32, 8192), _size(rng, 32, 8192)
        while m * n * k > MOST_PRODUCTS or m * n > MOST_VALUES:
            m = max(1, m // 2)
        case = {"op": op, "form": form, "m": m, "n": n, "k": k, "bias": rng.choice(("f32", "bf16")),
                "activation": rng.choice(("relu", "silu", "gelu"))}
        if form == "dense":
            case["activation"] = rng.choice((None, case["activation"]))
            case["residual"] = rng.random() < 0.6
            case["out"] = rng.choice(("bf16", "bf16", "f32"))
        elif form == "pack":
            case["keep"] = rng.random() < 0.7
        return case
    if op == "clip":
        case = {"op": op, "width": _size(rng, 16, 1024), "blocks": rng.randint(1, 24), "vocabulary": 0,
                "odd": rng.choice((0, 0, 1, 3)), "dtype": rng.choice(("f32", "f32", "bf16")),
                "share": rng.choice((0.03, 0.5, 4.0))}
        while _gradients(case) > MOST_GRADIENTS:
            case["blocks"] -= 1
        return case
    dtype = rng.choice(("bf16", "bf16", "f32"))
    case = {"op": op, "rows": _size(rng, 1, 65536), "cols": _size(rng, 16, 8192),
            "pad": rng.choice((0, 0, 1, 8, 128)), "dtype": dtype, "params": rng.choice((dtype, "f32")),
            "gate": rng.choice(("cols", "cols", "rows", "full")), "packed": rng.random() < 0.4}
    while case["rows"] * case["cols"] * (2 if dtype == "f32" else 1) > MOST_ROW_VALUES:
        case["rows"] = max(1, case["rows"] // 2)
    return case


def _shapes(case):
    """The gradients' shapes: a block's norm, its two products with their biases, four products of the attention."""
    c = case["width"]
    w = c + case["odd"]
    block = [(c,), (c,), (4 * c, w), (4 * c,), (c, 4 * c), (w,)]
    if case["vocabulary"]:
        block += [(c, c)] * 4
    return block * case["blocks"] + ([(case["vocabulary"], c)] if case["vocabulary"] else [])


def _gradients(case):
    return sum(math.prod(s) for s in _shapes(case))


def _packed_bytes(rows, cols):
    return rows * cols + -(-rows // BLOCK) * -(-cols // BLOCK)


def work(case):
    if case["op"] == "linear":
        m, n, k, form = case["m"], case["n"], case["k"], case["form"]
        moved = _packed_bytes(m, k) + (_packed_bytes(k, n) if form == "back" else _packed_bytes(n, k))
        if form == "dense":
            moved += n * BYTES[case["bias"]] + (2 if case["residual"] else 1) * m * n * BYTES[case["out"]]
        elif form == "pack":
            moved += n * BYTES[case["bias"]] + (2 if case["keep"] else 1) * _packed_bytes(m, n)
        else:
            moved += 2 * _packed_bytes(m, n) + 4 * n
        return {"bytes": moved, "flops": 2.0 * m * n * k}
    if case["op"] == "clip":
        n = _gradients(case)
        return {"bytes": n * (BYTES[case["dtype"]] + 4) + 4, "flops": 3.0 * n}
    r, c, b = case["rows"], case["cols"], BYTES[case["dtype"]]
    each = r * c
    gate = {"cols": c * BYTES[case["params"]], "rows": 4 * r, "full": b * each}[case["gate"]]
    if case["op"] == "norms":
        written = b * each + (2 * _packed_bytes(r, c) if case["packed"] else b * each) + 16 * r
        return {"bytes": 2 * b * each + gate + 4 * c * BYTES[case["params"]] + written, "flops": 20.0 * each}
    read = 2 * (_packed_bytes(r, c) if case["packed"] else b * each) + 2 * b * each + 16 * r + gate
    params = 3 * c * BYTES[case["params"]] + 16 * c
    dgate = {"cols": 4 * c, "rows": 4 * r, "full": b * each}[case["gate"]]
    return {"bytes": read + params + 2 * b * each + dgate, "flops": 36.0 * each}


# ------------------------------------------------------------------ inputs

def _rows(gen, case, std, outliers=False):
    """A [rows, cols] matrix inside a buffer `pad` values wider: normal values, a few columns larger."""
    r, c = case["rows"], case["cols"]
    t = torch.empty(r, c + case["pad"], device=DEV, dtype=DTYPES[case["dtype"]])
    t.normal_(0.0, std, generator=gen)
    if outliers:
        wide = torch.empty(c + case["pad"], device=DEV).uniform_(0, 1, generator=gen)
        t.mul_(torch.where(wide < 0.01, 12.0, 1.0).to(t.dtype))
        t.add_(torch.empty(r, 1, device=DEV, dtype=t.dtype).normal_(0.0, 0.2 * std, generator=gen))
    return t[:, :c]


def _spread(scale, rows, cols):
    """A block's value at each of its elements."""
    return scale.repeat_interleave(BLOCK, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _quantised(x):
    """(codes, scales) of a matrix in 32 bits: elementary operations only."""
    r, c = x.shape
    rb, cb = -(-r // BLOCK), -(-c // BLOCK)
    mag = torch.nn.functional.pad(x.abs(), (0, cb * BLOCK - c, 0, rb * BLOCK - r))
    mag = torch.where(torch.isfinite(mag), mag, torch.zeros_like(mag))
    amax = mag.view(rb, BLOCK, cb, BLOCK).amax(dim=(1, 3))
    part, exponent = torch.frexp(amax)                       # amax = part * 2^exponent, 1/2 <= part < 1
    exponent = exponent - 9 + (part > 0.875).to(exponent.dtype)    # 448 = 0.875 * 2^9
    exponent = torch.where(amax > 0, exponent.clamp(min=-126), torch.zeros_like(exponent))
    scale = torch.ldexp(torch.ones_like(amax), exponent)
    codes = (x * _spread(1.0 / scale, r, c)).to(torch.float8_e4m3fn)
    return codes, scale.to(torch.float8_e8m0fnu)


def _held(codes, scales):
    """Packed data as a program holds it: rows of codes at multiples of 16 bytes."""
    r, c = codes.shape
    hold = torch.empty(r, -(-c // 16) * 16, device=DEV, dtype=torch.float8_e4m3fn)
    hold[:, :c].copy_(codes)
    return hold[:, :c], scales


def _values(packed):
    codes, scales = packed
    return codes.float() * _spread(scales.float(), *codes.shape)


def _random_packed(gen, rows, cols, std):
    """The packed form of normal values whose size differs between blocks."""
    x = torch.empty(rows, cols, device=DEV).normal_(0.0, std, generator=gen)
    size = torch.empty(-(-rows // BLOCK), -(-cols // BLOCK), device=DEV).normal_(0.0, 0.5, generator=gen)
    return _held(*_quantised(x * _spread(torch.exp(size), rows, cols)))


def _vector(gen, n, dtype, mean, std):
    return torch.empty(n, device=DEV).normal_(mean, std, generator=gen).to(DTYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    op = case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        if case["form"] == "back":
            state["dy"] = _random_packed(gen, m, k, 1e-3)
            state["w"] = _random_packed(gen, k, n, k ** -0.5)
            state["a"] = _random_packed(gen, m, n, 1.5)
            return state
        state["x"] = _random_packed(gen, m, k, 1.0)
        state["w"] = _random_packed(gen, n, k, k ** -0.5)
        state["bias"] = _vector(gen, n, case["bias"], 0.0, 0.3)
        if case["form"] == "dense":
            state["residual"] = None
            if case["residual"]:
                state["residual"] = torch.empty(m, n, device=DEV).normal_(0.0, 2.0, generator=gen).to(DTYPES[case["out"]])
        return state
    if op == "clip":
        # the larger a parameter's fan-in the smaller its gradient, and a few values stand out
        state["grads"] = []
        total = 0.0
        for shape in _shapes(case):
            g = torch.empty(shape, device=DEV).normal_(0.0, shape[-1] ** -0.5, generator=gen)
            g.view(-1)[:: 97].mul_(8.0)
            state["grads"].append(g.to(DTYPES[case["dtype"]]))
            total += math.prod(shape) / shape[-1] * (1 + 63 / 97)
        state["most"] = case["share"] * math.sqrt(total)  # over, near or under the norm
        return state
    r, c, params = case["rows"], case["cols"], case["params"]
    state["scale"] = 0.9
    for name, mean in (("gamma", 1.0), ("beta", 0.0), ("post_gamma", 1.0), ("post_beta", 0.0)):
        state[name] = _vector(gen, c, params, mean, 0.1)
    if case["gate"] == "cols":
        state["gate"] = _vector(gen, c, params, 0.3, 0.1)
    elif case["gate"] == "rows":
        state["gate"] = torch.sigmoid(_vector(gen, r, "f32", 0.0, 1.0)).view(r, 1)
    else:
        state["gate"] = torch.sigmoid(_rows(gen, case, 1.0).float()).to(DTYPES[case["dtype"]])
    state["f"] = _rows(gen, case, 0.5, outliers=True)
    if op == "norms":
        state["x"] = _rows(gen, case, 1.0, outliers=True)
        return state
    z, f = _rows(gen, case, 1.0, outliers=True), state["f"]
    state["dn"], state["dz"] = _rows(gen, case, 1e-3), _rows(gen, case, 1e-3)
    stats = []
    for t in (f.float(), z.float()):
        mean = t.mean(1)
        stats += [mean, torch.rsqrt((t - mean[:, None]).square().mean(1) + EPS)]
    state["stats"] = torch.stack(stats)
    state["z"] = z
    if case["packed"]:
        state["f"], state["z"] = _held(*_quantised(f.float())), _held(*_quantised(z.float()))
    return state


# ------------------------------------------------------------------ one pass

ROOT_2_PI = math.sqrt(2.0 / math.pi)
CUBIC = 0.044715


def _activated(a, name):
    if name == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a))
    if name == "silu":
        return a / (1.0 + torch.exp(-a))
    if name == "gelu":
        return 0.5 * a * (1.0 + torch.tanh(ROOT_2_PI * (a + CUBIC * a * a * a)))
    return a


def _slope(a, name):
    if name == "relu":
        return (a > 0).to(a.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return s * (1.0 + a * (1.0 - s))
    t = torch.tanh(ROOT_2_PI * (a + CUBIC * a * a * a))
    return 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * ROOT_2_PI * (1.0 + 3.0 * CUBIC * a * a)


def _normal(v):
    mean = v.mean(1)
    centred = v - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + EPS)
    return centred * rstd[:, None], mean, rstd


def _normal_back(dy, hat, rstd):
    return (dy - dy.mean(1, keepdim=True) - hat * (dy * hat).mean(1, keepdim=True)) * rstd[:, None]


def _plain_norms(s, case):
    x, f = s["x"].float(), s["f"].float()
    hat, mean_f, rstd_f = _normal(f)
    p = hat * s["post_gamma"].float() + s["post_beta"].float()
    z = (s["scale"] * x + s["gate"].float() * p).to(s["x"].dtype)
    hat, mean_z, rstd_z = _normal(z.float())
    n = hat * s["gamma"].float() + s["beta"].float()
    stats = torch.stack((mean_f, rstd_f, mean_z, rstd_z))
    if case["packed"]:
        return (z, *_quantised(n), *_quantised(z.float()), stats)
    return z, n.to(z.dtype), stats


def _plain_norms_back(s, case):
    f = _values(s["f"]) if case["packed"] else s["f"].float()
    z = _values(s["z"]) if case["packed"] else s["z"].float()
    mean_f, rstd_f, mean_z, rstd_z = s["stats"]
    dn, gate, gamma, post = (s[t].float() for t in ("dn", "gate", "gamma", "post_gamma"))
    hat_f, hat_z = (f - mean_f[:, None]) * rstd_f[:, None], (z - mean_z[:, None]) * rstd_z[:, None]
    dz = s["dz"].float() + _normal_back(dn * gamma, hat_z, rstd_z)
    dp = dz * gate
    dgate = dz * (hat_f * post + s["post_beta"].float())
    if case["gate"] == "full":
        dgate = dgate.to(s["dn"].dtype)
    else:
        dgate = dgate.sum(0) if case["gate"] == "cols" else dgate.sum(1, keepdim=True)
    df = _normal_back(dp * post, hat_f, rstd_f)
    return ((s["scale"] * dz).to(s["dn"].dtype), df.to(s["dn"].dtype), dgate, (dn * hat_z).sum(0), dn.sum(0),
            (dp * hat_f).sum(0), dp.sum(0))


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "linear":
        if case["form"] == "back":
            da = (_values(s["dy"]) @ _values(s["w"])) * _slope(_values(s["a"]), case["activation"])
            return (*_quantised(da), da.sum(0))
        a = _values(s["x"]) @ _values(s["w"]).t() + s["bias"].float()
        y = _activated(a, case["activation"])
        if case["form"] == "pack":
            return (*_quantised(y), *_quantised(a)) if case["keep"] else _quantised(y)
        return (y if s["residual"] is None else y + s["residual"].float()).to(DTYPES[case["out"]])
    if op == "clip":
        flat = torch.cat([g.reshape(-1).float() for g in s["grads"]])
        norm = flat.double().square().sum().sqrt()
        return flat * torch.clamp(s["most"] / norm, max=1.0).float(), norm.float()
    return _plain_norms(s, case) if op == "norms" else _plain_norms_back(s, case)


def _library(s):
    from paper_2403_10616_b200 import inner
    case = s["case"]
    op = case["op"]
    if op == "linear":
        w = inner.Packed(*s["w"])
        if case["form"] == "back":
            da, dbias = inner.packed_linear_pack_backward(inner.Packed(*s["dy"]), w, inner.Packed(*s["a"]),
                                                          case["activation"])
            return da.codes, da.scales, dbias
        x = inner.Packed(*s["x"])
        if case["form"] == "pack":
            y, a = inner.packed_linear_pack(x, w, s["bias"], case["activation"], keep=case["keep"])
            return (y.codes, y.scales, a.codes, a.scales) if case["keep"] else (y.codes, y.scales)
        return inner.packed_linear(x, w, s["bias"], case["activation"], s["residual"], out_dtype=DTYPES[case["out"]])
    if op == "clip":
        return inner.gather_gradients(s["grads"], s["most"])
    if op == "norms":
        call = inner.residual_norm_pack if case["packed"] else inner.residual_norm
        out = call(s["x"], s["f"], s["gamma"], s["beta"], s["post_gamma"], s["post_beta"], s["gate"], s["scale"], eps=EPS)
        if case["packed"]:
            z, n, kept, stats = out
            return z, n.codes, n.scales, kept.codes, kept.scales, stats
        return out
    f, z = (inner.Packed(*s["f"]), inner.Packed(*s["z"])) if case["packed"] else (s["f"], s["z"])
    g = inner.residual_norm_backward(s["dn"], s["dz"], f, z, s["stats"], s["gamma"], s["post_gamma"], s["post_beta"],
                                     s["gate"], s["scale"])
    return g.x, g.f, g.gate, g.gamma, g.beta, g.post_gamma, g.post_beta


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------ 64 bits

def _packed_exactly(v):
    """Codes and scales from the definition: scale 2^e with the least e such that max|v| <= 448 * 2^e;
    a code is the nearest multiple of the spacing of e4m3 (three bits after the leading one, down to
    2^-9), the even one of two."""
    codes, scales = torch.empty_like(v), []
    for i in range(0, v.shape[0], BLOCK):
        line = torch.stack([part.abs().max() for part in v[i:i + BLOCK].split(BLOCK, 1)])
        e = torch.ceil(torch.log2(line / 448.0))
        e = torch.where(line > 448.0 * torch.exp2(e), e + 1, e)
        e = torch.where(line <= 448.0 * torch.exp2(e - 1), e - 1, e)
        scale = torch.where(line > 0, torch.exp2(e.clamp(min=-126)), torch.ones_like(line))
        t = v[i:i + BLOCK] / scale.repeat_interleave(BLOCK)[:v.shape[1]]
        spacing = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        codes[i:i + BLOCK] = torch.round(t / spacing) * spacing
        scales.append(scale)
    return codes, torch.stack(scales)


def _unpacked_exactly(packed):
    codes, scales = packed
    out = codes.double()
    for i in range(scales.shape[0]):
        at = slice(i * BLOCK, (i + 1) * BLOCK)
        out[at] *= scales[i].double().repeat_interleave(BLOCK)[:out.shape[1]]
    return out


def _share(a, name):
    """(s, ds/da) of an activation a * s(a)."""
    if name is None:
        return torch.ones_like(a), torch.zeros_like(a)
    if name == "relu":
        return (a > 0).double(), torch.zeros_like(a)
    # (1 + tanh u) / 2 = sigmoid(2u)
    u = a if name == "silu" else 2.0 * ROOT_2_PI * (a + CUBIC * a ** 3)
    du = 1.0 if name == "silu" else 2.0 * ROOT_2_PI * (1.0 + 3.0 * CUBIC * a ** 2)
    s = torch.sigmoid(u)
    return s, s * (1.0 - s) * du


def _standardised(v):
    var, mean = torch.var_mean(v, dim=1, unbiased=False)
    rstd = 1.0 / torch.sqrt(var + EPS)
    return (v - mean[:, None]) * rstd[:, None], mean, rstd


def _through_norm(g, hat, rstd):
    """The norm's Jacobian, (I - 1 1^T / C - hat hat^T / C) rstd, times g."""
    c = g.shape[1]
    along = torch.einsum("rc,rc->r", g, hat) / c
    return torch.addcmul(g - (g.sum(1) / c)[:, None], hat, along[:, None], value=-1.0) * rstd[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        w = _unpacked_exactly(s["w"])
        if case["form"] == "back":
            a = _unpacked_exactly(s["a"])
            share, change = _share(a, case["activation"])
            da = _unpacked_exactly(s["dy"]).matmul(w) * torch.addcmul(share, a, change)
            return (*_packed_exactly(da), torch.einsum("rc->c", da))
        a = torch.addmm(s["bias"].double(), _unpacked_exactly(s["x"]), w.transpose(0, 1))
        y = a * _share(a, case["activation"])[0]
        if case["form"] == "pack":
            return (*_packed_exactly(y), *_packed_exactly(a)) if case["keep"] else _packed_exactly(y)
        return y if s["residual"] is None else y + s["residual"].double()
    if op == "clip":
        flat = torch.cat([g.double().flatten() for g in s["grads"]])
        norm = torch.linalg.vector_norm(flat)
        return flat * min(1.0, s["most"] / float(norm)), norm
    gate, scale = s["gate"].double(), s["scale"]
    gamma, beta, post, shift = (s[name].double() for name in ("gamma", "beta", "post_gamma", "post_beta"))
    if op == "norms":
        hat, mean_f, rstd_f = _standardised(s["f"].double())
        z = torch.addcmul(scale * s["x"].double(), gate, torch.addcmul(shift, hat, post))
        kept = z.to(s["x"].dtype).double()  # what the stream holds, of which n is the norm
        hat, mean_z, rstd_z = _standardised(kept)
        n, stats = torch.addcmul(beta, hat, gamma), torch.stack((mean_f, rstd_f, mean_z, rstd_z))
        return (z, *_packed_exactly(n), *_packed_exactly(kept), stats) if case["packed"] else (z, n, stats)
    mean_f, rstd_f, mean_z, rstd_z = s["stats"].double()
    f, z = (_unpacked_exactly(s[t]) if case["packed"] else s[t].double() for t in ("f", "z"))
    f, z = (f - mean_f[:, None]) * rstd_f[:, None], (z - mean_z[:, None]) * rstd_z[:, None]
    dn = s["dn"].double()
    dz = s["dz"].double() + _through_norm(dn * gamma, z, rstd_z)
    sums = {"cols": "rc,rc->c", "rows": "rc,rc->r", "full": "rc,rc->rc"}[case["gate"]]
    dgate = torch.einsum(sums, dz, torch.addcmul(shift, f, post)).reshape(gate.shape)
    dp = dz * gate
    return (scale * dz, _through_norm(dp * post, f, rstd_f), dgate, torch.einsum("rc,rc->c", dn, z), dn.sum(0),
            torch.einsum("rc,rc->c", dp, f), dp.sum(0))
