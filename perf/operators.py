"""The operators of a path's inner training phase, measured: layer norm with its gradient, activation
checkpoints in 8 bits with their use in the backward pass, and the products of packed matrices.

A path of the mixture is a transformer of 12 blocks of width 896 (150M parameters) or of 24 blocks of
width 2048; its feed-forward part is four times as wide.  A training step of a path sees up to
65536 tokens, an evaluation step a handful or one.

Packed matrices: e4m3 codes with one power-of-two scale (an e8m0 byte) for each block of 128 x 128
values, the smallest that brings the block's largest finite magnitude to at most 448.

``run`` computes the plain form with torch's elementary operations in 32 bits, or, where ``own`` is
set, calls the library's operators.  ``exact`` states the same in 64 bits.
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
MOST_PRODUCTS = 16384 * 2048 * 8192


def listed():
    return [
        # a single token is normalised when a path answers: the latency of one call
        {"name": "norm, one token", "op": "norm", "rows": 1, "cols": 896, "pad": 0, "dtype": "bf16",
         "params": "bf16", "stats": False, "packed": False},
        # the norm before a block of the wide model, 16 sequences of 1024 tokens, kept in bf16
        {"name": "norm, wide model", "op": "norm", "rows": 16384, "cols": 2048, "pad": 0, "dtype": "bf16",
         "params": "bf16", "stats": True, "packed": False},
        # the norm of a training step that leaves nothing but 8-bit checkpoints: its result, which the
        # next product reads, and its input, which the backward pass reads
        {"name": "norm, 8-bit checkpoints", "op": "norm", "rows": 32768, "cols": 896, "pad": 0,
         "dtype": "bf16", "params": "bf16", "stats": True, "packed": True},
        # the gradient in 32 bits, an odd width and an odd number of tokens inside a wider buffer
        {"name": "norm back, odd sizes", "op": "norm back", "rows": 4999, "cols": 2047, "pad": 2,
         "dtype": "f32", "params": "f32", "packed": False},
        # the gradient from the 8-bit checkpoint of the norm's input
        {"name": "norm back, from 8 bits", "op": "norm back", "rows": 32768, "cols": 2048, "pad": 0,
         "dtype": "bf16", "params": "bf16", "packed": True},
        # a weight matrix packed at the start of a step
        {"name": "pack, a weight", "op": "pack", "rows": 3584, "cols": 896, "pad": 0, "dtype": "f32"},
        # the activation of a training step: its result and its input, both packed
        {"name": "gelu, 8-bit checkpoints", "op": "gelu", "rows": 32768, "cols": 3584, "pad": 0,
         "dtype": "bf16"},
        # its gradient, read from the checkpoint, packed for the two products that follow
        {"name": "gelu back, from 8 bits", "op": "gelu back", "rows": 32768, "cols": 3584, "pad": 0,
         "dtype": "bf16"},
        # one token through the widening product
        {"name": "product, one token", "op": "product", "form": "forward", "m": 1, "n": 3584, "k": 896,
         "out": "bf16"},
        # 32 sequences of 1024 tokens through the widening product
        {"name": "product, forward", "op": "product", "form": "forward", "m": 32768, "n": 3584, "k": 896,
         "out": "bf16"},
        # the gradient of the input of the wide model's widening product
        {"name": "product, input gradient", "op": "product", "form": "input", "m": 16384, "n": 2048,
         "k": 8192, "out": "bf16"},
        # a weight's gradient, summed over a ragged batch of tokens, in 32 bits
        {"name": "product, weight gradient", "op": "product", "form": "weight", "m": 3584, "n": 896,
         "k": 65501, "out": "f32"},
    ]


def _size(rng, low, high):
    """A whole number of [low, high], spread over the logarithm; half of them multiples of 64 or 8."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    unit = rng.choice((1, 1, 8, 64))
    return max(low, min(high, n // unit * unit))


def draw(rng):
    op = rng.choice(("norm", "norm back", "pack", "gelu", "gelu back", "product", "product"))
    if op == "product":
        form = rng.choice(("forward", "input", "weight"))
        m, n, k = _size(rng, 1, 65536), _size(rng, 32, 8192), _size(rng, 32, 8192)
        while m * n * k > MOST_PRODUCTS:
            m = max(1, m // 2)
        if form == "weight":
            m, k = k, m
        out = "f32" if form == "weight" else rng.choice(("bf16", "bf16", "f32"))
        return {"op": op, "form": form, "m": m, "n": n, "k": k, "out": out}
    dtype = rng.choice(("bf16", "bf16", "f32"))
    case = {"op": op, "rows": _size(rng, 1, 65536), "cols": _size(rng, 16, 8192),
            "pad": rng.choice((0, 0, 1, 8, 128)), "dtype": dtype}
    while case["rows"] * case["cols"] * (2 if dtype == "f32" else 1) > MOST_VALUES:
        case["rows"] = max(1, case["rows"] // 2)
    if op.startswith("norm"):
        case["params"] = rng.choice((dtype, "f32"))
        case["packed"] = rng.random() < 0.5
    if op == "norm":
        case["stats"] = case["packed"] or rng.random() < 0.7
    return case


def work(case):
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        blocks = -(-m // BLOCK) + -(-n // BLOCK)
        return {"bytes": m * k + n * k + blocks * -(-k // BLOCK) + m * n * BYTES[case["out"]],
                "flops": 2.0 * m * n * k}
    r, c, b = case["rows"], case["cols"], BYTES[case["dtype"]]
    each, scales = r * c, -(-r // BLOCK) * -(-c // BLOCK)
    packed = each + scales
    if case["op"] == "norm":
        weights = 2 * c * BYTES[case["params"]]
        written = 2 * packed if case["packed"] else b * each
        return {"bytes": b * each + weights + written + (8 * r if case["stats"] else 0), "flops": 8.0 * each}
    if case["op"] == "norm back":
        read = (packed if case["packed"] else b * each) + b * each + 8 * r + c * BYTES[case["params"]]
        return {"bytes": read + b * each + 8 * c, "flops": 14.0 * each}
    if case["op"] == "pack":
        return {"bytes": b * each + packed, "flops": 3.0 * each}
    if case["op"] == "gelu":
        return {"bytes": b * each + 2 * packed, "flops": 16.0 * each}
    return {"bytes": b * each + 2 * packed, "flops": 24.0 * each}


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
    size = torch.empty(-(-rows // BLOCK), -(-cols // BLOCK), device=DEV).normal_(0.0, 1.0, generator=gen)
    return _held(*_quantised(x * _spread(torch.exp(size), rows, cols)))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    op = case["op"]
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        shape_a = (k, m) if case["form"] == "weight" else (m, k)
        shape_b = (n, k) if case["form"] == "forward" else (k, n)
        state["a"] = _random_packed(gen, *shape_a, 1.0)
        state["b"] = _random_packed(gen, *shape_b, 0.02)
        return state
    c = case["cols"]
    if op.startswith("norm"):
        dt = DTYPES[case["params"]]
        state["gamma"] = torch.empty(c, device=DEV).normal_(1.0, 0.1, generator=gen).to(dt)
        state["beta"] = torch.empty(c, device=DEV).normal_(0.0, 0.1, generator=gen).to(dt)
        state["x"] = _rows(gen, case, 1.0, outliers=True)
        if op == "norm back":
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = torch.rsqrt((x - state["mean"][:, None]).square().mean(1) + EPS)
            state["dy"] = _rows(gen, case, 1e-3)
            if case["packed"]:
                state["x"] = _held(*_quantised(x))
        return state
    if op == "pack":
        state["x"] = _rows(gen, case, 0.02)
    elif op == "gelu":
        state["x"] = _rows(gen, case, 1.5)
    else:
        state["x"] = _held(*_quantised(_rows(gen, dict(case, pad=0), 1.5).float()))
        state["dy"] = _rows(gen, case, 1e-3)
    return state


# ------------------------------------------------------------------ one pass

ROOT_2_PI = math.sqrt(2.0 / math.pi)
CUBIC = 0.044715


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "product":
        a, b = _values(s["a"]), _values(s["b"])
        a = a.t() if case["form"] == "weight" else a
        b = b.t() if case["form"] == "forward" else b
        return (a @ b).to(DTYPES[case["out"]])
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        centred = x - mean[:, None]
        rstd = torch.rsqrt(centred.square().mean(1) + EPS)
        y = centred * rstd[:, None] * s["gamma"].float() + s["beta"].float()
        if not case["packed"]:
            y = y.to(s["x"].dtype)
            return (y, mean, rstd) if case["stats"] else (y,)
        return (*_quantised(y), *_quantised(x), mean, rstd)
    if op == "norm back":
        x = _values(s["x"]) if case["packed"] else s["x"].float()
        dy = s["dy"].float()
        hat = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["gamma"].float()
        dx = (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) * s["rstd"][:, None]
        return dx.to(s["dy"].dtype), (dy * hat).sum(0), dy.sum(0)
    if op == "pack":
        return _quantised(s["x"].float())
    if op == "gelu":
        a = s["x"].float()
        h = 0.5 * a * (1.0 + torch.tanh(ROOT_2_PI * (a + CUBIC * a * a * a)))
        return (*_quantised(h), *_quantised(a))
    a = _values(s["x"])
    t = torch.tanh(ROOT_2_PI * (a + CUBIC * a * a * a))
    slope = 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * ROOT_2_PI * (1.0 + 3.0 * CUBIC * a * a)
    return _quantised(s["dy"].float() * slope)


def _library(s):
    from paper_2403_10616_b200 import inner
    case = s["case"]
    op = case["op"]
    if op == "product":
        return inner.packed_matmul(inner.Packed(*s["a"]), inner.Packed(*s["b"]),
                                   transpose_a=case["form"] == "weight",
                                   transpose_b=case["form"] == "forward", out_dtype=DTYPES[case["out"]])
    if op == "norm":
        if case["packed"]:
            y, x, mean, rstd = inner.layer_norm_pack(s["x"], s["gamma"], s["beta"], eps=EPS)
            return y.codes, y.scales, x.codes, x.scales, mean, rstd
        if case["stats"]:
            return inner.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS, stats=True)
        return (inner.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS),)
    if op == "norm back":
        x = inner.Packed(*s["x"]) if case["packed"] else s["x"]
        return inner.layer_norm_backward(s["dy"], x, s["mean"], s["rstd"], s["gamma"])
    if op == "pack":
        p = inner.pack(s["x"])
        return p.codes, p.scales
    if op == "gelu":
        h, a = inner.gelu_pack(s["x"])
        return h.codes, h.scales, a.codes, a.scales
    p = inner.gelu_pack_backward(s["dy"], inner.Packed(*s["x"]))
    return p.codes, p.scales


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------ 64 bits

def _packed_exactly(v):
    """Codes and scales from the definition: scale 2^e with the least e such that max|v| <= 448 * 2^e;
    a code is the nearest multiple of the spacing of e4m3 (three bits after the leading one, down to
    2^-9), the even one of two."""
    codes, scales = torch.empty_like(v), []
    for i in range(0, v.shape[0], BLOCK):
        line = []
        for j in range(0, v.shape[1], BLOCK):
            block = v[i:i + BLOCK, j:j + BLOCK]
            line.append(block.abs().max())
        line = torch.stack(line)
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


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        a, b = _unpacked_exactly(s["a"]), _unpacked_exactly(s["b"])
        if case["form"] == "forward":
            return a.matmul(b.transpose(0, 1))
        return a.transpose(0, 1).matmul(b) if case["form"] == "weight" else a.matmul(b)
    if op == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["beta"].double(), (x - mean[:, None]) * rstd[:, None], s["gamma"].double())
        if case["packed"]:
            return (*_packed_exactly(y), *_packed_exactly(x), mean, rstd)
        return (y, mean, rstd) if case["stats"] else (y,)
    if op == "norm back":
        x = _unpacked_exactly(s["x"]) if case["packed"] else s["x"].double()
        dy, n = s["dy"].double(), case["cols"]
        hat = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        g = dy * s["gamma"].double()
        along = torch.einsum("rc,rc->r", g, hat) / n
        dx = (g - (g.sum(1) / n)[:, None] - hat * along[:, None]) * s["rstd"].double()[:, None]
        return dx, torch.einsum("rc,rc->c", dy, hat), dy.sum(0)
    if op == "pack":
        return _packed_exactly(s["x"].double())
    # a * sigmoid(2u) is the same function: (1 + tanh u) / 2 = sigmoid(2u)
    a = _unpacked_exactly(s["x"]) if op == "gelu back" else s["x"].double()
    share = torch.sigmoid(2.0 * ROOT_2_PI * (a + CUBIC * a ** 3))
    if op == "gelu":
        return (*_packed_exactly(a * share), *_packed_exactly(a))
    slope = share + a * share * (1.0 - share) * (2.0 * ROOT_2_PI) * (1.0 + 3.0 * CUBIC * a ** 2)
    return _packed_exactly(s["dy"].double() * slope)
