"""Plain 64-bit forms of the operators on a paged cache's contents, and how far 16- and 8-bit results may be from them."""
import math

import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
SMALL = 2.0 ** -100


def half_step(dtype) -> float:
    """Half a step of a floating type, relative to the value."""
    return torch.finfo(dtype).eps / 2


def generator(seed: int):
    return torch.Generator().manual_seed(seed)


# ---- rotary positions --------------------------------------------------------------------------------------------
def frequencies(rot, base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0):
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if factor == 1.0:
        return f
    out = []
    for x in f:
        w = 0.0
        if original > 0:
            w = min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low)))
        out.append(x * (w + (1 - w) / factor))
    return out


def rotate(x, pos, freq, interleaved, magnitude=1.0):
    """x [tokens, heads, dim] in 64 bits, its first 2 len(freq) dimensions rotated by pos."""
    x = x.double().clone()
    n = len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        c = torch.cos(pos.double() * f)[:, None] * magnitude
        s = torch.sin(pos.double() * f)[:, None] * magnitude
        x[..., a], x[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return x


# ---- 8-bit codes -------------------------------------------------------------------------------------------------
def codes_of(x, dtype):
    """(codes, scale) of vectors x [..., dim] in fp32, step by step as the header says."""
    x = x.float()
    top = x.abs().amax(-1)
    finite = torch.isfinite(x).all(-1)
    small = top < SMALL
    scale = torch.where(small, torch.ones_like(top), top / LARGEST[dtype])
    mul = torch.where(small, torch.zeros_like(top), torch.full_like(top, LARGEST[dtype]) / torch.where(small, 1.0, top))
    # (a number divided by a tensor would be the tensor's reciprocal times the number: two roundings)
    y = x * mul[..., None]
    y = torch.where(finite[..., None], y, 0.0)
    codes = y.to(dtype) if dtype is torch.float8_e4m3fn else torch.round(y).to(torch.int8)
    return codes, torch.where(finite, scale, math.nan)


def held(data, scale):
    """The values that a plane stands for, in 64 bits."""
    return data.double() if scale is None else data.double() * scale.double()[..., None]


# ---- attention ---------------------------------------------------------------------------------------------------
def attend(q, keys, values, table, seq, pos, scale, window=0, block=16):
    """q [tokens, heads, dim]; keys, values: [n_blocks, block, kv heads, dim] in 64 bits.  Returns (out, lse, weight sums of
    |v|, score bound): the last two say how far a result may be off (see ``tolerance``)."""
    T, Hq, D = q.shape
    n_blocks, block, H, _ = keys.shape
    G = Hq // H
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    mass = torch.zeros(T, Hq, D, dtype=torch.float64)
    size = torch.zeros(T, Hq, dtype=torch.float64)
    for t in range(T):
        s, p = int(seq[t]), int(pos[t])
        if s < 0 or s >= table.shape[0] or p < 0 or p >= table.shape[1] * block:
            continue
        at = torch.arange(max(0, p - window + 1) if window else 0, p + 1)
        entry = table[s].long()[at // block]
        at, entry = at[(entry >= 0) & (entry < n_blocks)], entry[(entry >= 0) & (entry < n_blocks)]
        if not len(at):
            continue
        k, v = keys[entry, at % block], values[entry, at % block]               # [n, H, D]
        for h in range(Hq):
            x = (k[:, h // G] @ q[t, h].double()) * scale
            size[t, h] = ((k[:, h // G].abs() @ q[t, h].double().abs()).max() + q[t, h].double().abs().max() * k[:, h // G].abs().sum(1).max() / 8) \
                * abs(scale)
            top = x.max()
            if top == -math.inf:
                continue
            w = torch.exp(x - top)
            lse[t, h] = top + torch.log(w.sum())
            w = w / w.sum()
            out[t, h], mass[t, h] = w @ v[:, h // G], w @ v[:, h // G].abs()
    return out, lse, mass, size


def tolerance(out, mass, size, lens, dim, out_dtype, weight_dtype, scales=None):
    """Bounds of (out, lse), element by element.

    A score is off by the roundings of its `dim` products' sum, one step each at the size of all of them together, and of
    three fp32 operations on it: d = size * (dim + 16) * 2^-23 in all.  (8-bit caches: queries in fp16 are off by at most 2^-24 of
    the row's largest, which `size` has room for, and the scale of a value enters by its logarithm: up to 2^-21 and one
    step of |log2 scale|.)  The exponential adds 2^-21.  A weight is then off by d + 2^-21 relative to itself, the
    normalised one by twice that; its rounding to `weight_dtype` adds half a step; adding n terms adds n steps of
    2^-24, twice (numerator and sum)."""
    d = size * (dim + 16) * 2.0 ** -23 + 2.0 ** -21
    if scales is not None:
        d = d + 2.0 ** -20 + (scales.log2().abs().max() + 4) * 2.0 ** -23
    n = torch.as_tensor(lens, dtype=torch.float64)[:, None]
    rel = 2 * d + n * 2.0 ** -23 + half_step(weight_dtype)
    least = torch.finfo(out_dtype).smallest_normal * half_step(out_dtype) * 2
    return rel[..., None] * mass + half_step(out_dtype) * out.abs() + least, d + n * 2.0 ** -24 + 2.0 ** -20 * (1 + size)
