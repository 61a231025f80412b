"""Plain 64-bit forms of the cache operators (rotation, 4-bit and FP8 codes, attention), from their definitions, on the CPU.

Nothing here is used by the product path.
"""
from __future__ import annotations

import torch


def rotate(x, cos, sin, pos, rot, interleaved):
    """x [T, H, d] in float64, rotated; and the bound |x| + |partner| that a product's rounding is relative to."""
    y, size = x.clone(), torch.zeros_like(x)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size[..., i], size[..., j] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, size


def rounded_close(got, want, size, dtype):
    """got is `want` rounded once to `dtype` after fp32 arithmetic whose terms have magnitudes `size`: each of the two products and the
    sum is off by half a unit of fp32 at most (2^-24 of `size` for both products together, 2^-24 of the result), and half a
    unit of the type (2^-8 of the result in bf16) comes on top."""
    tol = 2.0 ** -23 * size + 2.0 ** -24 * want.abs() + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
    return bool(((got.double() - want).abs() <= tol).all())


# ---------------------------------------------------------------- 4-bit rows
def scale_value(byte):
    e, m = (byte.long() >> 3).double(), (byte.long() & 7).double()
    return torch.where(e > 0, 2.0 ** (e - 15) * (1 + m / 8), 2.0 ** -14 * m / 8)


def int4_encode(x):
    """float64 rows [.., d] -> (codes -7..7 [.., d], scale bytes [.., d/32])."""
    g = x.double().unflatten(-1, (-1, 32))
    want = g.abs().amax(-1) / 7
    table = scale_value(torch.arange(256))
    allowed = torch.nonzero((table >= 2.0 ** -12) & (table <= 960)).flatten()
    byte = allowed[torch.searchsorted(table[allowed], want).clamp_max(len(allowed) - 1)]      # the smallest that is >= want
    q = g / table[byte][..., None]
    code = (torch.floor(q.abs() + 0.5) * torch.sign(q)).clamp(-7, 7)
    return code.flatten(-2), byte


def int4_value(code, byte):
    return (code.double().unflatten(-1, (-1, 32)) * scale_value(byte)[..., None]).flatten(-2)


def int4_unpack(packed):
    p = packed.long()
    return torch.stack([p & 15, p >> 4], -1).flatten(-2) - 8


def int4_pack(code):
    c = code.long() + 8
    return (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)


# ---------------------------------------------------------------- FP8 pages
def fp8_page(x, valid):
    """One page [g, d] of float64 (rows from `valid` on: zeros) -> (codes as values, scale)."""
    x = x.clone()
    x[valid:] = 0
    m, e = torch.frexp(x.abs().max() / 448)
    e = int(e) - (1 if float(m) == 0.5 else 0)
    scale = 2.0 ** max(-6, min(7, e))
    return (x / scale).clamp(-448, 448).float().to(torch.float8_e4m3fn), scale


# ---------------------------------------------------------------- attention
def attention(q, k, v, scale):
    """Rows q [n, d] over k, v [t, d] in float64: output, log-sum-exp, and bounds of what they may be off by.

    Scores: keys and queries are exact operands; the fp32 accumulator of the tensor cores rounds (or cuts) each of the d / 16
    partial sums by at most 2^-22 of the largest term's size, which sum |q||k| bounds; the exponential is within 2^-22.
    Weights are rounded to 11 bits (2^-11), those below 2^-14 to within 2^-25 of one whose weight is at least one; sums are fp32,
    the output is rounded to bf16 by the caller's bound."""
    t = k.shape[0]
    if t == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -float("inf"), dtype=torch.float64), torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.float64)
    s = q @ k.T * scale
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[:, None])
    size = (q.abs() @ k.abs().T * scale).amax(-1)
    ds = q.shape[1] / 16 * 2.0 ** -22 * size + 2.0 ** -20
    around = p @ v.abs()
    do = around * (2 * ds[:, None] + 2.0 ** -11 + 2.0 ** -19) + t * 2.0 ** -25 * v.abs().amax(0)
    return p @ v, lse, do, 2 * ds + 2.0 ** -22 * lse.abs()
