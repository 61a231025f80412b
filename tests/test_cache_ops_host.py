"""What of the cache operators needs no GPU: refusals before a device is touched, and the 4-bit format's rules on the plain form."""
import ctypes as C

import torch

import cache_ops_ref as ref
from paper_2604_12056_b200 import binding as B


def test_calls_without_a_context_are_refused():
    from paper_2604_12056_b200 import build
    build.build()
    lib = B.lib()
    t = B.NewTokensT()
    assert lib.losa_rope_append(None, None, None, C.byref(t), None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_rope_append(None, None, None, None, None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_int4_attn(None, None, None, None, None, None) == B.LOSA_ERR_INVALID_ARG


def test_scale_bytes_are_the_upper_bits_of_fp16_numbers():
    b = torch.arange(248)
    assert (ref.scale_value(b) == (b.to(torch.int16) << 7).view(torch.float16).double()).all()


def test_codes_pack_and_unpack():
    c = torch.randint(-7, 8, (5, 64))
    assert (ref.int4_unpack(ref.int4_pack(c)) == c).all()
    assert int(ref.int4_pack(torch.tensor([3, -2]))[0]) == (3 + 8) | ((-2 + 8) << 4)


def test_values_are_exact_in_16_bits_and_near_the_input():
    x = torch.randn(200, 128, generator=torch.Generator().manual_seed(1)).bfloat16().double()
    code, byte = ref.int4_encode(x)
    y, s = ref.int4_value(code, byte), ref.scale_value(byte).repeat_interleave(32, -1)
    assert (y.bfloat16().double() == y).all() and (y.half().double() == y).all()
    assert ((x - y).abs() <= s / 2).all() and code.abs().max() <= 7
    assert (s * 7 >= x.abs()).all() and (s * 7 < 8 / 7.0 * 8 / 7 * 7 * x.unflatten(-1, (-1, 32)).abs().amax(-1).repeat_interleave(32, -1)).all()


def test_every_bf16_value_rounds_by_the_multiplier_as_by_the_quotient():
    """The kernel multiplies by (1 + 2^-16) / s and rounds to nearest; the definition divides and takes halves away from zero.
    All bf16 values in (-8 s, 8 s) of three binades, all eight mantissas of s."""
    import numpy as np
    bits = np.arange(0x3000, 0x4200, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    for m in range(8):
        s = np.float32(0.25 * (1 + m / 8))
        v = x[x <= 7 * s]
        mul = np.float32(np.float32(1.0000152587890625) / s)
        # one rounding of x * mul + 12582920, as a fused multiply-add makes it: the double sum is exact to far below half a unit
        got = np.rint(v.astype(np.float64) * np.float64(mul))
        want = np.floor(v.astype(np.float64) / np.float64(s) + 0.5)
        assert (got == want).all()
