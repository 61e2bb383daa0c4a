"""The ends of the operators' ranges as far as they can be seen without a GPU: what a code of an 8-bit pool
becomes on its way into a matrix product, in the library's own arithmetic on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T

CODES = [c for c in range(256) if c & 0x7F != 0x7F]
VALUES = torch.tensor(CODES, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def widened(scale, dtype, top=None, values=False):
    """All codes at a scale among a step's scales of which `top` is the largest, as float64 (fp16: in the step's unit), and
    the exponent of the unit."""
    f, unit = T.load().tutti_many_widen_, C.c_int32()
    f.restype, f.argtypes = C.c_uint32, [C.c_uint32, C.c_float, C.c_float, C.c_uint32, C.c_uint32, C.POINTER(C.c_int32)]
    words = np.array([f(c, scale, scale if top is None else top, T.DTYPE_BF16 if dtype == "bf16" else T.DTYPE_FP16, values, unit)
                      for c in CODES], dtype=np.uint32)
    assert (words >> 16 == words & 0xFFFF).all()
    low = words & 0xFFFF
    x = (low << 16).view(np.float32).astype(np.float64) if dtype == "bf16" else low.astype(np.uint16).view(np.float16).astype(np.float64)
    return x, unit.value


def once(x):
    return x.astype(np.float16).astype(np.float64)


@pytest.mark.parametrize("e", range(-100, 120))
def test_bf16_holds_every_code_at_every_scale_that_append_makes(e):
    got, unit = widened(2.0 ** e, "bf16")
    assert unit == 0 and (got == VALUES * 2.0 ** e).all()


@pytest.mark.parametrize("e", range(-100, 65))
def test_fp16_values_at_powers_of_two_are_rounded_once(e):
    """Their unit is 2, or what keeps the largest code finite; everything in the normal range is exact."""
    got, unit = widened(2.0 ** e, "fp16", values=True)
    assert unit == max(1, e - 7)
    assert (got == once(VALUES * 2.0 ** (e - unit))).all(), (VALUES[got != once(VALUES * 2.0 ** (e - unit))], got)


@pytest.mark.parametrize("e", range(-100, 120))
def test_fp16_keys_at_powers_of_two(e):
    """Exact unless another scale of the step is more than 2^22 times larger (the largest is brought to 2^7, codes are
    multiples of 2^-9, f16 of 2^-24), one rounding below."""
    for above in (0, 1, 5, 15, 22, 23, 31, 60):
        top = min(e + above, 120)
        got, unit = widened(2.0 ** e, "fp16", 2.0 ** top)
        assert unit == top - 7
        want = VALUES * 2.0 ** (e - unit)
        assert (got == once(want)).all(), (e, above)
        if top - e <= 22:
            assert (got == want).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("above", [1.0, 1.3, 2000.0, 3e5])
def test_codes_at_other_scales(dtype, above):
    """The factor, the product with it and the product with a second factor are rounded: half a step each, and in
    f16 half its smallest step for the last product (the factor's own smallest step is 2^14 times less there)."""
    half = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    rng = np.random.default_rng(3)
    for e in range(-40, 40):
        for m in (1.001, 1.25, 1.5, 1.9, 1.999, *(1 + rng.random(3))):
            s = float(np.float32(m * 2.0 ** e))
            for values in (False, True):
                got, unit = widened(s, dtype, s * above, values)
                want = VALUES * s * 2.0 ** -unit
                tol = ((1 + half) ** 3 - 1) * np.abs(want) + (2.0 ** -25 * (1 + 2.0 ** -4) if dtype == "fp16" else 0)
                assert (np.abs(got - want) <= tol).all(), (e, m, VALUES[~(np.abs(got - want) <= tol)][:4])
