"""The ends of the operators' ranges as far as they can be seen without a GPU: what a code of an 8-bit pool
becomes on its way into a matrix product, in the library's own arithmetic on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T

CODES = [c for c in range(256) if c & 0x7F != 0x7F]
VALUES = torch.tensor(CODES, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()


def widened(scale, dtype):
    """All codes at a scale (fp16: at half of it) as float64."""
    f = T.load().tutti_many_widen_
    f.restype, f.argtypes = C.c_uint32, [C.c_uint32, C.c_float, C.c_uint32]
    words = np.array([f(c, scale, T.DTYPE_BF16 if dtype == "bf16" else T.DTYPE_FP16) for c in CODES], dtype=np.uint32)
    assert (words >> 16 == words & 0xFFFF).all()
    low = words & 0xFFFF
    return (low << 16).view(np.float32).astype(np.float64) if dtype == "bf16" else low.astype(np.uint16).view(np.float16).astype(np.float64)


@pytest.mark.parametrize("dtype,lo,hi", [("fp16", -100, 8), ("bf16", -100, 119)])
def test_codes_at_scales_that_are_powers_of_two_are_rounded_once(dtype, lo, hi):
    """bf16 holds every code at every scale that append makes, fp16 every one that is in its normal range."""
    for e in range(lo, hi + 1):
        want = VALUES * 2.0 ** e / (2 if dtype == "fp16" else 1)
        if dtype == "fp16":
            want = want.astype(np.float16).astype(np.float64)
        got = widened(2.0 ** e, dtype)
        assert (got == want).all(), (e, VALUES[got != want][:4], got[got != want][:4])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_codes_at_other_scales(dtype):
    """The factor, the product with it and the product with a second factor are rounded: half a step each, and in
    f16 half its smallest step for the last product (the factor's own smallest step is 2^14 times less there)."""
    half = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    rng = np.random.default_rng(3)
    for e in range(-40, 8):
        for m in (1.001, 1.25, 1.5, 1.9, 1.999, *(1 + rng.random(5))):
            s = float(np.float32(m * 2.0 ** e))
            want = VALUES * s / (2 if dtype == "fp16" else 1)
            tol = ((1 + half) ** 3 - 1) * np.abs(want) + (2.0 ** -25 * (1 + 2.0 ** -4) if dtype == "fp16" else 0)
            got = widened(s, dtype)
            assert (np.abs(got - want) <= tol).all(), (e, m, VALUES[~(np.abs(got - want) <= tol)][:4])
