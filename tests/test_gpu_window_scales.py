"""Attention under a window over an 8-bit pool whose scales are a caller's own: no powers of two, as append would leave them."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import check
from tests.pagecase import WindowCase
from tests.test_gpu_attend import fill_new
from tests.test_gpu_window import attend

pytestmark = pytest.mark.gpu

# What a key's or value's element code * scale is off by, relative to it.  More than 16 rows a KV head: the scale and the product are each
# rounded to the step's type (half a step: 2^-8, 2^-11), (1 + h)^2 - 1.  Up to 16 rows: scales are applied in 32 bits.
ROUNDED = {"bf16": 2.0 ** -7 + 2.0 ** -16, "fp16": 2.0 ** -10 + 2.0 ** -22}


def own_scales(c):
    for half in range(2):
        c.scale[half].copy_(torch.from_numpy(np.exp2(c.rng.uniform(-8, -5, tuple(c.scale[half].shape))).astype(np.float32)))
        c.scale_dev[half].copy_(c.scale[half])


def verify(c, out):
    """As the other tests' bounds, and `off` for each element that the products read."""
    g, sm = c.heads // c.hk, c.dim ** -0.5
    want, lse, tol, ltol = c.attend64(c.q, c.raw, c.scale, sm)
    off = ROUNDED[c.dtype] if c.max_new * g > 16 else 0.0
    q = c.q.float().double().cpu().numpy()
    for s, (p, n) in enumerate(c.lens):
        k, v = (np.abs(c.keys(c.raw, c.scale, h, s, p + n)) for h in range(2))
        signed = c.keys(c.raw, c.scale, 0, s, p + n)
        for i in range(n):
            at, row = c.seen(p + i), int(c.q_start[s]) + i
            for h in range(c.heads):
                x = signed[at, h // g] @ q[row, h] * sm
                w = np.exp(x - x.max())
                size = (w / w.sum()) @ v[at, h // g]
                d = off * (k[at, h // g] @ np.abs(q[row, h])).max() * sm
                tol[row, h] += (np.expm1(2 * d) + off * np.exp(2 * d)) * size
                ltol[row, h] += d
    n = int(c.q_start[-1])
    check(out.float().double().cpu().numpy()[:n], want, tol, "out")
    check(c.lse.double().cpu().numpy()[:n], lse, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens", [[(40, 1), (700, 1), (129, 1), (0, 1)], [(300, 4), (20, 2)], [(600, 40), (16, 130), (0, 70)]], ids=["decode", "few", "chunks"])
@pytest.mark.parametrize("dim,heads,kv_heads,block,hnd", [(128, 8, 2, 16, False), (64, 4, 2, 16, True), (128, 6, 2, 1, False), (64, 3, 3, 64, False)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (1 << 20, 0)])
def test_scales_that_are_no_powers_of_two(dtype, lens, dim, heads, kv_heads, block, hnd, window, sinks):
    c = WindowCase(lens, window, sinks, heads=heads, kv_heads=kv_heads, dim=dim, block=block, dtype=dtype, cache="8", hnd=hnd, seed=dim + block)
    try:
        own_scales(c)
        fill_new(c)
        c.clear()
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()
