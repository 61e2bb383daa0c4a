"""The operators on the pool at the ends of their ranges: scales of every power of two, against the statement in
64 bits."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import OpCase
from tests.test_gpu_attend import attend, fill_new, verify

pytestmark = pytest.mark.gpu


def set_scales(c, exponent):
    """Scale 2^exponent(sequence, block) on the blocks that sequences hold, keys and values alike."""
    for s in range(len(c.lens)):
        for b in range(-(-int(c.ctx_len[s]) // c.bs)):
            for half in range(2):
                c.scale[half][int(c.block_ids[c.blk_start[s] + b])] = 2.0 ** exponent(s, b)
    for a, b in zip(c.scale, c.scale_dev):
        b.copy_(a)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend8_at_every_power_of_two(dtype, new, dim):
    """A sequence for every scale from 2^-30 to 2^8, then one whose blocks have them all."""
    lens = [(60, new)] * 39 + [(39 * 16 - new, new)]
    c = OpCase(lens, heads=4, kv_heads=2, dim=dim, cache="8", dtype=dtype, seed=80 + dim)
    try:
        fill_new(c)
        set_scales(c, lambda s, b: (s if s < 39 else b) - 30)
        for scale in (1e-5, dim ** -0.5):
            verify(c, attend(c, scale), scale)
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_small_values_are_appended_and_attended(dtype):
    """A prompt chunk whose keys and values have peaks around 2^-6: append gives them the scales 2^-16 to 2^-13."""
    from tests.test_gpu_append import append, verify as append_verify
    c = OpCase([(33, 60), (0, 100)], heads=4, kv_heads=2, dim=128, cache="8", dtype=dtype, packed=False, seed=83)
    try:
        for half in range(2):
            c.scale[half].fill_(2.0 ** -17)
            c.scale_dev[half].copy_(c.scale[half])
        for dev, host in ((c.k, c.host_k), (c.v, c.host_v)):
            host *= 2.0 ** -9
            dev.copy_(host)
        append_verify(c, append(c))
        c.raw = c.pool.cpu().clone()
        used = torch.cat([s.log2().unique() for s in c.scale])
        assert {-15.0, -14.0} <= set(used.tolist())
        verify(c, attend(c))
    finally:
        c.close()
