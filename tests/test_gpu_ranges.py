"""The operators on the pool at the ends of their ranges: scales of every power of two, against the statement in
64 bits."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import OpCase, check
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


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,dim", [("fp16", 64), ("fp16", 128), ("bf16", 128)])
def test_attend8_keys_at_scales_beyond_those_of_fp16_rows(dtype, dim, new):
    """A pool that bf16 steps have filled: keys far beyond 65504, scores as small as any."""
    c = OpCase([(60, new), (3, new), (700, new)], heads=4, kv_heads=2, dim=dim, cache="8", dtype=dtype, seed=84)
    try:
        fill_new(c)
        for e in (9, 12, 17, 25, 40, 60):
            set_scales(c, lambda s, b: e - b % 3)
            c.scale[1].fill_(2.0 ** -7)
            c.scale_dev[1].copy_(c.scale[1])
            sm = 2.0 ** -e * 0.01
            verify(c, attend(c, sm), sm)
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,dim", [("fp16", 64), ("fp16", 128), ("bf16", 128)])
@pytest.mark.parametrize("order", [0, 1, 2])
def test_attend8_values_at_scales_beyond_those_of_fp16_rows(dtype, dim, new, order):
    """Values of up to 2^20 among small ones, in every order; outputs stay finite.  One sequence is shared by many workers."""
    c = OpCase([(60, new), (330, new), (3000, new)], heads=4, kv_heads=2, dim=dim, cache="8", dtype=dtype, seed=85)
    try:
        fill_new(c)
        exps = [-7, 9, 20, -7, 12, 17, 10, -12]                  # of the values' scales, by block
        least = {12: 8, 17: 8, 20: 2}                            # codes 0..7 are subnormal, 0 and 1 the two smallest
        at = lambda s, b: 0 if order == 1 and s == 2 and b < 150 else (b * (1, 3, 5)[order] + s) % 8  # noqa: E731
        set_scales(c, lambda s, b: exps[at(s, b)])
        c.scale[0].fill_(2.0 ** -7)
        c.scale_dev[0].copy_(c.scale[0])
        for s in range(3):
            for b in range(-(-int(c.ctx_len[s]) // c.bs)):
                x = c.block(c.raw, 1, int(c.block_ids[c.blk_start[s] + b]))
                n = min(c.bs, int(c.ctx_len[s]) - b * c.bs)
                if exps[at(s, b)] in least:
                    g = torch.Generator().manual_seed(b)
                    codes = torch.randint(0, least[exps[at(s, b)]], x.shape, generator=g, dtype=torch.uint8) + 128 * torch.randint(0, 2, x.shape, generator=g, dtype=torch.uint8)
                    x[:n] = codes.view(torch.float8_e4m3fn)[:n]
        c.pool.copy_(c.raw)
        out = attend(c)
        want, lse, tol, ltol = c.attend64(c.q, c.raw, c.scale, c.dim ** -0.5)
        if dtype == "fp16":
            # Probabilities are kept in the unit of the largest value scale, 2^13 here (2^20 is 2^7 of it), 2^12 of the
            # usual one: half f16's smallest step, 2^-25, against a largest probability of 2^6; and values as
            # much below that unit are off by 2^-25 of it.
            for s in range(3):
                v = np.abs(c.keys(c.raw, c.scale, 1, s, int(c.ctx_len[s]))).sum(0)
                tol[c.q_start[s]:c.q_start[s + 1]] += np.repeat(2.0 ** (-31 + 12) * v, 2, 0) + 2.0 ** (13 - 25)
        n = int(c.q_start[-1])
        assert np.abs(want).max() < 65504
        check(out[:n].float().double().cpu().numpy(), want, tol, "out")
        check(c.lse[:n].double().cpu().numpy(), lse, ltol, "lse")
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache,dtype", [("16", "bf16"), ("16", "fp16"), ("8", "bf16"), ("8", "fp16")])
@pytest.mark.parametrize("new", [1, 40])
def test_nan_scores_make_out_and_lse_nan(cache, dtype, new):
    """A query of NaN; keys of NaN in every block but the last, so that whole parts of a shared row have no other score."""
    c = OpCase([(3000, new), (60, new), (0, new)], heads=4, kv_heads=2, dim=128, cache=cache, dtype=dtype, seed=86)
    try:
        fill_new(c)
        row = int(c.q_start[1])
        c.q[row, 2, 5] = float("nan")
        out = attend(c)
        got, lse = torch.isnan(out.float()), torch.isnan(c.lse)
        assert got[row, 2].all() and lse[row, 2]
        got[row, 2], lse[row, 2] = False, False
        assert not got.any() and not lse.any() and torch.isfinite(c.lse[:int(c.q_start[-1])][~lse[:int(c.q_start[-1])]]).sum() == lse[:int(c.q_start[-1])].numel() - 1
        c.q[row, 2, 5] = 1
        for b in range(-(-3000 // c.bs) - 1):
            x = c.block(c.raw, 0, int(c.block_ids[b]))[:, 1, 77]
            x.copy_(torch.full(x.shape, float("nan")))
        c.pool.copy_(c.raw)
        out = attend(c)
        verify(c, out, skip=(0,))
        got, lse = torch.isnan(out[:new].float()), torch.isnan(c.lse[:new])
        assert got[:, 2:].all() and lse[:, 2:].all() and not got[:, :2].any() and torch.isfinite(c.lse[:new, :2]).all()
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 40])
def test_scores_that_are_all_minus_infinity(new):
    c = OpCase([(60, new), (5, new)], heads=4, kv_heads=2, dim=64, packed=False, seed=87)
    try:
        fill_new(c)
        q = c.q.clone()
        c.q.zero_()
        c.q[:, :, 0] = 1
        for b in range(-(-int(c.ctx_len[0]) // c.bs)):
            c.block(c.raw, 0, int(c.block_ids[b]))[:, 0, 0] = float("-inf")
        c.pool.copy_(c.raw)
        out = attend(c)
        assert (out[:new, :2] == 0).all() and (c.lse[:new, :2] == -float("inf")).all()
        assert torch.isfinite(c.lse[:new, 2:]).all() and torch.isfinite(c.lse[new:2 * new]).all() and torch.isfinite(out[:2 * new].float()).all()
        c.q.copy_(q)
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,cache", [("bf16", "16"), ("bf16", "8"), ("fp16", "8")])
def test_scales_of_zero_and_next_to_it(new, dtype, cache):
    """Products of queries and keys of 2^60 and more, which a scale makes ordinary scores again, or nothing."""
    c = OpCase([(60, new), (500, new)], heads=4, kv_heads=2, dim=64, dtype=dtype, cache=cache, packed=False, seed=88)
    try:
        fill_new(c)
        q_up, k_up = (60, 55) if dtype == "bf16" else (0, 110)
        c.q *= 2.0 ** q_up
        if cache == "8":
            set_scales(c, lambda s, b: k_up)
            c.scale[1].fill_(2.0 ** -7)
            c.scale_dev[1].copy_(c.scale[1])
        else:
            for s in range(2):
                for b in range(-(-int(c.ctx_len[s]) // c.bs)):
                    c.block(c.raw, 0, int(c.block_ids[c.blk_start[s] + b])).mul_(2.0 ** k_up)
            c.pool.copy_(c.raw)
        small = 2.0 ** -(q_up + k_up) / (100 if cache == "8" else 1)
        for scale in (small, -small, 0.0, -0.0, 2.0 ** -149):
            verify(c, attend(c, scale), scale)
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache,dtype", [("16", "bf16"), ("8", "fp16")])
@pytest.mark.parametrize("most", [1, 3, 17, 5000])
def test_a_generous_bound_on_new_rows(cache, dtype, most):
    """max_new may be larger than any sequence's rows: single tokens then go through whichever kernel it selects."""
    c = OpCase([(300, 1), (0, 1), (1000, 1), (5, 0), (63, 1)], heads=16, kv_heads=2, dim=128, cache=cache, dtype=dtype, seed=97)
    try:
        fill_new(c)
        c.step = T.make_step(c.t_q_start, c.t_ctx, c.t_blk_start, c.t_ids, c.n_tok, most, c.status)
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()
