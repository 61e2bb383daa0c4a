"""Causal attention over the paged pool (tutti_kv_attend_layer) against a plain statement in 64
bits.  Pool bytes that no sequence holds are NaN, so a key too many shows."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import DTYPES, OpCase, check

pytestmark = pytest.mark.gpu


def fill_new(c):
    """The step's own keys and values, written by the host as a 16-bit or 8-bit pool holds them."""
    raw = c.raw
    for s, (p, n) in enumerate(c.lens):
        for i in range(n):
            pos = int(c.ctx_len[s]) - n + i
            if pos < 0:
                continue
            b = int(c.block_ids[c.blk_start[s] + pos // c.bs])
            for half in range(2):
                x = torch.from_numpy(c.rng.standard_normal((c.hk, c.dim)))
                c.block(raw, half, b)[pos % c.bs] = (x * 60).clamp(-448, 448).to(torch.float8_e4m3fn) if c.size == 1 else x.to(DTYPES[c.dtype])
    c.pool.copy_(raw)


def attend(c, scale=None, stream=None, attn=None, lse=True):
    out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
    c.lse = torch.full((c.n_tok, c.heads), 7.5, dtype=torch.float32, device=c.dev) if lse else None
    (attn or c.attn).tutti_kv_attend_layer(1, c.step, T.make_attend(c.q, out, c.lse), c.dim ** -0.5 if scale is None else scale, stream)
    return out


def verify(c, out, scale=None, skip=()):
    want, lse, tol, ltol = c.attend64(c.q, c.raw, c.scale, c.dim ** -0.5 if scale is None else scale)
    n = int(c.q_start[-1])
    got, got_lse = out.float().double().cpu().numpy(), None if c.lse is None else c.lse.double().cpu().numpy()
    keep = np.ones(n, bool)
    for s in skip:
        keep[c.q_start[s]:c.q_start[s + 1]] = False
    check(got[:n][keep], want[keep], tol[keep], "out")
    assert (got[n:] == 7.5).all(), "rows behind the last sequence changed"
    if got_lse is not None:
        empty = np.isinf(lse) & keep[:, None]
        assert (got_lse[:n][empty] == -np.inf).all() and (got[:n][empty] == 0).all()
        full = ~np.isinf(lse) & keep[:, None]
        check(got_lse[:n][full], lse[full], ltol[full], "lse")
        assert (got_lse[n:] == 7.5).all()


RAGGED = [(0, 1), (40, 1), (129, 1), (0, 0), (511, 1), (15, 1), (16, 1), (63, 1), (64, 1), (5, 0)]
CHUNKS = [(0, 5), (37, 1), (16, 130), (300, 18), (3, 0), (0, 257), (127, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("lens", [RAGGED, CHUNKS], ids=["decode", "chunks"])
@pytest.mark.parametrize("dim,heads,kv_heads,block,hnd", [
    (128, 8, 2, 16, False), (64, 8, 2, 16, True), (128, 7, 1, 1, False), (64, 4, 4, 64, False), (128, 40, 2, 5, True)])
def test_attend_matches_the_statement(dtype, cache, lens, dim, heads, kv_heads, block, hnd):
    c = OpCase(lens, heads=heads, kv_heads=kv_heads, dim=dim, block=block, dtype=dtype, cache=cache, hnd=hnd, pad=16, seed=dim + block + heads)
    try:
        fill_new(c)
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("lens,kw", [
    ([(9000, 1)], dict(heads=8, kv_heads=1)), ([(4097, 1), (1, 1), (2047, 1)], dict(heads=32, kv_heads=8)),
    ([(3000, 3)], dict(heads=16, kv_heads=2)), ([(2500, 200)], dict(heads=4, kv_heads=2, interleaved=True)),
    ([(0, 700)], dict(heads=2, kv_heads=2)), ([(1500, 64), (0, 64), (900, 1)], dict(heads=6, kv_heads=3, packed=False)),
    ([(int(p), 1) for p in np.random.default_rng(1).integers(0, 300, 150)], dict(heads=4, kv_heads=2))])
def test_attend_long_and_many(cache, lens, kw):
    c = OpCase(lens, cache=cache, dim=128, seed=20, **kw)
    try:
        fill_new(c)
        verify(c, attend(c))
    finally:
        c.close()


@pytest.mark.parametrize("lens", [[(200, 1)], [(200, 90)]])
def test_attend_sharp_scores_and_other_scales(lens):
    """Scores of a few hundred: one key carries a row; and a negative and a zero scale."""
    c = OpCase(lens, heads=4, kv_heads=2, dim=64, dtype="fp16", seed=21, spread=1.0)
    try:
        fill_new(c)
        for scale in (3.0, -0.5, 0.0):
            verify(c, attend(c, scale), scale)
    finally:
        c.close()


@pytest.mark.parametrize("new", [4, 100])
def test_attend_rows_that_see_nothing(new):
    c = OpCase([(0, new), (0, 1), (50, 2)], heads=4, kv_heads=2, seed=22)
    try:
        c.ctx_len = np.array([2, 0, 52], dtype=np.int32)
        c.t_ctx.copy_(torch.from_numpy(c.ctx_len))
        c.lens = [(2 - new, new), (-1, 1), (50, 2)]
        fill_new(c)
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_attend_shared_prefix_blocks(cache):
    c = OpCase([(64, 1), (64, 1), (70, 20)], heads=8, kv_heads=2, cache=cache, seed=23, share=4)
    try:
        fill_new(c)
        verify(c, attend(c))
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 40])
def test_attend_bad_blocks_and_sequences(new):
    c = OpCase([(100, new), (40, new), (7, new)], heads=4, kv_heads=2, seed=24)
    try:
        fill_new(c)
        ids, ctx = c.block_ids.copy(), c.ctx_len.copy()
        ids[c.blk_start[0] + 2] = -5                      # keys 32..47 of sequence 0 are left out
        c.t_ids.copy_(torch.from_numpy(ids))
        out = attend(c)
        assert int(c.status) == T.EFAULT
        verify(c, out, skip=(0,))
        first = out[:new].clone()
        assert torch.isfinite(first.float()).all()
        c.status.zero_()
        c.t_ids.copy_(torch.from_numpy(c.block_ids))
        ctx[1] = 4000
        c.t_ctx.copy_(torch.from_numpy(ctx))
        out = attend(c)
        assert int(c.status) == T.EINVAL
        assert (out[new:2 * new] == 7.5).all() and (c.lse[new:2 * new] == 7.5).all()
        verify(c, out, skip=(1,))
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 33])
def test_attend_is_the_same_every_time_and_on_any_stream(new):
    c = OpCase([(3000, new), (17, new), (800, new)], heads=8, kv_heads=2, seed=25)
    try:
        fill_new(c)
        first = attend(c)
        side, other = torch.cuda.Stream(), T.Attn(c.ctx)
        torch.cuda.synchronize()
        for _ in range(5):
            a = attend(c)
            with torch.cuda.stream(side):
                b = attend(c, stream=side, attn=other)
            torch.cuda.synchronize()
            assert torch.equal(a, first) and torch.equal(b, first)
        other.close()
        c.lse = None
        assert torch.equal(attend(c, lse=False), first)
    finally:
        c.close()


@pytest.mark.parametrize("new", [1, 20])
def test_attend_captured_and_replayed_with_other_lengths(new):
    c = OpCase([(500, new), (40, new), (0, new)], heads=8, kv_heads=2, seed=26, spare_ids=40)
    try:
        fill_new(c)
        out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        c.lse = torch.full((c.n_tok, c.heads), 7.5, dtype=torch.float32, device=c.dev)
        io = T.make_attend(c.q, out, c.lse)
        side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            c.attn.tutti_kv_attend_layer(1, c.step, io, c.dim ** -0.5, side)
        for grown in (0, 100, -30):
            c.ctx_len = np.maximum(np.array([500, 40, 0]) + new + np.array([grown, 0, max(grown, 0)]), 0).astype(np.int32)
            c.lens = [(int(x) - new, new) for x in c.ctx_len]
            c.t_ctx.copy_(torch.from_numpy(c.ctx_len))
            for s in range(3):                              # whatever lies in front of the new rows
                for pos in range(max(0, int(c.ctx_len[s]))):
                    b = int(c.block_ids[c.blk_start[s] + pos // c.bs])
                    for half in range(2):
                        row = c.block(c.raw, half, b)[pos % c.bs]
                        if torch.isnan(row).any():
                            row.copy_(torch.from_numpy(c.rng.standard_normal((c.hk, c.dim))))
            c.pool.copy_(c.raw)
            out.fill_(7.5)
            c.lse.fill_(7.5)
            g.replay()
            torch.cuda.synchronize()
            verify(c, out)
    finally:
        c.close()


def test_attend_refusals_on_a_context():
    c = OpCase([(4, 2)], seed=27)
    try:
        out = torch.zeros((c.n_tok, c.heads, c.dim), dtype=DTYPES[c.dtype], device=c.dev)
        io = T.make_attend(c.q, out)
        call = lambda layer, i, sc=1.0: c.attn.tutti_kv_attend_layer(layer, c.step, i, sc, allow=(T.EINVAL,))  # noqa: E731
        assert call(0, io) == T.EINVAL and call(2, io) == T.EINVAL
        assert call(1, io, float("nan")) == T.EINVAL and call(1, io, float("inf")) == T.EINVAL
        io.q += 2
        assert call(1, io) == T.EINVAL
        with pytest.raises(T.TuttiError):
            T.make_attend(c.q, out.float())
        torch.cuda.synchronize()
        assert (out == 0).all()
    finally:
        c.close()
