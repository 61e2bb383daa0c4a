"""Attention with a window and first tokens (tutti_kv_attend_window_layer) against a plain statement in 64 bits.  Blocks behind
the window have no id, and their bytes are NaN."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import DTYPES
from tests.pagecase import WindowCase
from tests.test_gpu_attend import attend as attend_all, fill_new, verify

pytestmark = pytest.mark.gpu


def attend(c, scale=None, stream=None, attn=None, lse=True):
    out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
    c.lse = torch.full((c.n_tok, c.heads), 7.5, dtype=torch.float32, device=c.dev) if lse else None
    (attn or c.attn).tutti_kv_attend_window_layer(1, c.step, T.make_attend(c.q, out, c.lse), c.dim ** -0.5 if scale is None else scale,
                                                  T.make_window(c.window, c.sinks), stream)
    return out


def run(lens, window, sinks, scale=None, **kw):
    c = WindowCase(lens, window, sinks, **kw)
    try:
        fill_new(c)
        c.clear()
        verify(c, attend(c, scale), scale)
        assert int(c.status) == T.OK
    finally:
        c.close()


RAGGED = [(0, 1), (40, 1), (129, 1), (0, 0), (511, 1), (15, 1), (1000, 1), (63, 1), (300, 1), (5, 0)]
CHUNKS = [(0, 5), (37, 1), (16, 130), (600, 18), (3, 0), (0, 257), (527, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("lens", [RAGGED, CHUNKS], ids=["decode", "chunks"])
@pytest.mark.parametrize("window,sinks", [(100, 4), (1, 0), (33, 130)])
@pytest.mark.parametrize("dim,heads,kv_heads,block,hnd", [(128, 8, 2, 16, False), (64, 8, 2, 16, True), (128, 7, 1, 1, False), (64, 4, 4, 64, False)])
def test_window_matches_the_statement(dtype, cache, lens, window, sinks, dim, heads, kv_heads, block, hnd):
    run(lens, window, sinks, heads=heads, kv_heads=kv_heads, dim=dim, block=block, dtype=dtype, cache=cache, hnd=hnd, pad=16, seed=dim + block + heads)


@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("lens,window,sinks,kw", [
    ([(9000, 1)], 1000, 4, dict(heads=8, kv_heads=1)), ([(4097, 1), (1, 1), (2047, 1)], 2000, 1, dict(heads=32, kv_heads=8)),
    ([(2500, 3)], 700, 200, dict(heads=16, kv_heads=2)), ([(2500, 200)], 128, 128, dict(heads=4, kv_heads=2, interleaved=True)),
    ([(0, 700)], 64, 0, dict(heads=2, kv_heads=2)), ([(1500, 64), (0, 64), (900, 1)], 257, 5, dict(heads=6, kv_heads=3, packed=False)),
    ([(int(p), 1) for p in np.random.default_rng(1).integers(0, 300, 150)], 50, 3, dict(heads=4, kv_heads=2)),
    ([(3000, 1), (3001, 1)], (1 << 31) - 1, 0, dict(heads=4, kv_heads=2)), ([(700, 40)], 1, (1 << 31) - 1, dict(heads=4, kv_heads=2)),
    ([(1100, 2), (500, 2)], 3, 0, dict(heads=8, kv_heads=2)), ([(1100, 4), (500, 1)], 2, 2, dict(heads=8, kv_heads=2)),
    ([(260, 600)], 130, 4, dict(heads=16, kv_heads=2))])
def test_window_long_and_many(cache, lens, window, sinks, kw):
    run(lens, window, sinks, cache=cache, dim=128, seed=20, **kw)


@pytest.mark.parametrize("seed", range(12))
def test_window_random(seed):
    rng = np.random.default_rng(100 + seed)
    n = int(rng.integers(1, 6))
    chunk = rng.random() < 0.6
    lens = [(int(rng.integers(0, 1500)), int(rng.integers(1, 200 if chunk else 3))) for _ in range(n)]
    heads, kv_heads = [(8, 2), (4, 4), (6, 2), (5, 1), (16, 8)][rng.integers(0, 5)]
    cache = str(rng.choice(["16", "8"]))
    run(lens, int(np.exp(rng.uniform(0, 7))), int(rng.choice([0, 1, 4, 60, 129, 300])), heads=heads, kv_heads=kv_heads, dim=int(rng.choice([64, 128])),
        block=int(rng.choice([1, 3, 8, 16, 32, 128])), cache=cache, dtype=str(rng.choice(["bf16", "fp16"])), hnd=bool(rng.random() < 0.4), seed=seed)


@pytest.mark.parametrize("lens", [[(200, 1), (90, 1)], [(200, 90), (30, 4)]])
def test_window_sharp_scores_and_other_scales(lens):
    c = WindowCase(lens, 70, 3, heads=4, kv_heads=2, dim=64, dtype="fp16", seed=21, spread=1.0)
    try:
        fill_new(c)
        c.clear()
        for scale in (3.0, -0.5, 0.0):
            verify(c, attend(c, scale), scale)
    finally:
        c.close()


@pytest.mark.parametrize("new", [4, 100])
@pytest.mark.parametrize("window,sinks", [(1, 0), (30, 2)])
def test_window_rows_that_see_nothing(new, window, sinks):
    c = WindowCase([(0, new), (0, 1), (50, 2)], window, sinks, heads=4, kv_heads=2, seed=22, gone=None)
    try:
        c.ctx_len = np.array([2, 0, 52], dtype=np.int32)
        c.t_ctx.copy_(torch.from_numpy(c.ctx_len))
        c.lens = [(2 - new, new), (-1, 1), (50, 2)]
        fill_new(c)
        c.clear()
        verify(c, attend(c))
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache,dtype", [("16", "bf16"), ("8", "bf16"), ("8", "fp16"), ("16", "fp16")])
@pytest.mark.parametrize("lens", [[(900, 1), (100, 1), (1999, 1)], [(900, 100), (100, 30), (1024, 128)]])
def test_a_window_that_holds_all_is_plain_attention(cache, dtype, lens):
    """The same bits as tutti_kv_attend_layer: the keys' units and the order of sums are the same."""
    c = WindowCase(lens, (1 << 31) - 1, 7, heads=8, kv_heads=2, cache=cache, dtype=dtype, seed=30, gone=None)
    try:
        fill_new(c)
        a, la = attend(c), c.lse.clone()
        b, lb = attend_all(c), c.lse
        assert torch.equal(a, b) and torch.equal(la, lb)
    finally:
        c.close()


@pytest.mark.parametrize("lens", [[(900, 1), (333, 1)], [(900, 40), (333, 200)]])
@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("gone", [-1, 1 << 30, -(1 << 31)])
def test_blocks_behind_the_window_are_not_looked_at(lens, cache, gone):
    """The same bits whether they are there or not, and nothing is reported."""
    got = []
    for g in (None, gone):
        c = WindowCase(lens, 150, 20, heads=8, kv_heads=2, cache=cache, seed=31, gone=g)
        try:
            fill_new(c)
            c.clear()
            got.append(attend(c))
            assert int(c.status) == T.OK
        finally:
            c.close()
    assert torch.equal(*got)


@pytest.mark.parametrize("new", [1, 60])
def test_missing_blocks_inside_the_window(new):
    """A block outside the pool that a row would see is left out and reported, the first tokens' block too."""
    for block in (0, 35):
        c = WindowCase([(600, new)], 80, 5, heads=4, kv_heads=2, block=16, seed=32)
        try:
            fill_new(c)
            c.clear()
            c.block_ids[c.blk_start[0] + block] = -1
            c.t_ids.copy_(torch.from_numpy(c.block_ids))
            seen = WindowCase.seen
            c.seen = lambda pos: np.array([j for j in seen(c, pos) if j // 16 != block])
            verify(c, attend(c))
            assert int(c.status) == T.EFAULT
        finally:
            c.close()


def test_refusals():
    c = WindowCase([(30, 1)], 8, 2, heads=4, kv_heads=2, seed=33)
    try:
        out = torch.empty(c.n_tok, c.heads, c.dim, dtype=DTYPES[c.dtype], device=c.dev)
        io = T.make_attend(c.q, out)
        for w in (T.Window(0, 4), T.Window(1 << 31, 0), T.Window(4, 1 << 31)):
            assert c.attn.tutti_kv_attend_window_layer(1, c.step, io, 0.1, w, allow=(T.EINVAL,)) == T.EINVAL
        assert c.attn.tutti_kv_attend_window_layer(0, c.step, io, 0.1, T.make_window(4), allow=(T.EINVAL,)) == T.EINVAL
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("most", [12, 40])
def test_many_short_chunks(cache, most):
    """Tiles of a few rows, of one half and of two, hundreds of them, most of one or two units."""
    rng = np.random.default_rng(most)
    lens = [(int(rng.integers(0, 300)), int(rng.integers(5, most))) for _ in range(90)]
    run(lens, 60, 3, heads=8, kv_heads=2, dim=64, cache=cache, dtype="fp16", seed=most)
    run(lens, 1 << 20, 0, heads=8, kv_heads=2, dim=64, cache=cache, dtype="fp16", seed=most, gone=None)
