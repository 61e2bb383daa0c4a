"""Appending keys and values to the paged pool (tutti_kv_append_layer) against a plain statement in
64 bits.  The pool starts as NaN bytes wherever no sequence holds a token, and every byte that a
step has no business with must stay what it was."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.opcase import DTYPES, F32, HALF, OpCase, check, pow2_scale, rotate64

pytestmark = pytest.mark.gpu

RAGGED = [(0, 5), (37, 1), (16, 16), (15, 18), (3, 0), (0, 0), (31, 33)]


def table_of(n_pos, rot, seed=0):
    a = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


def append(c, style="half", rot=None, rope=True, with_q=True, stream=None):
    """(q_out before, q_out after) of one call on the case."""
    q_out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
    c.table = table_of(int(c.ctx_len.max()) + 1, rot or c.dim)
    r = T.make_rope(c.table, T.ROPE_HALF if style == "half" else T.ROPE_PAIRS) if rope else None
    tok = T.make_tokens(c.k, c.v, c.q, q_out) if with_q else T.make_tokens(c.k, c.v)
    c.ctx.tutti_kv_append_layer(1, c.step, tok, r, stream)
    return q_out


def expected_rows(c, style, rope):
    """Per sequence: position of every row, rotated keys, values, their magnitudes."""
    for s, (_, n) in enumerate(c.lens):
        rows = slice(int(c.q_start[s]), int(c.q_start[s]) + n)
        pos = int(c.ctx_len[s]) - n + np.arange(n)
        keep = pos >= 0
        rows = np.arange(rows.start, rows.stop)[keep]
        pos = pos[keep]
        k, v, q = (t[torch.from_numpy(rows)].float().double().numpy() for t in (c.host_k, c.host_v, c.host_q))
        km, qm = np.abs(k), np.abs(q)
        if rope:
            tab = c.table.cpu().numpy()
            k, km = rotate64(k, pos, tab, style)
            q, qm = rotate64(q, pos, tab, style)
        yield s, rows, pos, (k, km), (v, np.abs(v)), (q, qm)


def verify(c, q_out, style="half", rope=True, with_q=True, skip_blocks=()):
    half, tiny = HALF[c.dtype]
    want_raw = c.raw.clone()
    got_raw = c.pool.cpu()
    got_q = q_out.float().double().cpu().numpy()
    seen_q = np.zeros(c.n_tok, bool)
    for s, rows, pos, k, v, q in expected_rows(c, style, rope):
        if with_q:
            # three 32-bit roundings of products and sum, then the type's
            check(got_q[rows], q[0], half * np.abs(q[0]) + tiny + 4 * F32 * q[1], f"q of sequence {s}")
            seen_q[rows] = True
        for half_i, (x, mag) in enumerate((k, v)):
            for b in sorted(set(pos // c.bs)):
                i = int(c.block_ids[c.blk_start[s] + b])
                at = pos // c.bs == b
                got, want = c.block(got_raw, half_i, i), c.block(want_raw, half_i, i)
                r = pos[at] % c.bs
                if c.cache == "16":
                    check(got[r].float().double().numpy(), x[at], half * np.abs(x[at]) + tiny + 4 * F32 * mag[at], f"plane {half_i} block {i}")
                else:
                    for h in range(c.hk):
                        new = pow2_scale(np.abs(x[at][:, h]).max())
                        held = int(r[0])
                        old = float(c.scale[half_i][i, h])
                        if held:
                            new = max(new, old)
                        sc = float(c.scale_dev[half_i][i, h])
                        assert sc == new, (s, half_i, i, h, sc, new)
                        y = got[r, h].float().double().numpy() * sc
                        hs, ht = HALF["e4m3"]
                        check(y, x[at][:, h], hs * np.abs(x[at][:, h]) + ht * sc + 4 * F32 * mag[at][:, h], f"plane {half_i} block {i}")
                        if held:
                            was = want[:held, h].float().double().numpy() * old
                            check(got[:held, h].float().double().numpy() * sc, was, (sc != old) * (hs * np.abs(was) + ht * sc), f"held rows of block {i}")
                            want[:held, h] = got[:held, h]
                        c.scale[half_i][i, h] = sc
                want[r] = got[r]
    assert torch.equal(got_raw, want_raw), "bytes that belong to nobody's new tokens changed"
    assert (got_q[~seen_q] == 7.5).all(), "rows behind the last sequence (or padding) changed"
    if c.scale:
        for a, b in zip(c.scale, c.scale_dev):
            assert torch.equal(a, b.cpu()), "scales of untouched blocks changed"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["16", "8"])
@pytest.mark.parametrize("dim,rot,style,block,hnd", [
    (128, 128, "half", 16, False), (128, 64, "pairs", 16, True), (64, 64, "half", 1, False), (64, 32, "half", 8, True),
    (80, 80, "half", 16, False), (96, 48, "pairs", 5, False), (256, 256, "half", 64, True), (16, 16, "pairs", 32, False)])
def test_append_matches_the_statement(dtype, cache, dim, rot, style, block, hnd):
    c = OpCase(RAGGED, heads=6, kv_heads=2, dim=dim, block=block, dtype=dtype, cache=cache, hnd=hnd, pad=48, seed=dim + block)
    try:
        verify(c, append(c, style, rot), style)
        assert int(c.status) == T.OK
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_append_without_rotation_and_without_queries(cache):
    c = OpCase(RAGGED, heads=4, kv_heads=4, dim=64, cache=cache, interleaved=True, packed=False, seed=3)
    try:
        q_out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k, c.v))
        verify(c, q_out, rope=False, with_q=False)
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_append_one_token_each_for_many_sequences(cache):
    rng = np.random.default_rng(9)
    c = OpCase([(int(p), 1) for p in rng.integers(0, 200, 77)], heads=32, kv_heads=8, dim=128, cache=cache, seed=4)
    try:
        verify(c, append(c))
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_append_in_place_queries_and_many_tokens(cache):
    c = OpCase([(100, 700), (0, 333)], heads=8, kv_heads=1, dim=128, cache=cache, dtype="fp16", seed=5)
    try:
        c.table = table_of(900, 128)
        q = c.q.clone()
        c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k, c.v, q, q), T.make_rope(c.table))
        n = int(c.q_start[-1])
        assert torch.equal(q[n:], c.q[n:])
        q[n:] = 7.5
        verify(c, q)
    finally:
        c.close()


def test_append_twice_is_append_once():
    c = OpCase(RAGGED, cache="8", seed=6)
    try:
        append(c)
        torch.cuda.synchronize()
        pool, sc = c.pool.clone(), [s.clone() for s in c.scale_dev]
        append(c)
        assert torch.equal(pool, c.pool) and all(torch.equal(a, b) for a, b in zip(sc, c.scale_dev))
    finally:
        c.close()


def test_append_rows_at_negative_positions_are_padding():
    c = OpCase([(0, 4), (0, 1), (20, 2)], seed=7)
    try:
        c.ctx_len = np.array([2, 0, 22], dtype=np.int32)     # two rows of the first, the only one of the second
        c.t_ctx.copy_(torch.from_numpy(c.ctx_len))
        c.lens = [(-2, 4), (-1, 1), (20, 2)]
        verify(c, append(c))
        assert int(c.status) == T.OK
    finally:
        c.close()


def test_append8_infinities_and_nan():
    c = OpCase([(3, 4)], heads=2, kv_heads=2, dim=64, cache="8", seed=8)
    try:
        c.v[0, 0, 3], c.v[1, 0, 5], c.v[2, 1, 7] = float("inf"), float("nan"), float("-inf")
        append(c, rope=False)
        i = int(c.block_ids[0])
        got = c.block(c.pool.cpu(), 1, i).float()
        assert got[3, 0, 3] == 448 and torch.isnan(got[4, 0, 5]) and got[5, 1, 7] == -448
        x = c.host_v[:4].float().double()
        x[0, 0, 3] = x[1, 0, 5] = x[2, 1, 7] = 0
        for h in range(2):
            assert float(c.scale_dev[1][i, h]) == max(pow2_scale(float(x[:, h].abs().max())), float(c.scale[1][i, h]))
    finally:
        c.close()


def test_append8_scale_grows_and_zero_rows():
    """Zero keys in a fresh block take the floor; a large value behind small ones rounds them again."""
    c = OpCase([(16, 1), (5, 1)], heads=2, kv_heads=2, dim=64, cache="8", packed=False, seed=10)
    try:
        c.k.zero_()
        c.host_k.zero_()
        c.v[1] *= 1000
        c.host_v[1] *= 1000
        verify(c, append(c))
        i = int(c.block_ids[c.blk_start[0] + 1])
        assert (c.scale_dev[0][i].cpu() == 2.0 ** -100).all()
    finally:
        c.close()


def test_append_reports_and_skips_bad_sequences():
    c = OpCase([(16, 3), (40, 2), (7, 2), (30, 4)], seed=11)
    try:
        ids, ctx = c.block_ids.copy(), c.ctx_len.copy()
        ids[c.blk_start[0] + 1] = c.n_blocks                       # the block that sequence 0 writes
        ctx[1] = 1000                                              # more tokens than blocks
        c.t_ids.copy_(torch.from_numpy(ids))
        c.t_ctx.copy_(torch.from_numpy(ctx))
        before = c.pool.clone()
        append(c)
        assert int(c.status) in (T.EFAULT, T.EINVAL)
        after, want = c.pool.cpu(), before.cpu()
        for s in (2, 3):                                           # the good ones are written
            for half in range(2):
                for b in range(c.lens[s][0] // c.bs, -(-int(c.ctx_len[s]) // c.bs)):
                    i = int(c.block_ids[c.blk_start[s] + b])
                    assert not torch.equal(c.block(after, half, i), c.block(want, half, i))
                    c.block(want, half, i).copy_(c.block(after, half, i))
        assert torch.equal(after, want)
        c.t_ids.copy_(torch.from_numpy(c.block_ids))
        c.status.zero_()
        append(c)
        assert int(c.status) == T.EINVAL
    finally:
        c.close()


def test_append_rotation_table_too_short():
    c = OpCase([(30, 2), (3, 2)], seed=12)
    try:
        q_out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        c.ctx.tutti_kv_append_layer(1, c.step, T.make_tokens(c.k, c.v, c.q, q_out), T.make_rope(table_of(10, 128)))
        assert int(c.status) == T.EINVAL
        assert (q_out[:2] == 7.5).all() and (q_out[4:] == 7.5).all() and not (q_out[2:4] == 7.5).all()
    finally:
        c.close()


@pytest.mark.parametrize("cache", ["16", "8"])
def test_append_captured_and_replayed_with_other_lengths(cache):
    c = OpCase([(20, 1), (40, 1), (0, 1)], cache=cache, seed=13)
    try:
        tab = table_of(64, 128)
        q_out = torch.full((c.n_tok, c.heads, c.dim), 7.5, dtype=DTYPES[c.dtype], device=c.dev)
        tok, rope = T.make_tokens(c.k, c.v, c.q, q_out), T.make_rope(tab)
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            c.ctx.tutti_kv_append_layer(1, c.step, tok, rope, side)
        assert torch.equal(c.pool.cpu(), c.raw)                    # capturing runs nothing
        c.table = tab
        g.replay()
        torch.cuda.synchronize()
        verify(c, q_out)
        c.raw = c.pool.cpu().clone()
        c.lens = [(p + 1, 1) for p, _ in c.lens]
        c.ctx_len = c.ctx_len + 1
        c.t_ctx += 1
        q_out.fill_(7.5)
        g.replay()
        torch.cuda.synchronize()
        verify(c, q_out)
    finally:
        c.close()


def test_append_refusals_on_a_context():
    c = OpCase([(4, 2)], seed=14)
    try:
        tok = T.make_tokens(c.k, c.v)
        call = lambda layer, t: c.ctx.tutti_kv_append_layer(layer, c.step, t, None, allow=(T.EINVAL,))  # noqa: E731
        before = c.pool.clone()
        assert call(0, tok) == T.EINVAL                            # not registered
        assert call(2, tok) == T.EINVAL                            # no such layer
        tok.k += 8
        assert call(1, tok) == T.EINVAL                            # alignment
        assert torch.equal(before, c.pool)
        with pytest.raises(T.TuttiError):
            T.make_tokens(c.k.float(), c.v.float())
        with pytest.raises(T.TuttiError):
            c.ctx.tutti_scales_register(1, c.pool.data_ptr(), c.pool.data_ptr(), c.n_blocks)     # a 16-bit pool has none
    finally:
        c.close()
    e = OpCase([(4, 2)], cache="8", seed=15)
    try:
        e.ctx.tutti_pool_register(1, e.pool.data_ptr() + e.k_off, e.pool.data_ptr() + e.v_off, e.stride, e.n_blocks)
        assert e.ctx.tutti_kv_append_layer(1, e.step, T.make_tokens(e.k, e.v), None, allow=(T.EINVAL,)) == T.EINVAL
    finally:
        e.close()
