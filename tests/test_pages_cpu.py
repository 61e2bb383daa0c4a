"""What the pages' operators and a window's attention refuse, and how a window's tiles are counted, without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests.test_operators_cpu import check_fn, geom


def tables(**kw):
    t = T.Tables(2, 8, 0x1000, 0x2000, 0x3000, None)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def other(**kw):
    return tables(**{"block_ids": 0x12000, "len": 0x13000, **kw})


def call(name, *args):
    f = check_fn(name)
    conv = []
    for a in args:
        conv.append(C.byref(a) if isinstance(a, C.Structure) else C.c_void_p(a) if a is None or a > 0xfff else C.c_uint32(a))
    return f(*conv)


BAD = [dict(blk_start=None), dict(block_ids=None), dict(len=None), dict(n_seq=T.PAGES_MAX_SEQ + 1), dict(n_blk=1 << 31), dict(blk_start=0x1002),
       dict(block_ids=0x2001), dict(len=0x3003), dict(status=0x4002)]


@pytest.mark.parametrize("kw", BAD)
def test_tables_that_are_refused(kw):
    assert call("tutti_tables_check_", tables(**kw)) == T.EINVAL
    assert call("tutti_fork_check_", tables(**kw), 0x5000, other(), 0) == T.EINVAL
    assert call("tutti_fork_check_", other(), 0x5000, tables(**kw), 0) == T.EINVAL
    assert call("tutti_extend_check_", tables(**kw), 0x6000, 0x7000) == T.EINVAL
    assert call("tutti_compact_check_", tables(**kw), 0x7000, 4, 0x8000) == T.EINVAL


def test_calls_that_are_taken():
    assert call("tutti_tables_check_", tables()) == T.OK and call("tutti_tables_check_", tables(status=0x4000, n_seq=T.PAGES_MAX_SEQ)) == T.OK
    assert call("tutti_tables_check_", T.Tables()) == T.OK
    assert call("tutti_fork_check_", tables(), 0x5000, other(), 0) == T.OK and call("tutti_fork_check_", tables(), 0x5000, other(), 1) == T.OK
    assert call("tutti_fork_check_", tables(), None, T.Tables(), 1) == T.OK
    assert call("tutti_extend_check_", tables(), 0x6000, 0x7000) == T.OK and call("tutti_extend_check_", T.Tables(), None, None) == T.OK
    assert call("tutti_compact_check_", tables(), 0x7000, 4, 0x8000) == T.OK
    assert call("tutti_compact_check_", T.Tables(), None, 0, 0x8000) == T.OK


def test_calls_that_are_refused():
    assert call("tutti_fork_check_", tables(), 0x5000, tables(), 0) == T.EINVAL              # shared arrays
    assert call("tutti_fork_check_", tables(), 0x5000, tables(block_ids=0x12000), 0) == T.EINVAL
    assert call("tutti_fork_check_", tables(), 0x5000, tables(len=0x13000), 0) == T.EINVAL
    assert call("tutti_fork_check_", tables(), 0x5000, other(), 2) == T.EINVAL
    assert call("tutti_fork_check_", tables(), None, other(), 0) == T.EINVAL
    assert call("tutti_fork_check_", tables(), 0x5002, other(), 0) == T.EINVAL
    assert call("tutti_extend_check_", tables(), None, 0x7000) == T.EINVAL
    assert call("tutti_extend_check_", tables(), 0x6000, None) == T.EINVAL
    assert call("tutti_extend_check_", tables(), 0x6001, 0x7000) == T.EINVAL
    assert call("tutti_extend_check_", tables(), 0x6000, 0x7002) == T.EINVAL
    assert call("tutti_compact_check_", tables(), None, 4, 0x8000) == T.EINVAL
    assert call("tutti_compact_check_", tables(), 0x7004, 4, 0x8000) == T.EINVAL             # pairs are read as 8 bytes
    assert call("tutti_compact_check_", tables(), 0x7000, 4, None) == T.EINVAL
    assert call("tutti_compact_check_", tables(), 0x7000, 4, 0x8002) == T.EINVAL


@pytest.mark.parametrize("window,sinks,ok", [(1, 0, True), (4096, 4, True), ((1 << 31) - 1, (1 << 31) - 1, True), (0, 4, False), (1 << 31, 0, False), (5, 1 << 31, False)])
def test_windows(window, sinks, ok):
    assert check_fn("tutti_window_check_")(C.byref(T.Window(window, sinks))) == (T.OK if ok else T.EINVAL)
    if ok:
        assert T.make_window(window, sinks).window == window
    else:
        with pytest.raises(T.TuttiError):
            T.make_window(window, sinks)
    assert check_fn("tutti_window_check_")(None) == T.EINVAL


def test_copies_of_blocks():
    g = geom(n_layers=4)
    ok = lambda *a: call("tutti_copy_check_", g, *a)  # noqa: E731
    assert ok(0, 4, 0x1000, 8, None, None) == T.OK and ok(3, 1, 0x1000, 8, 0x2000, 0x3000) == T.OK and ok(4, 0, None, 0, None, None) == T.OK
    for bad in ((0, 5, 0x1000, 8, None, None), (4, 1, 0x1000, 8, None, None), (5, 0, 0x1000, 8, None, None), (0, 4, None, 8, None, None),
                (0, 4, 0x1004, 8, None, None), (0, 4, 0x1000, 8, 0x2002, None), (0, 4, 0x1000, 8, None, 0x3001)):
        assert ok(*bad) == T.EINVAL, bad
    f = check_fn("tutti_copy_check_")
    assert f(C.byref(g), C.c_uint32(0), C.c_uint32(0xffffffff), C.c_void_p(0x1000), C.c_uint32(8), None, None) == T.EINVAL
    assert f(C.byref(g), C.c_uint32(0), C.c_uint32(1), C.c_void_p(0x1000), C.c_uint32(1 << 31), None, None) == T.EINVAL


def test_null_handles():
    lib = T.load()
    t, w = tables(), T.Window(4, 0)
    assert lib.tutti_pages_create(None, None, 0, None) == T.EINVAL and lib.tutti_pages_destroy(None) == T.EINVAL
    assert lib.tutti_pages_fork(None, t, 0x5000, other(), 0, None) == T.EINVAL
    assert lib.tutti_pages_extend(None, t, 0x6000, 0x7000, None) == T.EINVAL
    assert lib.tutti_pages_release(None, t, None, None) == T.EINVAL and lib.tutti_pages_trim(None, t, w, None) == T.EINVAL
    assert lib.tutti_pages_compact(None, t, 0x7000, 4, 0x8000, None) == T.EINVAL
    assert lib.tutti_kv_copy_blocks(None, 0, 1, 0x7000, 4, None, None, None) == T.EINVAL
    assert lib.tutti_kv_attend_window_layer(None, 0, T.Step(), T.Attend(), w, None) == T.EINVAL
    assert C.sizeof(T.Tables) == 40 and C.sizeof(T.Window) == 8


def refused(call, *words):
    with pytest.raises(T.TuttiError) as e:
        call()
    assert e.value.code == T.EINVAL and all(w in str(e.value) for w in words), str(e.value)


def test_binding():
    ints = lambda n, dtype=torch.int32: torch.zeros(n, dtype=dtype)  # noqa: E731
    t = T.make_tables(ints(3), ints(8), ints(2), ints(1))
    assert (t.n_seq, t.n_blk) == (2, 8) and t.status
    assert T.make_tables(ints(9), ints(8), ints(2)).n_seq == 2 and not T.make_tables(ints(9), ints(8), ints(2)).status
    refused(lambda: T.make_tables(ints(2), ints(8), ints(2)), "entry more")
    refused(lambda: T.make_tables(ints(3), ints(8, torch.int64), ints(2)), "int32")
    refused(lambda: T.make_tables(ints(3), ints(16)[::2], ints(2)), "contiguous")
    refused(lambda: T.make_tables(ints(3), ints(8), ints(2), ints(0)), "status")
    ctx = T.Context.__new__(T.Context)
    ctx.lib, ctx.h, ctx.device, ctx._row = T.load(), C.c_void_p(None), -1, (2, 64)           # "GPU" -1: tensors in host memory
    refused(lambda: T.Pages(ctx, ints(8, torch.float32)), "refs")
    refused(lambda: T.Pages(ctx, ints(0)), "refs")
    refused(lambda: T.Pages(ctx, ints(8)), "tutti_pages_create")                             # reaches the library: no context
    p = T.Pages.__new__(T.Pages)
    p.ctx, p.lib, p.h = ctx, ctx.lib, C.c_void_p(None)
    allow = dict(allow=(T.EINVAL,))
    assert p.tutti_pages_fork(t, ints(2), t, **allow) == T.EINVAL                            # these reach the library
    assert p.tutti_pages_extend(t, ints(2), torch.zeros(2, 2, dtype=torch.int32), **allow) == T.EINVAL
    assert p.tutti_pages_release(t, torch.zeros(2, dtype=torch.bool), **allow) == T.EINVAL
    assert p.tutti_pages_trim(t, T.make_window(4), **allow) == T.EINVAL
    assert p.tutti_pages_compact(t, torch.zeros(3, 2, dtype=torch.int32), ints(1), **allow) == T.EINVAL
    refused(lambda: p.tutti_pages_fork(t, ints(1), t), "parent")
    refused(lambda: p.tutti_pages_fork(t, ints(2, torch.int64), t), "parent")
    refused(lambda: p.tutti_pages_extend(t, ints(1), torch.zeros(2, 2, dtype=torch.int32)), "n_new")
    refused(lambda: p.tutti_pages_extend(t, ints(2), ints(3)), "pairs")
    refused(lambda: p.tutti_pages_release(t, ints(2)), "which")
    refused(lambda: p.tutti_pages_release(t, torch.zeros(1, dtype=torch.bool)), "which")
    refused(lambda: p.tutti_pages_compact(t, ints(6), ints(1)), "[n, 2]")
    refused(lambda: p.tutti_pages_compact(t, torch.zeros(3, 2, dtype=torch.int32), ints(0)), "n_pairs")
    refused(lambda: ctx.tutti_kv_copy_blocks(0, 1, ints(6)), "[n, 2]")
    refused(lambda: ctx.tutti_kv_copy_blocks(0, 1, torch.zeros(3, 2)), "pairs")
    refused(lambda: ctx.tutti_kv_copy_blocks(0, 1, torch.zeros(2, 3, dtype=torch.int32).t()), "pairs")
    refused(lambda: ctx.tutti_kv_copy_blocks(0, 1, torch.zeros(3, 2, dtype=torch.int32), ints(0)), "n_pairs")
    ctx.device = 0
    refused(lambda: p.tutti_pages_trim(t, T.make_window(4)), "cpu", "GPU 0")
    p.h = None
    refused(lambda: p.tutti_pages_trim(t, T.make_window(4)), "closed")


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 64, 300])
def test_a_windows_tiles_have_every_key_that_a_row_sees_once(group):
    """The keys of a tile, laid end to end without the ones that none of its rows sees: all that a row sees are among them, none
    is there twice, a unit is at most lost to rounding, and the units of the tiles in front are counted in closed form."""
    f = check_fn("tutti_many_window_units_")
    f.argtypes = [C.c_uint32] * 7 + [C.POINTER(C.c_uint64)]
    rng = np.random.default_rng(group)
    out = (C.c_uint64 * 4)()
    cases = [(1, 1, 1, 0, 16), (5000, 700, 1024, 4, 16), (2000, 2000, 1, 0, 1), (2000, 2000, 128, 128, 64), (40000, 3, 4096, 16, 128), (10, 30, 5, 2, 16), (0, 5, 7, 1, 16),
             (131072, 1000, 4096, 200, 8), (5000, 5000, (1 << 31) - 1, (1 << 31) - 1, 16), (5000, 5000, 100, (1 << 31) - 1, 16), (5000, 5000, (1 << 31) - 1, 0, 24)]
    cases += [tuple(int(x) for x in c) for c in zip(rng.integers(0, 6000, 60), rng.integers(1, 900, 60), np.exp(rng.uniform(0, 9, 60)), rng.integers(0, 400, 60),
                                                   rng.choice([1, 2, 5, 8, 16, 24, 32, 64, 128, 192], 60))]
    for ctx, new, window, sinks, bs in cases:
        rows, first = new * group, ctx - new
        tiles = -(-rows // 256)
        grain = bs if 64 % bs == 0 else 64 if bs % 64 == 0 else 16
        total, front = 0, -(-sinks // grain) * grain
        for q in range(tiles):
            a, b = first + q * 256 // group, first + (min(rows, (q + 1) * 256) - 1) // group
            assert f(ctx, new, group, window, sinks, bs, q, out) == tiles
            units, before, got_front, shift = tuple(out)
            assert (before, got_front) == (total, front), (ctx, new, window, sinks, bs, q)
            full = b // 128 + 1 if first >= 0 and ctx else max(1, -(-ctx // 128))
            if shift:
                assert first >= 0 and shift >= 128 and shift % grain == 0
                v = np.arange(128 * units)
                keys = np.where(v < front, v, v + shift)
                lo = max(0, a - window + 1)
                need = np.concatenate([np.arange(min(sinks, lo)), np.arange(lo, b + 1)])
                assert len(np.unique(keys)) == len(keys) and np.isin(need, keys).all(), (ctx, new, window, sinks, bs, q)
                assert units <= full and 128 * units < front + 256 // group + 3 + window + 2 * grain + 128
            else:
                assert units == full
            total += units
        f(ctx, new, group, window, sinks, bs, tiles, out)
        assert out[1] == total
