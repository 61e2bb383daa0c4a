"""What the operators on the pool refuse, and how they see a step's tables, without a GPU: the
checks of arguments, of a sequence's numbers and of block ids are the library's own."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_03375_b200 import tutti as T


def check_fn(name):
    f = getattr(T.load(), name)
    f.restype = C.c_int
    return f


def geom(**kw):
    g = dict(n_layers=1, n_kv_heads=2, head_dim=128, elem_bytes=2, block_tokens=16, obj_tokens=16, n_devices=1, layout=1, n_slots=1)
    g.update(kw)
    return T.Geom(*g.values())


def step(**kw):
    s = T.Step(2, 4, 8, 3, 0x1000, 0x2000, 0x3000, 0x4000, None)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def tokens(**kw):
    t = T.Tokens(T.DTYPE_BF16, 8, 1536, 1536, 1536, 1024, 0x10000, 0x20000, 0x30000, 0x40000)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def rope(**kw):
    r = T.Rope(T.ROPE_HALF, 128, 100, 0x50000)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def attend(**kw):
    a = T.Attend(T.DTYPE_FP16, 8, 1536, 1024, 0x10000, 0x20000, 0x30000, 0.1, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def append_rc(g=None, s=None, t=None, r=None):
    return check_fn("tutti_append_check_")(C.byref(g or geom()), C.byref(s or step()), C.byref(t or tokens()), C.byref(r) if r else None)


def attend_rc(g=None, s=None, a=None):
    return check_fn("tutti_attend_check_")(C.byref(g or geom()), C.byref(s or step()), C.byref(a or attend()))


BAD_STEPS = [dict(q_start=None), dict(ctx_len=None), dict(blk_start=None), dict(block_ids=None), dict(max_new=0),
             dict(q_start=0x1001), dict(ctx_len=0x2002), dict(block_ids=0x4003), dict(status=0x5001), dict(n_tok=1 << 31)]


@pytest.mark.parametrize("kw", BAD_STEPS)
def test_steps_that_are_refused(kw):
    assert append_rc(s=step(**kw)) == T.EINVAL
    assert attend_rc(s=step(**kw)) == T.EINVAL


def test_calls_that_are_taken():
    assert append_rc() == T.OK and append_rc(r=rope()) == T.OK and append_rc(r=rope(rot_dim=16, style=T.ROPE_PAIRS)) == T.OK
    assert append_rc(geom(head_dim=80, elem_bytes=1)) == T.OK
    assert append_rc(t=tokens(n_q_heads=0, q=None, q_out=None, q_stride=0, q_out_stride=0)) == T.OK
    assert append_rc(s=step(n_tok=0)) == T.OK and append_rc(s=T.Step()) == T.OK
    assert attend_rc() == T.OK and attend_rc(geom(head_dim=64, elem_bytes=1)) == T.OK and attend_rc(a=attend(lse=None)) == T.OK
    assert attend_rc(s=T.Step()) == T.OK and attend_rc(a=attend(scale=-1.0)) == T.OK


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(n_q_heads=7), dict(q_stride=1020), dict(k_stride=128), dict(v_stride=1540), dict(q_out_stride=1016),
    dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(k=0x20008), dict(q_out=0x40002), dict(n_q_heads=0)])
def test_tokens_that_are_refused(kw):
    assert append_rc(t=tokens(**kw)) == T.EINVAL


def test_queries_in_place_have_one_stride():
    q = dict(q=0x10000, q_out=0x10000, q_stride=1536)
    assert append_rc(t=tokens(q_out_stride=1536, **q)) == T.OK
    assert append_rc(t=tokens(q_out_stride=1024, **q)) == T.EINVAL
    assert append_rc(t=tokens(q_out_stride=1024, **q), s=step(n_tok=1)) == T.OK


@pytest.mark.parametrize("kw", [dict(style=2), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(table=None),
                                dict(table=0x50008), dict(n_pos=0)])
def test_rotations_that_are_refused(kw):
    assert append_rc(r=rope(**kw)) == T.EINVAL


@pytest.mark.parametrize("kw", [dict(elem_bytes=4), dict(head_dim=72), dict(head_dim=272)])
def test_geometries_that_append_refuses(kw):
    assert append_rc(geom(**kw), t=tokens(q_stride=4096, k_stride=4096, v_stride=4096, q_out_stride=4096)) == T.EINVAL


@pytest.mark.parametrize("kw", [dict(elem_bytes=4), dict(head_dim=96), dict(head_dim=256), dict(n_kv_heads=3)])
def test_geometries_that_attend_refuses(kw):
    assert attend_rc(geom(**kw), a=attend(q_stride=4096, out_stride=4096)) == T.EINVAL


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(n_q_heads=0), dict(n_q_heads=5), dict(q_stride=1000), dict(out_stride=1020),
                                dict(q=None), dict(out=None), dict(out=0x10000), dict(q=0x10008), dict(lse=0x30002), dict(scale=float("inf")),
                                dict(scale=float("nan")), dict(reserved=1)])
def test_attends_that_are_refused(kw):
    assert attend_rc(a=attend(**kw)) == T.EINVAL


def test_more_rows_than_are_counted_in_31_bits():
    assert attend_rc(s=step(n_tok=1 << 28), a=attend(n_q_heads=8)) == T.EINVAL
    assert attend_rc(s=step(n_tok=(1 << 28) - 1), a=attend(n_q_heads=8)) == T.OK


def test_null_handles():
    lib = T.load()
    assert lib.tutti_kv_append_layer(None, 0, step(), tokens(), None, None) == T.EINVAL
    assert lib.tutti_kv_attend_layer(None, 0, step(), attend(), None) == T.EINVAL
    assert lib.tutti_attn_create(None, None) == T.EINVAL and lib.tutti_attn_destroy(None) == T.EINVAL
    assert lib.tutti_scales_register(None, 0, None, None, 0) == T.EINVAL
    assert check_fn("tutti_append_check_")(None, C.byref(step()), C.byref(tokens()), None) == T.EINVAL
    assert check_fn("tutti_append_check_")(C.byref(geom()), None, C.byref(tokens()), None) == T.EINVAL
    assert check_fn("tutti_append_check_")(C.byref(geom()), C.byref(step()), None, None) == T.EINVAL
    assert check_fn("tutti_attend_check_")(C.byref(geom()), C.byref(step()), None) == T.EINVAL


def test_struct_sizes_match_the_header():
    assert C.sizeof(T.Step) == 56 and C.sizeof(T.Tokens) == 72 and C.sizeof(T.Rope) == 24 and C.sizeof(T.Attend) == 56


def views(q_start, ctx, blk_start, n_tok, n_blk, max_new, bs=16):
    a = [np.asarray(x, dtype=np.uint32) for x in (q_start, ctx, blk_start)]
    s = T.Step(len(ctx), n_tok, n_blk, max_new, *(x.ctypes.data for x in a), None, None)
    f, out, got = check_fn("tutti_seq_view_"), (C.c_uint32 * 4)(), []
    for i in range(len(ctx)):
        rc = f(C.byref(s), bs, i, out)
        got.append((rc, *out) if rc == T.OK else rc)
    return got


def test_sequences_that_contradict_their_sizes():
    ok = T.OK
    assert views([0, 1, 3], [16, 20], [0, 1, 3], 3, 3, 2) == [(ok, 0, 1, 16, 0), (ok, 1, 2, 20, 1)]
    assert views([0, 1, 3], [17, 20], [0, 1, 3], 3, 3, 2)[0] == T.EINVAL           # more tokens than its blocks hold
    assert views([0, 1, 3], [16, 20], [0, 1, 3], 2, 3, 2)[1] == T.EINVAL           # rows behind the arrays
    assert views([0, 1, 3], [16, 20], [0, 1, 3], 3, 2, 2)[1] == T.EINVAL           # blocks behind the array
    assert views([0, 1, 3], [16, 20], [0, 1, 3], 3, 3, 1)[1] == T.EINVAL           # more rows than max_new
    assert views([2, 1, 3], [16, 20], [0, 1, 3], 3, 3, 2)[0] == T.EINVAL           # starts that go back
    assert views([0, 1, 3], [16, 20], [2, 1, 3], 3, 3, 2)[0] == T.EINVAL
    assert views([0, 1, 3], [0xffffffff, 0], [0, 1, 1], 3, 3, 2) == [T.EINVAL, (ok, 1, 2, 0, 1)]
    assert views([0, 0], [0], [0, 0], 0, 0, 1) == [(ok, 0, 0, 0, 0)]
    assert views([0, 1], [5], [0, 5], 1, 5, 1, bs=1) == [(ok, 0, 1, 5, 0)]


def test_block_ids_outside_the_pool():
    f = check_fn("tutti_block_offset_")
    f.restype, f.argtypes = C.c_int64, [C.c_uint32, C.c_uint64, C.c_int32]
    assert [f(10, 4096, i) for i in (0, 9, 10, -1, -(1 << 31), (1 << 31) - 1)] == [0, 9 * 4096, -1, -1, -1, -1]
    assert f(1 << 30, 32768, (1 << 30) - 1) == ((1 << 30) - 1) * 32768            # offsets pass 32 bits


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 64, 300])
def test_units_of_causal_tiles_in_closed_form(group):
    """The number of 128-key units that 256-row tiles of a sequence see, against counting them."""
    f = check_fn("tutti_many_units_")
    f.argtypes = [C.c_uint32] * 4 + [C.POINTER(C.c_uint64)]
    rng = np.random.default_rng(group)
    out = (C.c_uint64 * 2)()
    for ctx, new in [(1, 1), (128, 128), (129, 1), (5000, 700), (2000, 2000), (40000, 3), (10, 30), (0, 5), (131072, 1000)] + \
            [(int(c), int(n)) for c, n in zip(rng.integers(0, 3000, 30), rng.integers(1, 900, 30))]:
        rows, first = new * group, ctx - new
        tiles = -(-rows // 256)
        total = 0
        for q in range(tiles):
            last = first + (min(rows, (q + 1) * 256) - 1) // group
            want = last // 128 + 1 if first >= 0 and ctx else max(1, -(-ctx // 128))
            assert f(ctx, new, group, q, out) == tiles
            assert (out[0], out[1]) == (want, total), (ctx, new, group, q)
            total += want
        f(ctx, new, group, tiles, out)
        assert out[1] == total


def test_shares_of_workers_cover_tiles_once_and_agree_on_their_parts():
    """Cuts moved to tile ends: shares are consecutive, and the workers that a tile's formula names are the ones that hold its parts."""
    lib = T.load()
    cut, parts = lib.tutti_many_cut_, lib.tutti_many_parts_
    cut.argtypes = [C.c_void_p, C.c_uint32, C.c_uint64, C.c_uint64, C.POINTER(C.c_uint64)]
    parts.argtypes = [C.c_uint64, C.c_uint32, C.c_uint64, C.c_uint64, C.POINTER(C.c_uint64)]
    rng = np.random.default_rng(5)
    out = (C.c_uint64 * 2)()
    for trial in range(300):
        n = rng.integers(1, [3, 8, 40, 300][trial % 4], rng.integers(1, 60)).astype(np.uint32)
        total = int(n.sum())
        workers = int(rng.integers(1, min(148, total) + 1))
        shares = []
        for w in range(workers):
            cut(n.ctypes.data, len(n), workers, w, out)
            shares.append((out[0], out[1]))
        assert shares[0][0] == 0 and shares[-1][1] == total
        assert all(a[1] == b[0] and a[0] <= a[1] for a, b in zip(shares, shares[1:] + [(total, total)]))
        start = 0
        for k in n:
            holders = [w for w, (a, b) in enumerate(shares) if max(a, start) < min(b, start + int(k))]
            parts(start, int(k), workers, total, out)
            assert holders == list(range(out[0], out[1] + 1)), (trial, start, k, holders, out[0], out[1])
            if k <= 6:
                assert len(holders) == 1
            start += int(k)


def test_structs_from_tensors():
    """The binding's own checks of types, shapes and strides."""
    import torch
    k, q = torch.zeros(4, 2, 64, dtype=torch.float16), torch.zeros(4, 8, 64, dtype=torch.float16)
    t = T.make_tokens(k, k, q, q)
    assert (t.dtype, t.n_q_heads, t.q_stride, t.k_stride, t.v_stride, t.q_out_stride) == (T.DTYPE_FP16, 8, 512, 128, 128, 512)
    one = torch.zeros(4, 3, 64, dtype=torch.float16)[:, 1:2]               # one head of a packed row
    assert T.make_tokens(one, one).k_stride == 192
    a = T.make_attend(q, q, torch.zeros(4, 8))
    assert (a.n_q_heads, a.q_stride, a.out_stride) == (8, 512, 512) and a.lse
    assert T.make_rope(torch.zeros(10, 32), T.ROPE_PAIRS).rot_dim == 32
    half = torch.float16
    for bad in (lambda: T.make_tokens(k, k.float()), lambda: T.make_tokens(k.float(), k.float()),
                lambda: T.make_tokens(k, k, torch.zeros(4, 8, 32, dtype=half), q), lambda: T.make_tokens(k.transpose(1, 2), k),
                lambda: T.make_tokens(k, torch.zeros(4, 2, 128, dtype=half)[:, :, ::2]), lambda: T.make_tokens(one, torch.zeros(4, 1, 32, dtype=half)),
                lambda: T.make_tokens(k, torch.zeros(2, 4, 64, dtype=half).transpose(0, 1)), lambda: T.make_attend(q, q.transpose(0, 1)),
                lambda: T.make_attend(q, q, torch.zeros(4, 8, dtype=half)), lambda: T.make_rope(torch.zeros(10, 32, dtype=half)),
                lambda: T.make_step(torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                                    torch.zeros(1, dtype=torch.int32), 1, 1)):
        with pytest.raises(T.TuttiError):
            bad()
