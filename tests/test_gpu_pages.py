"""The operators on pages against their statement row by row (whole numbers: equal), and copies of blocks byte by byte."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests import pagecase as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def contexts():
    made = {}

    def get(bs):
        if bs not in made:
            made[bs] = T.Context(T.Geom(1, 2, 64, 2, bs, bs, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
        return made[bs]
    yield get
    torch.cuda.synchronize()
    for c in made.values():
        c.close()


def ints(v, dev="cuda:0"):
    return torch.tensor(v, dtype=torch.int32, device=dev)


SHAPES = [(1, 1, 1, 3), (5, 16, 60, 90), (64, 16, 4097, 700), (300, 1, 12000, 60), (1500, 8, 20000, 100), (7, 24, 33, 200), (2, 1, 9001, 4500)]


@pytest.mark.parametrize("n_seq,bs,n_blocks,most", SHAPES)
@pytest.mark.parametrize("move", [T.FORK_KEEP, T.FORK_MOVE])
def test_fork(contexts, n_seq, bs, n_blocks, most, move):
    rng = np.random.default_rng(n_seq + move)
    frm, refs = P.random_book(rng, n_seq, bs, n_blocks, most, trimmed=0.1)
    n_to = 64 if n_seq == 64 else int(rng.integers(1, 2 * n_seq + 1))
    parent = np.arange(64) if n_seq == 64 else rng.integers(-1, n_seq, n_to)       # 64: every row takes its own place
    room = max([frm.row(s)[3] for s in range(n_seq)]) + 2
    to = P.Book(np.arange(n_to + 1) * room + 3, [-9] * (n_to * room + 5), [77] * n_to, bs)
    b = P.Bound(contexts(bs), [frm, to], refs)
    try:
        b.pages.tutti_pages_fork(b.tables(0), ints(parent), b.tables(1), move)
        P.fork(frm, parent, to, refs, move)
        b.same(refs, 0)
        b.same(refs, 1)
    finally:
        b.close()


@pytest.mark.parametrize("n_seq,bs,n_blocks,most", SHAPES)
@pytest.mark.parametrize("most_new", [1, 40])
def test_extend(contexts, n_seq, bs, n_blocks, most, most_new):
    rng = np.random.default_rng(n_seq + most_new)
    spare = P.blocks_of(most_new, bs) + 1
    book, refs = P.random_book(rng, n_seq, bs, max(1, n_blocks * 3 // 4), most, share=0.6, spare=0)
    # room for new blocks behind every row
    start, ids = [0], []
    for s in range(n_seq):
        a, _, _, h = book.row(s)
        ids += book.ids[a:a + h] + [-7] * spare
        start.append(len(ids))
    book = P.Book(start, ids, book.lens, bs)
    refs += [0] * (n_blocks - len(refs) + n_seq * spare)
    n_new = rng.integers(0 if most_new > 1 else 1, most_new + 1, n_seq)
    b = P.Bound(contexts(bs), [book], refs)
    pairs = torch.full((n_seq, 2), 55, dtype=torch.int32, device=b.dev)
    try:
        for _ in range(3):                                      # the workspace is ready again each time
            b.pages.tutti_pages_extend(b.tables(), ints(n_new), pairs)
            want = P.extend(book, refs, n_new)
            b.same(refs)
            assert pairs.tolist() == [list(p) for p in want]
            n_new = np.minimum(n_new, 0)
            n_new[:] = [1 if s % 3 == 0 and (book.lens[s] % bs or (n := book.row(s))[3] < n[1]) else 0 for s in range(n_seq)]
    finally:
        b.close()


def test_extend_shares_of_one_block(contexts):
    """Rows that write to one block: with and without another holder, first and last, and one that does not write."""
    bs = 16
    rows = [[0, 1], [0, 1], [0, 1], [2, 3], [2, 3], [4], [4], [5, 6], [5, 6]]
    lens = [20, 20, 20, 30, 30, 7, 7, 32, 32]
    n_new = [1, 1, 1, 3, 0, 9, 10, 1, 17]
    for extra in ([], [1], [3, 6]):
        start, ids = [0], []
        for r in rows:
            ids += r + [-7] * 3
            start.append(len(ids))
        refs = [0] * 30
        for i in sum(rows, []) + extra:
            refs[i] += 1
        book = P.Book(start, ids, list(lens), bs)
        b = P.Bound(contexts(bs), [book], refs)
        pairs = torch.zeros(len(rows), 2, dtype=torch.int32, device=b.dev)
        try:
            b.pages.tutti_pages_extend(b.tables(), ints(n_new), pairs)
            want = P.extend(book, refs, n_new)
            assert sum(p != (-1, -1) for p in want) >= 4
            b.same(refs)
            assert pairs.tolist() == [list(p) for p in want]
        finally:
            b.close()


def test_extend_behind_an_entry_without_a_block(contexts):
    """A row whose partly filled block is gone grows: nothing is copied, nobody shares it."""
    book = P.Book([0, 3, 6], [0, -1, -7, 0, -1, -7], [6, 7], 4)
    refs = [2, 0, 0, 0]
    b = P.Bound(contexts(4), [book], refs)
    pairs = torch.zeros(2, 2, dtype=torch.int32, device=b.dev)
    try:
        b.pages.tutti_pages_extend(b.tables(), ints([1, 2]), pairs)
        assert pairs.tolist() == [list(p) for p in P.extend(book, refs, [1, 2])] and not book.status
        assert book.lens == [7, 9] and book.ids[5] == 1
        b.same(refs)
    finally:
        b.close()


@pytest.mark.parametrize("n_free", [0, 1, 6, 7])
def test_extend_takes_all_or_nothing(contexts, n_free):
    bs = 4
    book = P.Book([0, 4, 8, 12], [0, 1, -7, -7, 0, 1, -7, -7, 2, -7, -7, -7], [7, 7, 4], bs)
    refs = [2, 2, 1] + [3] * 5 + [0] * n_free
    n_new = [8, 8, 8]                                           # 1 copied, 2 + 2 + 2 new: 7
    b = P.Bound(contexts(bs), [book], refs)
    pairs = torch.zeros(3, 2, dtype=torch.int32, device=b.dev)
    try:
        for _ in range(2):
            b.pages.tutti_pages_extend(b.tables(), ints(n_new), pairs)
            want = P.extend(book, refs, n_new)
            b.same(refs)
            assert pairs.tolist() == [list(p) for p in want]
            assert (book.status == {T.EAGAIN}) == (n_free < 7)
            if n_free == 7:
                break
        if n_free < 7:                                          # the workspace is as it was: with blocks it goes on
            b.pages.refs[3:6] = 0
            refs[3:6] = [0] * 3
            b.t[0][4].zero_()
            book.status.clear()
            if n_free >= 4:
                b.pages.tutti_pages_extend(b.tables(), ints(n_new), pairs)
                want = P.extend(book, refs, n_new)
                b.same(refs)
                assert pairs.tolist() == [list(p) for p in want]
    finally:
        b.close()


def test_extend_rows_that_lie_over_each_other(contexts):
    """Starts that go back make rows of the same entries: more new blocks than entries are refused, before any list runs out."""
    book = P.Book([0, 5, 0, 5], [-7] * 5, [0, 0, 0], 4)
    refs = [0] * 20
    b = P.Bound(contexts(4), [book], refs)
    pairs = torch.zeros(3, 2, dtype=torch.int32, device=b.dev)
    try:
        b.pages.tutti_pages_extend(b.tables(), ints([20, 0, 20]), pairs)
        assert pairs.tolist() == [list(p) for p in P.extend(book, refs, [20, 0, 20])]
        assert not any(refs) and book.status == {T.EINVAL}
        b.same(refs)
    finally:
        b.close()


def test_extend_among_millions_of_blocks(contexts):
    """More tiles of counts than threads; the lowest free ids are far behind."""
    bs, n = 16, 5_000_000
    book = P.Book(np.arange(5) * 3000, [-7] * 12000, [0] * 4, bs)
    b = P.Bound(contexts(bs), [book], [0])
    try:
        b.pages.close()
        refs = torch.ones(n, dtype=torch.int32, device=b.dev)
        free = torch.tensor([4_300_000, 4_300_001, 4_999_999], device=b.dev)
        refs[free] = 0
        refs[4_400_000:4_405_000] = 0
        b.pages = T.Pages(contexts(bs), refs)
        pairs = torch.zeros(4, 2, dtype=torch.int32, device=b.dev)
        order = [4_300_000, 4_300_001] + list(range(4_400_000, 4_405_000)) + [4_999_999]
        take = [3 * bs, 0, 2900 * bs - 5, 2 * bs]
        b.pages.tutti_pages_extend(b.tables(), ints(take), pairs)
        ids, at = b.t[0][2].tolist(), 0
        for s, k in enumerate([3, 0, 2900, 2]):
            assert ids[s * 3000:s * 3000 + k] == order[at:at + k] and ids[s * 3000 + k] == -7
            at += k
        assert int(refs.sum()) == n - 5003 + at and b.t[0][3].tolist() == take and (pairs == -1).all()
    finally:
        b.close()


def test_extend_more_rows_than_fit_in_shared_memory(contexts):
    rng = np.random.default_rng(3)
    n_seq, bs = 9000, 4
    lens = rng.integers(0, 9, n_seq)
    start = np.arange(n_seq + 1) * 4
    ids, refs, at = [-7] * (4 * n_seq), [], 0
    for s, n in enumerate(lens):
        for k in range(P.blocks_of(int(n), bs)):
            ids[4 * s + k] = at
            at += 1
    refs = [1] * at + [0] * (2 * n_seq)
    book = P.Book(start, ids, lens, bs)
    n_new = rng.integers(0, 6, n_seq)
    b = P.Bound(contexts(bs), [book], refs)
    pairs = torch.zeros(n_seq, 2, dtype=torch.int32, device=b.dev)
    try:
        b.pages.tutti_pages_extend(b.tables(), ints(n_new), pairs)
        P.extend(book, refs, n_new)
        b.same(refs)
    finally:
        b.close()


@pytest.mark.parametrize("n_seq,bs,n_blocks,most", SHAPES)
@pytest.mark.parametrize("all_rows", [False, True])
def test_release(contexts, n_seq, bs, n_blocks, most, all_rows):
    rng = np.random.default_rng(n_seq)
    book, refs = P.random_book(rng, n_seq, bs, n_blocks, most, trimmed=0.2)
    which = rng.random(n_seq) < 0.5
    b = P.Bound(contexts(bs), [book], refs)
    try:
        for _ in range(2):                                      # the second time there is nothing left
            b.pages.tutti_pages_release(b.tables(), None if all_rows else torch.from_numpy(which).to(b.dev))
            P.release(book, refs, None if all_rows else which)
            b.same(refs)
        assert not all_rows or not any(refs)
    finally:
        b.close()


@pytest.mark.parametrize("n_seq,bs,n_blocks,most", SHAPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (50, 16), (17, 33), ((1 << 31) - 1, 0), (1, (1 << 31) - 1)])
def test_trim(contexts, n_seq, bs, n_blocks, most, window, sinks):
    rng = np.random.default_rng(n_seq + window % 100)
    book, refs = P.random_book(rng, n_seq, bs, n_blocks, most)
    b = P.Bound(contexts(bs), [book], refs)
    try:
        for _ in range(2):
            b.pages.tutti_pages_trim(b.tables(), T.make_window(window, sinks))
            P.trim(book, refs, window, sinks)
            b.same(refs)
    finally:
        b.close()


@pytest.mark.parametrize("n_seq,bs,n_blocks,most", SHAPES)
@pytest.mark.parametrize("max_pairs", [0, 1, 5, 100000])
def test_compact(contexts, n_seq, bs, n_blocks, most, max_pairs):
    rng = np.random.default_rng(n_seq)
    book, refs = P.random_book(rng, n_seq, bs, n_blocks, most, trimmed=0.1)
    other = rng.choice(n_blocks, n_blocks // 5, replace=False)  # blocks of holders that the table does not name
    for i in other:
        refs[i] += 1
    b = P.Bound(contexts(bs), [book], refs)
    pairs = torch.full((max_pairs, 2), 55, dtype=torch.int32, device=b.dev)
    n_pairs = torch.full((1,), 55, dtype=torch.int32, device=b.dev)
    try:
        for _ in range(3):                                      # goes on where the moves ended
            b.pages.tutti_pages_compact(b.tables(), pairs, n_pairs)
            moves = P.compact(book, refs, max_pairs)
            b.same(refs)
            assert int(n_pairs) == len(moves) and pairs[:len(moves)].tolist() == [list(m) for m in moves] and (pairs[len(moves):] == -1).all()
        n = sum(x > 0 for x in refs)
        assert max_pairs < 100000 or all(refs[:n])
    finally:
        b.close()


@pytest.mark.parametrize("n_blocks", [1, 4, 4096, 8191])
@pytest.mark.parametrize("used", ["none", "all", "low", "high"])
def test_compact_at_the_ends(contexts, n_blocks, used):
    k = {"none": 0, "all": n_blocks}.get(used, n_blocks // 2)
    refs = [1] * k + [0] * (n_blocks - k)
    if used == "high":
        refs.reverse()
    book = P.Book([0], [], [], 16)
    b = P.Bound(contexts(16), [book], refs)
    pairs, n_pairs = torch.zeros(n_blocks, 2, dtype=torch.int32, device=b.dev), torch.zeros(1, dtype=torch.int32, device=b.dev)
    try:
        b.pages.tutti_pages_compact(T.Tables(), pairs, n_pairs)
        moves = P.compact(book, refs, n_blocks)
        assert b.refs.tolist() == refs and int(n_pairs) == len(moves) and pairs[:len(moves)].tolist() == [list(m) for m in moves]
    finally:
        b.close()


def broken_book(bs=4):
    """Rows that contradict their sizes between rows that do not."""
    start = [0, 3, 6, 5, 9, 12, 15, 99, 18]
    ids = list(range(18))
    lens = [9, 20, 4, 12, MAXL, 8, 4, 4]
    return P.Book(start, ids, lens, bs)


MAXL = 0xffffffff


@pytest.mark.parametrize("what", ["fork", "extend", "release", "trim", "compact"])
def test_rows_that_contradict_their_sizes_are_skipped(contexts, what):
    bs, book = 4, broken_book()
    refs = [1] * 18 + [0] * 10
    n_seq = len(book.lens)
    to = P.Book(np.arange(n_seq + 1) * 3, [-9] * (3 * n_seq), [1] * n_seq, bs)
    b = P.Bound(contexts(bs), [book, to], refs)
    pairs, one = torch.zeros(n_seq, 2, dtype=torch.int32, device=b.dev), torch.zeros(1, dtype=torch.int32, device=b.dev)
    try:
        if what == "fork":
            parent = [0, 1, 3, 7, -1, 5, 8, -5]
            b.pages.tutti_pages_fork(b.tables(0), ints(parent), b.tables(1), T.FORK_MOVE)
            P.fork(book, parent, to, refs, T.FORK_MOVE)
            b.same(refs, 1)
        elif what == "extend":
            n_new = [1, 1, 1, 0, 1, 4, MAXL >> 1, 1]
            b.pages.tutti_pages_extend(b.tables(0), ints(n_new), pairs)
            assert pairs.tolist() == [list(p) for p in P.extend(book, refs, n_new)]
        elif what == "release":
            b.pages.tutti_pages_release(b.tables(0))
            P.release(book, refs, None)
        elif what == "trim":
            b.pages.tutti_pages_trim(b.tables(0), T.make_window(1))
            P.trim(book, refs, 1, 0)
        else:
            refs[2] = 0
            b.refs[2] = 0
            b.pages.tutti_pages_compact(b.tables(0), pairs, one)
            P.compact(book, refs, n_seq)
        assert book.status
        b.same(refs)
    finally:
        b.close()


@pytest.mark.parametrize("what", ["fork", "extend", "release", "trim", "compact"])
def test_ids_outside_the_pool_are_reported(contexts, what):
    bs = 4
    book = P.Book([0, 4, 8], [0, 99, -5, 2, 3, 99, -7, -7], [16, 6], bs)
    refs = [1] * 5 + [0] * 3
    to = P.Book([0, 4, 8], [-9] * 8, [0] * 2, bs)
    b = P.Bound(contexts(bs), [book, to], refs)
    pairs, one = torch.zeros(2, 2, dtype=torch.int32, device=b.dev), torch.zeros(1, dtype=torch.int32, device=b.dev)
    try:
        if what == "fork":
            b.pages.tutti_pages_fork(b.tables(0), ints([0, 0]), b.tables(1))
            P.fork(book, [0, 0], to, refs, T.FORK_KEEP)
            b.same(refs, 1)
        elif what == "extend":
            b.pages.tutti_pages_extend(b.tables(0), ints([0, 1]), pairs)
            assert pairs.tolist() == [list(p) for p in P.extend(book, refs, [0, 1])]
        elif what == "release":
            b.pages.tutti_pages_release(b.tables(0))
            P.release(book, refs, None)
        elif what == "trim":
            b.pages.tutti_pages_trim(b.tables(0), T.make_window(3))
            P.trim(book, refs, 3, 0)
        else:
            b.pages.tutti_pages_compact(b.tables(0), pairs, one)
            P.compact(book, refs, 2)
        assert book.status == {T.EFAULT}
        b.same(refs)
    finally:
        b.close()


def test_counts_do_not_pass_zero(contexts):
    bs = 4
    book = P.Book([0, 2, 4, 6], [0, 1, 0, 2, 0, 3], [8, 8, 8], bs)
    refs = [1, 1, 0, 1, 5]
    b = P.Bound(contexts(bs), [book], refs)
    try:
        b.pages.tutti_pages_release(b.tables())
        P.release(book, refs, None)
        assert refs == [0, 0, 0, 0, 5] and book.status == {T.EINVAL}
        b.same(refs)
        b.t[0][4].zero_()
        # a written block whose count is 0
        book.lens, book.ids, book.status = [6, 4, 0], [4, 0, 4, 3, 4, 4], set()
        b.t[0][2].copy_(ints(book.ids))
        b.t[0][3].copy_(ints(book.lens))
        pairs = torch.zeros(3, 2, dtype=torch.int32, device=b.dev)
        b.pages.tutti_pages_extend(b.tables(), ints([1, 1, 1]), pairs)
        assert pairs.tolist() == [list(p) for p in P.extend(book, refs, [1, 1, 1])] and book.status == {T.EINVAL}
        b.same(refs)
    finally:
        b.close()


def test_empty_tables(contexts):
    p = T.Pages(contexts(16), torch.zeros(5, dtype=torch.int32, device="cuda:0"))
    none = T.make_tables(ints([0]), ints([]), ints([]))
    one = torch.full((1,), 55, dtype=torch.int32, device="cuda:0")
    try:
        p.tutti_pages_fork(none, ints([]), T.Tables(), T.FORK_MOVE)
        p.tutti_pages_extend(none, ints([]), torch.zeros(0, 2, dtype=torch.int32, device="cuda:0"))
        p.tutti_pages_release(none)
        p.tutti_pages_trim(none, T.make_window(4))
        p.tutti_pages_compact(none, torch.zeros(0, 2, dtype=torch.int32, device="cuda:0"), one)
        assert int(one) == 0 and not p.refs.any()
    finally:
        torch.cuda.synchronize()
        p.close()


# ---------------------------------------------------------------------------- copies

def pool_of(hk, dim, size, bs, layers, n_blocks, pad=0, interleaved=False, rows=None, seed=0):
    """A context with `layers` registered layers of random bytes, and their tensors [plane, block, bytes] as views."""
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    bb = bs * hk * dim * size
    stride = (2 if interleaved else 1) * bb + pad
    ctx = T.Context(T.Geom(layers + 1, hk, dim, size, bs, bs, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
    raw = torch.randint(0, 256, (layers, (1 if interleaved else 2) * n_blocks * stride), dtype=torch.uint8, generator=g, device="cuda:0")
    scales = torch.randn(layers, 2, n_blocks, rows, generator=g, device="cuda:0") if rows else None
    for l in range(layers):
        k = raw[l].data_ptr()
        ctx.tutti_pool_register(l + 1, k, k + (bb if interleaved else n_blocks * stride), stride, n_blocks)
        if rows:
            ctx.tutti_scales_register_rows(l + 1, scales[l, 0].data_ptr(), scales[l, 1].data_ptr(), n_blocks, rows)
    return ctx, raw, scales, bb, stride


def copied(raw, scales, pairs, bb, stride, n_blocks, interleaved, hk):
    raw, scales = raw.clone(), None if scales is None else scales.clone()
    for a, b in pairs:
        if a == -1 or a == b:
            continue
        for plane in range(2):
            o = (bb if interleaved else n_blocks * stride) * plane
            raw[:, o + b * stride:o + b * stride + bb] = raw[:, o + a * stride:o + a * stride + bb]
        if scales is not None:
            scales[:, :, b, :hk] = scales[:, :, a, :hk]
    return raw, scales


@pytest.mark.parametrize("hk,dim,size,bs,layers,n_blocks,kw", [
    (8, 128, 2, 16, 3, 40, {}), (8, 128, 2, 1, 2, 900, {}), (1, 8, 2, 1, 5, 64, {}), (3, 16, 1, 1, 2, 64, dict(rows=5)), (2, 64, 1, 16, 70, 12, dict(rows=2)),
    (8, 128, 2, 64, 1, 20, dict(interleaved=True)), (5, 24, 2, 7, 2, 30, dict(pad=48)), (2, 128, 4, 300, 1, 9, dict(pad=16, interleaved=True)), (4, 1, 4, 1, 3, 100, {})])
@pytest.mark.parametrize("how_many", [0, 1, 0.5])
def test_copy_blocks(hk, dim, size, bs, layers, n_blocks, kw, how_many):
    rng = np.random.default_rng(n_blocks)
    ctx, raw, scales, bb, stride = pool_of(hk, dim, size, bs, layers, n_blocks, seed=1, **kw)
    try:
        n = how_many if how_many != 0.5 else n_blocks // 2
        order = rng.permutation(n_blocks)
        pairs = [(int(a), int(b)) for a, b in zip(order[:n], order[n:2 * n])]
        pairs = [(-1, -1)] * 3 + [p for q in pairs for p in (q, (-1, 5), (q[1], q[1]) if rng.random() < 0.2 else (-1, -1))]
        status = ints([0])
        want, want_scales = copied(raw, scales, pairs, bb, stride, n_blocks, kw.get("interleaved"), hk)
        ctx.tutti_kv_copy_blocks(1, layers, ints(pairs), status=status)
        assert torch.equal(raw, want) and (scales is None or torch.equal(scales, want_scales)) and int(status) == T.OK
    finally:
        torch.cuda.synchronize()
        ctx.close()


@pytest.mark.parametrize("n_pairs", [0, 1, 2047, 2048, 2049, 5000, 9000])
def test_copy_blocks_in_rounds_and_up_to_a_count(n_pairs):
    n_blocks = 12000
    ctx, raw, scales, bb, stride = pool_of(2, 64, 1, 2, 2, n_blocks, rows=4, seed=2)
    try:
        pairs = np.stack([np.arange(6000), np.arange(6000) + 6000], 1)
        pairs[::7] = -1
        want, want_scales = copied(raw, scales, pairs[:n_pairs].tolist(), bb, stride, n_blocks, False, 2)
        ctx.tutti_kv_copy_blocks(1, 2, ints(pairs), ints([n_pairs]))
        assert torch.equal(raw, want) and torch.equal(scales, want_scales)
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_copy_blocks_outside_the_pool_and_other_layers():
    ctx, raw, _, bb, stride = pool_of(2, 64, 2, 4, 3, 20, seed=3)
    try:
        # layer 3 is registered again with fewer blocks
        ctx.tutti_pool_register(3, raw[2].data_ptr(), raw[2].data_ptr() + 20 * stride, stride, 10)
        want, _ = copied(raw[:2], None, [(1, 15), (2, 3)], bb, stride, 20, False, 2)
        last, _ = copied(raw[2:], None, [(2, 3)], bb, stride, 20, False, 2)
        status = ints([0])
        ctx.tutti_kv_copy_blocks(1, 3, ints([(1, 15), (2, 3), (20, 4), (5, -1), (-2, 6)]), status=status)
        assert torch.equal(raw[:2], want) and torch.equal(raw[2:], last) and int(status) == T.EFAULT
        first = raw.clone()
        ctx.tutti_kv_copy_blocks(2, 1, ints([(7, 8)]))
        first[1:2], _ = copied(first[1:2], None, [(7, 8)], bb, stride, 20, False, 2)
        assert torch.equal(raw, first)
        for a, n in ((0, 1), (0, 4), (3, 2)):                   # layer 0 is not registered, there is no layer 4
            with pytest.raises(T.TuttiError):
                ctx.tutti_kv_copy_blocks(a, n, ints([(7, 8)]))
        ctx.tutti_kv_copy_blocks(1, 0, ints([(7, 9)]))
        assert torch.equal(raw, first)
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_copy_blocks_behind_four_gigabytes():
    n = (5 << 30) // 32768
    ctx = T.Context(T.Geom(1, 8, 128, 2, 16, 16, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
    pool = torch.zeros(2, n, 32768, dtype=torch.uint8, device="cuda:0")
    try:
        ctx.tutti_pool_register(0, pool[0].data_ptr(), pool[1].data_ptr(), 32768, n)
        g = torch.Generator(device="cuda:0").manual_seed(4)
        pool[:, :2] = torch.randint(0, 256, (2, 2, 32768), dtype=torch.uint8, generator=g, device="cuda:0")
        ctx.tutti_kv_copy_blocks(0, 1, ints([(0, n - 1), (1, n // 2)]))
        assert torch.equal(pool[:, n - 1], pool[:, 0]) and torch.equal(pool[:, n // 2], pool[:, 1])
        assert int(pool[:, 2:n // 2].count_nonzero()) == 0 and int(pool[:, n // 2 + 1:n - 1].count_nonzero()) == 0
    finally:
        torch.cuda.synchronize()
        ctx.close()


# ---------------------------------------------------------------------------- long runs of everything

@pytest.mark.parametrize("seed", range(8))
def test_random_runs_over_two_tables(contexts, seed):
    """Forks there and back, extensions, rows freed, windows and compactions over the same counts, in a random order."""
    rng = np.random.default_rng(seed)
    bs = int(rng.choice([1, 4, 16]))
    n_seq, n_blocks = int(rng.integers(1, 40)), int(rng.integers(30, 900))
    cap = 24
    books = [P.Book(np.arange(n_seq + 1) * cap, [-7] * (cap * n_seq), [0] * n_seq, bs) for _ in range(2)]
    refs = [0] * n_blocks
    b = P.Bound(contexts(bs), books, refs)
    pairs = torch.zeros(n_seq, 2, dtype=torch.int32, device=b.dev)
    moves, moved = torch.zeros(20, 2, dtype=torch.int32, device=b.dev), ints([0])
    try:
        for step in range(60):
            k = int(rng.integers(0, 2))
            t, book = b.tables(k), books[k]
            what = rng.choice(["extend", "extend", "extend", "move", "keep", "release", "trim", "compact"])
            if what == "extend":
                n_new = rng.integers(0, rng.choice([2, 2, 3 * bs]), n_seq)
                n_new = np.array([n if book.lens[s] + n <= cap * bs else 0 for s, n in enumerate(n_new)])
                b.pages.tutti_pages_extend(t, ints(n_new), pairs)
                assert pairs.tolist() == [list(p) for p in P.extend(book, refs, n_new)], (step, what)
            elif what in ("move", "keep"):
                # the other table's rows are given up first
                b.pages.tutti_pages_release(b.tables(1 - k))
                P.release(books[1 - k], refs, None)
                parent = rng.integers(-1 if what == "keep" else 0, n_seq, n_seq)
                b.pages.tutti_pages_fork(t, ints(parent), b.tables(1 - k), T.FORK_MOVE if what == "move" else T.FORK_KEEP)
                P.fork(book, parent, books[1 - k], refs, what == "move")
                if what == "move":                              # its rows hold nothing any longer
                    book.lens = [0] * n_seq
                    b.t[k][3].zero_()
            elif what == "release":
                which = rng.random(n_seq) < 0.3
                b.pages.tutti_pages_release(t, torch.from_numpy(which).to(b.dev))
                P.release(book, refs, which)
            elif what == "trim":
                w = int(rng.integers(1, 6 * bs + 2))
                b.pages.tutti_pages_trim(t, T.make_window(w, 2))
                P.trim(book, refs, w, 2)
            else:
                # rows of both tables: one call over arrays of their own would do; here the other table follows the pairs
                other = books[1 - k]
                b.pages.tutti_pages_compact(t, moves, moved)
                place = dict(P.compact(book, refs, len(moves)))
                for s in range(n_seq):
                    a, _, _, h = other.row(s)
                    other.ids[a:a + h] = [place.get(i, i) for i in other.ids[a:a + h]]
                b.t[1 - k][2].copy_(ints(other.ids))
                assert int(moved) == len(place)
            for k in range(2):
                status = books[k].status
                b.same(refs, k)
                assert status <= {T.EAGAIN}
                status.clear()
                b.t[k][4].zero_()
            held = [i for book in books for s in range(n_seq) for i in book.ids[book.row(s)[0]:book.row(s)[0] + book.row(s)[3]] if i >= 0]
            assert np.array_equal(np.bincount(held, minlength=n_blocks), refs)
    finally:
        b.close()
