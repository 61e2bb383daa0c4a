"""Tables of as many rows as there may be."""
import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests import pagecase as P
from tests.test_pages_cpu import call, tables

ROWS = 65536


@pytest.mark.parametrize("n_seq,code", [(16385, T.OK), (ROWS, T.OK), (ROWS + 1, T.EINVAL), (0xffffffff, T.EINVAL)])
def test_how_many_rows_are_taken(n_seq, code):
    assert call("tutti_tables_check_", tables(n_seq=n_seq)) == code and T.PAGES_MAX_SEQ == ROWS


@pytest.mark.gpu
def test_all_operators_on_the_most_rows():
    """Extended, handed on, trimmed, freed and moved together: every row as the statement says, the last ones too."""
    rng = np.random.default_rng(5)
    bs, cap, n_blocks = 4, 4, 3 * ROWS
    ctx = T.Context(T.Geom(1, 2, 64, 2, bs, bs, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
    books = [P.Book(np.arange(ROWS + 1) * cap, [-7] * (cap * ROWS), [0] * ROWS, bs) for _ in range(2)]
    refs = [0] * n_blocks
    b = P.Bound(ctx, books, refs)
    ints = lambda v: torch.tensor(np.asarray(v, np.int32), device=b.dev)  # noqa: E731
    pairs, moved = torch.zeros(ROWS, 2, dtype=torch.int32, device=b.dev), ints([0])
    try:
        for k, most in ((0, 8), (1, 5)):
            n_new = rng.integers(0, most, ROWS)
            n_new[-3:] = 3                                      # the last row holds a block that it shares later on
            b.pages.tutti_pages_extend(b.tables(k), ints(n_new), pairs)
            assert pairs.tolist() == [list(p) for p in P.extend(books[k], refs, n_new)]
            b.same(refs, k)
            if k == 0:
                parent = rng.integers(0, ROWS, ROWS)
                parent[-3:] = ROWS - 1
                b.pages.tutti_pages_fork(b.tables(0), ints(parent), b.tables(1), T.FORK_MOVE)
                P.fork(books[0], parent, books[1], refs, True)
                b.same(refs, 0)
                b.same(refs, 1)
        assert pairs[-3:-1].min() >= 0
        b.pages.tutti_pages_trim(b.tables(1), T.make_window(2, 1))
        P.trim(books[1], refs, 2, 1)
        b.same(refs, 1)
        which = rng.random(ROWS) < 0.5
        which[-2:] = False, True
        b.pages.tutti_pages_release(b.tables(1), torch.from_numpy(which).to(b.dev))
        P.release(books[1], refs, which)
        b.same(refs, 1)
        b.pages.tutti_pages_compact(b.tables(1), pairs, moved)
        moves = P.compact(books[1], refs, ROWS)
        b.same(refs, 1)
        assert int(moved) == len(moves) > 1000 and pairs[:len(moves)].tolist() == [list(m) for m in moves]
        assert not books[0].status and not books[1].status
    finally:
        b.close()
        ctx.close()
