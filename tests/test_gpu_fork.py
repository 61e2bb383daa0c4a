"""Forks of tables whose numbers contradict each other: ids that are no block's, counts that say less than the rows hold."""
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests import pagecase as P

pytestmark = pytest.mark.gpu
BS = 4


@pytest.fixture(scope="module")
def ctx():
    c = T.Context(T.Geom(1, 2, 64, 2, BS, BS, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
    yield c
    torch.cuda.synchronize()
    c.close()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("move,parent,reported", [
    (T.FORK_MOVE, [0, 1], True), (T.FORK_MOVE, [1, 0], True),      # a child a row: no count changes
    (T.FORK_MOVE, [0, 0], True),                                   # what one row gains its neighbour loses
    (T.FORK_MOVE, [-1, -1], True), (T.FORK_KEEP, [0, -1], True), (T.FORK_KEEP, [0, 1], True),
    (T.FORK_KEEP, [-1, -1], False)])                               # kept rows that nobody takes are not looked at
def test_ids_outside_the_pool_are_reported_whatever_becomes_of_the_counts(ctx, move, parent, reported):
    frm = P.Book([0, 3, 6], [0, 99, 1, 2, 99, 3], [12, 12], BS)
    to = P.Book([0, 3, 6], [-9] * 6, [0] * 2, BS)
    refs = [1] * 4 + [0] * 4
    b = P.Bound(ctx, [frm, to], refs)
    try:
        b.pages.tutti_pages_fork(b.tables(0), ints(parent), b.tables(1), move)
        P.fork(frm, parent, to, refs, move)
        assert frm.status == ({T.EFAULT} if reported else set()) and not to.status
        b.same(refs, 0)
        b.same(refs, 1)
    finally:
        b.close()


def test_counts_do_not_pass_zero(ctx):
    """More rows hold a block than its count says, in groups that different CTAs see to."""
    n_seq, n_blocks = 90, 40
    for seed in range(6):
        frm = P.Book([n_blocks * s for s in range(n_seq + 1)], list(range(n_blocks)) * n_seq, [n_blocks * BS - seed] * n_seq, BS)
        to = P.Book([0, n_blocks], [-9] * n_blocks, [5], BS)
        refs = [(7 * i + seed) % 120 for i in range(n_blocks)]
        b = P.Bound(ctx, [frm, to], refs)
        try:
            b.pages.tutti_pages_fork(b.tables(0), ints([-1]), b.tables(1), T.FORK_MOVE)
            P.fork(frm, [-1], to, refs, True)
            held = frm.row(0)[3]
            assert frm.status == {T.EINVAL} and refs == [max(0, (7 * i + seed) % 120 - n_seq * (i < held)) for i in range(n_blocks)]
            b.same(refs, 0)
            b.same(refs, 1)
        finally:
            b.close()
