"""What a fork does to counts that say less than the rows hold, and which arrays it refuses, without a GPU."""
import itertools

import pytest

from paper_2605_03375_b200 import tutti as T
from tests.test_operators_cpu import check_fn
from tests.test_pages_cpu import call, other, tables


def orders(n):
    """Every order in which n writers, each of which takes first and gives back later, may come to one count."""
    return sorted(set(itertools.permutations([w for w in range(n) for _ in range(2)])))


@pytest.mark.parametrize("takes", [(1,), (2,), (1, 1), (2, 2), (16, 1), (3, 5, 2), (1, 1, 1)])
@pytest.mark.parametrize("count", [0, 1, 2, 3, 7, 40])
def test_a_count_does_not_pass_zero_in_any_order(takes, count):
    given_back = check_fn("tutti_fork_given_back_")
    for order in orders(len(takes)):
        now, back = count, {}
        for w in order:
            if w in back:
                now += back[w]
            else:
                now -= takes[w]
                back[w] = given_back(now, -takes[w])
        assert now == max(0, count - sum(takes)), order


def test_who_adds_gives_nothing_back():
    given_back = check_fn("tutti_fork_given_back_")
    assert [given_back(now, 2) for now in (-3, -1, 0, 2)] == [0] * 4 and [given_back(now, -2) for now in (-3, -2, -1, 0)] == [2, 2, 1, 0]


# tables(): blk_start 0x1000 .. 0x100c, block_ids 0x2000 .. 0x2020, len 0x3000 .. 0x3008; other(): the same blk_start, 0x12000, 0x13000
@pytest.mark.parametrize("kw", [
    dict(block_ids=0x201c), dict(block_ids=0x1fe4), dict(block_ids=0x2004), dict(len=0x3004), dict(len=0x2ffc),     # in part
    dict(block_ids=0x3000), dict(block_ids=0x2fe4), dict(len=0x2000), dict(len=0x201c),                             # the one kind over the other
    dict(block_ids=0x1000), dict(block_ids=0xfe4), dict(len=0x1008), dict(len=0xffc),                               # over blk_start
    dict(block_ids=0x5004), dict(len=0x4ffc),                                                                       # over the parents
    dict(len=0x1201c), dict(len=0x11ffc)])                                                                          # over each other
def test_forks_whose_arrays_lie_over_each_other_are_refused(kw):
    for move in (T.FORK_KEEP, T.FORK_MOVE):
        assert call("tutti_fork_check_", tables(), 0x5000, other(**kw), move) == T.EINVAL


@pytest.mark.parametrize("kw", [dict(), dict(block_ids=0x2020), dict(block_ids=0x1fe0), dict(len=0x3008), dict(len=0x2ff8), dict(block_ids=0x100c), dict(len=0x5008),
                                dict(len=0x12020), dict(len=0x11ff8), dict(blk_start=0x1004), dict(blk_start=0x3000), dict(blk_start=0x5000)])
def test_forks_whose_arrays_lie_side_by_side_are_taken(kw):
    assert call("tutti_fork_check_", tables(), 0x5000, other(**kw), T.FORK_MOVE) == T.OK


def test_forks_of_empty_tables_are_taken():
    none = T.Tables(0, 0, 0x1000, None, 0x3000, None)
    assert call("tutti_fork_check_", tables(), None, none, T.FORK_MOVE) == T.EINVAL          # the same lengths' array, as before
    none.len = 0x3004
    assert call("tutti_fork_check_", tables(), None, none, T.FORK_MOVE) == T.OK
    assert call("tutti_fork_check_", none, 0x5000, other(), T.FORK_KEEP) == T.OK
