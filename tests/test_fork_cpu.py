"""What a fork does to counts that say less than the rows hold, without a GPU."""
import itertools

import pytest

from tests.test_operators_cpu import check_fn


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
