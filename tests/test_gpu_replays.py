"""The pages' operators in captured graphs: every replay works on inputs that the one before did not have, so that a graph without
one of its calls shows."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2605_03375_b200 import tutti as T
from tests import pagecase as P
from tests.test_gpu_more_cases import ROOT, same, small

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    spec = importlib.util.spec_from_file_location("more_operator_cases", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    yield m
    m.own = False


@pytest.mark.parametrize("op,cache", [("attend", "16"), ("copy", "16"), ("copy", "8"), ("beams", "16"), ("beams", "8"), ("slide", "16"), ("compact", "16"), ("compact", "8")])
def test_a_replay_works_on_what_lies_there_now(ops, op, cache):
    case = small(ops, op, cache)

    def wanted(seed):
        ops.own = False
        out = ops.run(ops.prepare(case, seed))
        ops.own = True
        return {k: None if x is None else x.clone() for k, x in out.items()}

    wants = [wanted(seed) for seed in range(4)]
    ops.own = True
    s = ops.prepare(case, 0)
    ops.run(s)                                                  # registers its layers
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = ops.run(s)
    tensors = [k for k, x in s.items() if isinstance(x, torch.Tensor)]
    for seed in (1, 2, 3, 0):
        fresh = ops.prepare(case, seed)
        for k in tensors:
            s[k].copy_(fresh[k])
        for x in got.values():                                  # results that are not the state's own
            if x is not None and x.is_floating_point():
                x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        same(got, wants[seed], 2.0 ** -11)
        assert any(x is not None and not torch.equal(x, wants[seed - 1][k]) for k, x in wants[seed].items())


@pytest.mark.parametrize("bs", [1, 4, 16])
def test_tables_that_change_between_replays(bs):
    """Handed on, grown, freed in part, trimmed, moved together, and handed back: one graph, with other parents, numbers of tokens
    and rows to free each time, against the statement row by row; eager calls in between change the tables, too."""
    rng = np.random.default_rng(bs)
    n_seq, cap, n_blocks, max_pairs = 23, 12, 23 * 14, 40
    ctx = T.Context(T.Geom(1, 2, 64, 2, bs, bs, 1, T.LAYOUT_LAYER_MAJOR, 1), 0)
    books = [P.Book(np.arange(n_seq + 1) * cap, [-7] * (cap * n_seq), [0] * n_seq, bs) for _ in range(2)]
    refs = [0] * n_blocks
    b = P.Bound(ctx, books, refs)
    ints = lambda v: torch.tensor(np.asarray(v, np.int32), device=b.dev)  # noqa: E731
    parent, back, n_new = (ints([0] * n_seq) for _ in range(3))
    which = torch.zeros(n_seq, dtype=torch.bool, device=b.dev)
    pairs, moves, moved = (torch.zeros(n, 2, dtype=torch.int32, device=b.dev) for n in (n_seq, max_pairs, 1))
    window = (3 * bs, 1)
    try:
        def grow(k, most):
            n = rng.integers(0, most + 1, n_seq)
            return np.array([x if books[k].lens[s] + x <= cap * bs else 0 for s, x in enumerate(n)])

        n = grow(0, 5 * bs)
        b.pages.tutti_pages_extend(b.tables(0), ints(n), pairs)
        P.extend(books[0], refs, n)
        b.same(refs, 0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st = torch.cuda.current_stream()
            b.pages.tutti_pages_fork(b.tables(0), parent, b.tables(1), T.FORK_MOVE, st)
            b.pages.tutti_pages_extend(b.tables(1), n_new, pairs, st)
            b.pages.tutti_pages_release(b.tables(1), which, st)
            b.pages.tutti_pages_trim(b.tables(1), T.make_window(*window), st)
            b.pages.tutti_pages_compact(b.tables(1), moves, moved, st)
            b.pages.tutti_pages_fork(b.tables(1), back, b.tables(0), T.FORK_MOVE, st)
        b.same(refs, 0)                                         # nothing has run yet
        for i in range(25):
            p, q, w = rng.integers(-1 if i % 5 == 4 else 0, n_seq, n_seq), rng.permutation(n_seq), rng.random(n_seq) < 0.2
            for t, v in ((parent, p), (back, q)):
                t.copy_(ints(v))
            which.copy_(torch.from_numpy(w))
            for t in (pairs, moves, moved):
                t.fill_(55)
            P.fork(books[0], p, books[1], refs, True)
            n = grow(1, 2 * bs)
            n_new.copy_(ints(n))
            g.replay()
            want = P.extend(books[1], refs, n)
            P.release(books[1], refs, w)
            P.trim(books[1], refs, *window)
            moving = P.compact(books[1], refs, max_pairs)
            P.fork(books[1], q, books[0], refs, True)
            b.same(refs, 0)
            b.same(refs, 1)
            assert pairs.tolist() == [list(x) for x in want], i
            assert int(moved[0, 0]) == len(moving) and moves[:len(moving)].tolist() == [list(m) for m in moving] and (moves[len(moving):] == -1).all(), i
            if i % 4 == 1:                                      # an eager step in between
                n = grow(0, 4 * bs)
                b.pages.tutti_pages_extend(b.tables(0), ints(n), pairs)
                assert pairs.tolist() == [list(x) for x in P.extend(books[0], refs, n)]
                b.same(refs, 0)
        assert not books[0].status and not books[1].status
    finally:
        b.close()
        ctx.close()
