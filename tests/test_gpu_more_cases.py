"""The cases of the pages and of attention under a window as their file makes the calls: against their plain forms, with many
states of one geometry, on a side stream and in a graph."""
import importlib.util
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ops():
    spec = importlib.util.spec_from_file_location("more_operator_cases", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    yield m
    m.own = False


def small(ops, op, cache="16"):
    return {
        "attend": lambda: ops.attend_("x", cache, "fp16", 8, 2, 64, 16, 3, (60, 90), (1, 5), 32, 4),
        "copy": lambda: ops.pages_("x", "copy", cache, 2, 64, 16, 3, blocks=30, pairs=9),
        "beams": lambda: ops.pages_("x", "beams", cache, 2, 64, 16, 3, requests=3, beams=4, prompt_lo=20, prompt_hi=90, apart=21),
        "slide": lambda: ops.pages_("x", "slide", "16", 2, 64, 16, 0, seqs=9, len_lo=10, len_hi=300, window=64, sinks=4, new=3, blocks=300),
        "compact": lambda: ops.pages_("x", "compact", cache, 2, 64, 16, 3, seqs=9, len_lo=10, len_hi=90, share=32, gone=0.4)}[op]()


def both(ops, case, seed):
    ops.own = False
    want = ops.run(ops.prepare(case, seed))
    ops.own = True
    return ops.run(ops.prepare(case, seed)), want


def same(got, want, half):
    for k, w in want.items():
        if w is None:
            assert got[k] is None
        elif w.is_floating_point():
            # each is off from the formula by a rounding of the result and one of the probabilities, lse by 32-bit sums
            d, size = (got[k].double() - w.double()).abs().max(), w.double().abs().max()
            assert d <= 4 * half * size if w.dtype != torch.float32 else d <= 2.0 ** -18 * (1 + size), k
        else:
            assert torch.equal(got[k], w), k


@pytest.mark.parametrize("op,cache", [("attend", "16"), ("attend", "8"), ("copy", "16"), ("copy", "8"), ("beams", "16"), ("beams", "8"), ("slide", "16"),
                                      ("compact", "16"), ("compact", "8")])
def test_small_cases_and_more_states_than_layers(ops, op, cache):
    for seed in range(50):
        got, want = both(ops, small(ops, op, cache), seed)
        same(got, want, 2.0 ** -11)


@pytest.mark.parametrize("seed", range(14))
def test_drawn_cases(ops, seed):
    case = ops.draw(random.Random(1000 + seed))
    if ops.work(case)["flops"] > 5e10 or ops.work(case)["bytes"] > 5e8:
        case = small(ops, case["op"], case["cache"])
    got, want = both(ops, case, seed)
    same(got, want, 2.0 ** -8 if case.get("dtype") == "bf16" else 2.0 ** -11)


@pytest.mark.parametrize("op", ["attend", "copy", "beams", "slide", "compact"])
def test_a_side_stream_and_a_graph(ops, op):
    case = small(ops, op)
    want = both(ops, case, 3)[1]
    s = ops.prepare(case, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(5_000_000)
        got = ops.run(s)
    torch.cuda.synchronize()
    same(got, want, 2.0 ** -11)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = ops.run(s)
    for x in got.values():
        if x is not None and x.is_floating_point():
            x.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    same(got, want, 2.0 ** -11)
