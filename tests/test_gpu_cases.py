"""The operators' cases through the library, as their file makes the calls: many states of one geometry, side streams
and graphs."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def ops():
    spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.own = True
    return m


def small(ops, op, cache, new=1):
    return ops.case_("small", op, cache, "bf16", 8, 2, 64, 16, 2, (30, 50), (new, new))


@pytest.mark.parametrize("cache", ["16", "8"])
def test_more_states_than_layers(ops, cache):
    c = small(ops, "attend", cache)
    states = [ops.prepare(c, seed) for seed in range(70)]
    first = [ops.run(s)["out"] for s in states]
    for s, want in zip(states, first):
        assert torch.equal(ops.run(s)["out"], want)
    assert not torch.equal(first[0], first[64]) and not torch.equal(first[5], first[69])


@pytest.mark.parametrize("op", ["append", "attend"])
@pytest.mark.parametrize("new", [1, 20])
def test_a_side_stream_and_a_graph(ops, op, new):
    c = small(ops, op, "16", new)
    s = ops.prepare(c, 1)
    key = "q" if op == "append" else "out"
    want = ops.run(s)[key]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(5_000_000)
        s["q"].mul_(2)
        got = ops.run(s)[key]
        s["q"].div_(2)
        again = ops.run(s)[key]
    torch.cuda.synchronize()
    assert torch.equal(again, want) and not torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = ops.run(s)[key]
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
