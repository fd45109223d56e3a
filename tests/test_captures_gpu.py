"""Captures are not ended by what earlier tests have left behind."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


def graph(fn):
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


def test_a_graph_is_left_in_a_cycle():
    x = torch.zeros(8, device="cuda")
    cycle = [graph(lambda: x.add_(1.0))]
    cycle.append(cycle)


def test_a_capture_that_makes_many_objects():
    assert not gc.isenabled()
    x = torch.zeros(8, device="cuda")
    made = []

    def fn():
        x.add_(1.0)
        made.extend([i] for i in range(100000))      # (the collector would run, were it not for the fixture)
        x.add_(1.0)

    g = graph(fn)
    g.replay()
    torch.cuda.synchronize()
    assert bool((x == 2).all()) and len(made) == 100000
