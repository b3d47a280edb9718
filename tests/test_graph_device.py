"""Attention over a graph of another device than the current one is refused
before anything is launched (CPU only: the devices are stand-ins)."""
import pytest
import torch

from paper_1909_01315_amd import gnnk


class Elsewhere:
    """a graph's workspace on cuda:1"""
    is_cuda = True

    def get_device(self):
        return 1


@pytest.fixture
def graph(monkeypatch):
    monkeypatch.setattr(gnnk, "_device", lambda: 0)
    g = object.__new__(gnnk.Graph)
    g._h, g._keep, g.num_src, g.num_dst, g.num_edges = None, [Elsewhere()], 3, 3, 4
    return g


def test_forward_and_backward(graph):
    t = torch.ones(3, 2, 8)
    with pytest.raises(ValueError, match="cuda:1"):
        gnnk.dot_aggregate(graph, t, t, t)
    with pytest.raises(ValueError, match="cuda:1"):
        gnnk.dot_aggregate_backward(graph, t, t, t, t, torch.ones(3, 2, 2), t)


def test_the_current_device_passes_on(graph):
    graph._keep[0].get_device = lambda: 0
    with pytest.raises(ValueError, match="must be on the GPU"):  # (the tensors are the host's)
        gnnk.dot_aggregate(graph, *(torch.ones(3, 2, 8),) * 3)
