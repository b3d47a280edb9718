"""Scratch buffers that the binding replaces: one that no captured call has
used goes back to torch's allocator, one that a captured call holds the
address of stays with the handle, and a buffer that is large enough already
is not replaced."""
import pytest
import torch

from paper_1909_01315_amd import gnnk, synth

pytestmark = pytest.mark.gpu

MB = 1 << 20


@pytest.fixture
def graph():
    gnnk.set_option("seg_edges", 64)  # long rows need partial results
    sg = synth.graph_c2()
    g = gnnk.Graph.from_coo(torch.from_numpy(sg.src).cuda(), torch.from_numpy(sg.dst).cuda(), sg.n_src, sg.n_dst)
    assert g.info()["segments_in"] > 0
    yield g
    torch.cuda.synchronize()
    g.destroy()
    gnnk.set_option("seg_edges", 0)


def held(g):
    """bytes that the handle's buffers keep from the allocator"""
    torch.cuda.synchronize()
    with_g = torch.cuda.memory_allocated()
    lent, replaced = g._lent, getattr(g, "_replaced", None)
    total = sum(t.numel() for t in lent.values()) + sum(t.numel() for t in replaced or ())
    assert with_g >= total
    return total


def test_growth_without_capture_keeps_one_buffer(graph):
    s = torch.cuda.Stream()
    for size in (64 * MB, 66 * MB, 90 * MB, 200 * MB):
        before = held(graph)
        graph.lend_scratch(size, s)
        assert size <= held(graph) <= max(size, before * 5 // 4), "one buffer, at most a quarter larger than asked for"


def test_growth_by_calls_keeps_one_buffer(graph):
    n = graph.num_src
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for cols in (64, 128, 512):
            gnnk.gspmm(graph, "copy_lhs", "sum", torch.ones(n, 1, cols, device="cuda"))
    s.synchronize()
    assert len(graph._lent) == 1 and held(graph) == graph._lent[s.cuda_stream].numel()


def test_a_buffer_that_is_large_enough_stays(graph):
    s = torch.cuda.Stream()
    graph.lend_scratch(8 * MB, s)
    first = graph._lent[s.cuda_stream]
    for size in (8 * MB, MB, 1, 8 * MB):
        graph.lend_scratch(size, s)
        assert graph._lent[s.cuda_stream] is first
    assert held(graph) == first.numel()


def test_captured_buffers_stay_and_others_go(graph):
    """Two streams: the buffer that a capture used stays when it is outgrown,
    also where it was handed over again in between, the other stream's goes."""
    n = graph.num_src
    small, large = torch.ones(n, 1, 32, device="cuda"), torch.ones(n, 1, 512, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            want = gnnk.gspmm(graph, "copy_lhs", "sum", small)
    torch.cuda.synchronize()
    first = [graph._lent[s.cuda_stream].data_ptr() for s in streams]
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured, stream=streams[0]):
        got = gnnk.gspmm(graph, "copy_lhs", "sum", small)
    graph.lend_scratch(1, streams[0])  # (large enough: the same buffer)
    for s in streams:
        with torch.cuda.stream(s):
            gnnk.gspmm(graph, "copy_lhs", "sum", large)
    torch.cuda.synchronize()
    assert [graph._lent[s.cuda_stream].data_ptr() for s in streams] != first
    assert [t.data_ptr() for t in graph._replaced] == first[:1]
    for _ in range(3):
        got.fill_(float("nan"))
        captured.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        _ = (small * 2).sum().item()
