"""Recorded calls of the learning operators beside calls that are not."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_graph_replays_after_a_larger_call():
    """A larger call between the replays takes a workspace of its own; the graph's is not given to anyone."""
    import torch
    from paper_2608_16329_amd import Learner
    m, E, dev = 20000, 7, torch.device("cuda:0")
    ids = (torch.arange(m, device=dev) * 5 % (E + 1)).to(torch.int32)
    many = (torch.arange(3000000, device=dev) * 11 % 250).to(torch.int32)
    offsets, order = torch.zeros(E + 1, dtype=torch.int32, device=dev), torch.zeros(m, dtype=torch.int32, device=dev)
    all_offsets, all_order = torch.zeros(251, dtype=torch.int32, device=dev), torch.zeros(len(many), dtype=torch.int32, device=dev)
    want_all = torch.sort(many.cpu(), stable=True).indices.to(torch.int32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L = Learner(stream=s)
    with torch.cuda.stream(s):
        L.group(ids, offsets, order)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.group(ids, offsets, order)
    held = L.memory_bytes()
    assert held > 0
    for turn in range(3):
        ids.copy_(ids.roll(turn + 1))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            L.group(many, all_offsets, all_order)
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(order.cpu(), torch.sort(ids.cpu(), stable=True).indices.to(torch.int32))
        assert torch.equal(all_order.cpu(), want_all)
        order.zero_(), all_order.zero_()
        if turn == 0:
            more = L.memory_bytes()
            assert more > 2 * held                   # both workspaces are counted
    assert L.memory_bytes() == more
    L.close()
