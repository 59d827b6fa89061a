"""Recorded calls of the learning operators beside calls that are not, and
streams: a potential and a learner on streams of their own."""
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


def test_potential_on_another_stream():
    """Descriptors, heads and forces on three streams, positions made on a fourth: the bits of one stream."""
    import torch
    import synth
    from paper_2608_16329_amd import Learner, Potential, binding
    w = synth.make_workload("fcc-hea6-128", seed=3, n=6)
    dev = torch.device("cuda:0")
    pos0, types = torch.from_numpy(w.pos).to(dev), torch.from_numpy(w.types).to(dev)
    n, H = len(pos0), w.hp.reg_hidden

    def build(side):
        pot = Potential(w.hp, w.weights, stream=torch.cuda.Stream() if side else None)
        L = Learner(stream=torch.cuda.Stream() if side else None)
        pot.build_neighbors(pos0, types, w.box)
        pot.set_fusion(binding.MLIP_FUSION_PARTIAL)
        values = 64 * pot.width + 64 + (H - 1) * 4160 + 65
        tables = torch.from_numpy(w.weights[-6 * values:].reshape(6, -1)).to(dev, torch.float32).contiguous()
        offsets, order = torch.empty(7, dtype=torch.int32, device=dev), torch.empty(n, dtype=torch.int32, device=dev)
        rows, dx = torch.empty((n, pot.width), device=dev), torch.empty((n, pot.width), device=dev)
        energy, forces = torch.empty(n, device=dev), torch.empty_like(pos0)

        def evaluate(pos):
            pot.descriptors(pos, rows)
            L.group(types, offsets, order)
            L.heads(rows, tables, offsets, order, hidden=H, energy=energy, dx=dx)
            pot.forces_from_descriptors(pos, dx, forces)
            return rows.clone(), energy.clone(), forces.clone()
        return evaluate, (pot, L)

    torch.cuda.synchronize()
    one, keep_one = build(False)
    many, keep_many = build(True)
    torch.cuda.synchronize()
    for turn in range(3):
        big = torch.randn((4096, 4096), device=dev)
        shift = (big @ big).double()[0, 0].tanh() * 1e-3        # late on the current stream
        pos = pos0 + shift
        a, b = many(pos), one(pos)
        del pos
        for x, y in zip(a[:2], b[:2]):
            assert torch.equal(x, y)
        # forces are sums of atomic additions: their order is not fixed
        assert float((a[2] - b[2]).abs().max()) <= 1e-9 * max(1.0, float(b[2].abs().max()))
    for p in keep_one + keep_many:
        p.close()
