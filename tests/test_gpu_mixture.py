"""Descriptors and forces outside the fused evaluation, and the operators run
together as examples/mixture_heads.py does."""
import os
import sys

import numpy as np
import pytest

import synth
from tests.gpu_helpers import log, to_dev

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def values_of(D, H):
    return 64 * D + 64 + (H - 1) * (64 * 64 + 64) + 65


@pytest.mark.parametrize("precision", [64, 32])
@pytest.mark.parametrize("lmax", [3, 1])
def test_species_heads_give_the_potentials_forces(precision, lmax):
    """The potential's own heads through descriptors, heads and forces from
    descriptors: energies and forces of mlip_compute.  The descriptors and their
    gradient pass through float32 (2^-24 relative each, amplified by the head's
    four layers and by sums of some 50 pairs): 2e-5 of the largest value."""
    import torch
    from paper_2608_16329_amd import Learner, Potential, binding
    w = synth.make_workload("fcc-hea6-128", seed=5, n=5, hp_overrides={"precision": precision, "lmax": lmax})
    pot = Potential(w.hp, w.weights)
    pos, types = to_dev(w.pos), to_dev(w.types)
    n = len(pos)
    pot.build_neighbors(pos, types, w.box)
    F0, V0 = torch.empty_like(pos), torch.empty((n, 9), dtype=torch.float64, device="cuda")
    E0 = torch.empty(n, dtype=torch.float64, device="cuda")
    pot.compute(pos, F0, E0, V0)
    pot.set_fusion(binding.MLIP_FUSION_PARTIAL)
    D, H = pot.width, w.hp.reg_hidden
    rows = torch.full((n, D), float("nan"), device="cuda")
    pot.descriptors(pos, rows)
    tables = torch.from_numpy(w.weights[-6 * values_of(D, H):].reshape(6, -1)).to("cuda", torch.float32).contiguous()
    L = Learner()
    offsets, order = torch.empty(7, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    L.group(types, offsets, order)
    E, dx = torch.empty(n, device="cuda"), torch.empty((n, D), device="cuda")
    L.heads(rows, tables, offsets, order, hidden=H, energy=E, dx=dx)
    F, V = torch.full_like(F0, float("nan")), torch.full_like(V0, float("nan"))
    pot.forces_from_descriptors(pos, dx, F, V)
    torch.cuda.synchronize()
    tol = 2e-5 if precision == 64 else 1e-4       # the float32 network's own bar is 1e-4
    for name, a, b in (("energy", E.double(), E0), ("forces", F, F0), ("virial", V, V0)):
        err = float((a - b).abs().max()) / float(b.abs().max())
        log(f"[mixture] precision {precision} lmax {lmax} {name}: {err:.1e}")
        assert err <= tol, (name, err)
    # and an evaluation of its own afterwards is what it was
    F1 = torch.empty_like(F0)
    pot.compute(pos, F1, E0, V0)
    assert float((F1 - F0).abs().max()) <= (1e-9 if precision == 64 else 1e-4 * float(F0.abs().max()))
    pot.close()


def test_descriptors_are_refused_in_other_configurations():
    import torch
    from paper_2608_16329_amd import MlipError, Potential, binding
    w = synth.make_workload("fcc-binary-4", seed=1)
    pot = Potential(w.hp, w.weights)
    pos, types = to_dev(w.pos), to_dev(w.types)
    rows = torch.empty((len(pos), 128), device="cuda")
    with pytest.raises(MlipError, match="STATE"):
        binding.mlip_descriptors(pot.ctx, pos.data_ptr(), rows.data_ptr())
    pot.build_neighbors(pos, types, w.box)
    with pytest.raises(MlipError, match="STATE.*PARTIAL"):
        pot.descriptors(pos, rows)
    with pytest.raises(MlipError, match="STATE.*PARTIAL"):
        pot.forces_from_descriptors(pos, rows, torch.empty_like(pos))
    pot.set_fusion(binding.MLIP_FUSION_PARTIAL)
    with pytest.raises(AssertionError, match="rows"):
        pot.descriptors(pos, rows[:, :64].contiguous())
    with pytest.raises(MlipError, match="NULL"):
        binding.mlip_forces_from_descriptors(pot.ctx, pos.data_ptr(), None, pos.data_ptr())
    pot.descriptors(pos, rows)
    pot.close()


def test_mixture_learns_and_runs():
    """A short fit lowers the error, forces are the energies' gradient, and a run
    with them keeps its total energy."""
    import torch
    import mixture_heads
    for bits in (32, 8):
        potential, w, pos, errors = mixture_heads.fit(cells=5, steps=120, bits=bits, say=log)
        assert errors[-1] < 0.25 * errors[0], (errors[0], errors[-1])
    # forces against central differences of the energy along random directions;
    # energies are float32 sums, 500 atoms of O(1): steps of 2e-3 A leave about
    # 1e-3 of the difference
    forces = torch.empty_like(pos)
    potential.energy_forces(pos, forces)
    g = torch.Generator(device="cuda").manual_seed(1)
    scratch = torch.empty_like(pos)
    for _ in range(3):
        d = torch.randn(pos.shape, generator=g, device="cuda", dtype=torch.float64)
        up = float(potential.energy_forces(pos + 2e-3 * d, scratch).double().sum())
        down = float(potential.energy_forces(pos - 2e-3 * d, scratch).double().sum())
        slope = (up - down) / 4e-3
        along = -float((forces * d).sum())
        log(f"[mixture] slope {slope:.5f} against {along:.5f}")
        assert abs(slope - along) <= 2e-2 * float(forces.norm())
    totals = mixture_heads.run(potential, w, pos, steps=30, say=log)
    assert max(totals) - min(totals) < 0.02 * np.mean(np.abs(totals))


def test_captured_training_step_replays():
    """Routing, grouping, heads, their gradients and AdamW recorded in a graph: every replay, with the program's own
    work between, gives the bits of the calls one by one."""
    import torch
    from paper_2608_16329_amd import AdamW, Learner
    n, D, H, E, K = 3000, 64, 3, 5, 2
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(2)
    x, logits = (torch.randn(s, generator=g, device=dev) for s in ((n, D), (n, E)))
    w0 = torch.randn((E, values_of(D, H)), generator=g, device=dev) * 0.1
    up = torch.randn(n, generator=g, device=dev)
    one = torch.ones(1, device=dev)

    def build(stream):
        L = Learner(stream=stream)
        t = dict(w=w0.clone(), dw=torch.zeros_like(w0), ids=torch.empty((n, K), dtype=torch.int32, device=dev),
                 gates=torch.empty((n, K), device=dev), counts=torch.empty(E + 1, dtype=torch.int32, device=dev),
                 loss=torch.empty(1, device=dev), offsets=torch.empty(E + 1, dtype=torch.int32, device=dev),
                 order=torch.empty(n * K, dtype=torch.int32, device=dev), energy=torch.empty(n, device=dev),
                 dx=torch.empty((n, D), device=dev), dgates=torch.empty((n, K), device=dev), dz=torch.empty((n, E), device=dev))
        opt = AdamW([t["w"]], [t["dw"]], bits=8, stream=stream)

        def step():
            L.route(logits, t["ids"], t["gates"], t["counts"], t["loss"])
            L.group(t["ids"], t["offsets"], t["order"])
            L.heads(x, t["w"], t["offsets"], t["order"], hidden=H, top_k=K, gates=t["gates"], denergy=up, energy=t["energy"],
                    dx=t["dx"], dweights=t["dw"], dgates=t["dgates"])
            L.route_backward(logits, t["ids"], t["counts"], t["dz"], dgates=t["dgates"], dloss=one)
            opt.step(1, lr=1e-3, seed=7)
        return t, opt, step, L

    eager, opt_e, step_e, keep_e = build(torch.cuda.current_stream())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    t, opt, step, keep = build(s)
    with torch.cuda.stream(s):
        step()                                       # the workspace is laid out here
        t["w"].copy_(w0)
        for m in (opt.m, opt.v, opt.m_exp, opt.v_exp):
            m.zero_()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for _ in range(4):
        step_e()
        graph.replay()
        torch.cuda.synchronize()
        for k in t:
            assert torch.equal(t[k], eager[k]), k
        assert torch.equal(opt.m, opt_e.m) and torch.equal(opt.v, opt_e.v)
        up.mul_(0.5).add_(0.1)                       # other inputs the next time
        x.add_(0.01)
        torch.cuda.synchronize()
    keep.close(), keep_e.close(), opt.close(), opt_e.close()


def test_a_recorded_call_does_not_enlarge_the_workspace():
    """A first call of its size is refused while its stream is recorded; what else is recorded stays, and the call
    works once it was made before."""
    import torch
    from paper_2608_16329_amd import Learner, MlipError
    m, E = 20000, 7
    ids = (torch.arange(m, device="cuda:0") * 5 % (E + 1)).to(torch.int32)
    offsets, order = torch.zeros(E + 1, dtype=torch.int32, device="cuda:0"), torch.zeros(m, dtype=torch.int32, device="cuda:0")
    few = torch.zeros(100, dtype=torch.int32, device="cuda:0")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L = Learner(stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.group(ids[:100], offsets, few)             # needs no workspace
        with pytest.raises(MlipError, match="recorded"):
            L.group(ids, offsets, order)
    graph.replay()
    torch.cuda.synchronize()
    assert L.memory_bytes() == 0 and few.long().bincount().tolist() == [1] * 100 and not bool(order.any())
    with torch.cuda.stream(s):
        L.group(ids, offsets, order)
    torch.cuda.synchronize()
    want = torch.sort(ids.cpu(), stable=True).indices.to(torch.int32)
    assert torch.equal(order.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.group(ids, offsets, order)
    for turn in range(3):
        ids.copy_(ids.roll(turn + 1))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(order.cpu(), torch.sort(ids.cpu(), stable=True).indices.to(torch.int32))
    L.close()
