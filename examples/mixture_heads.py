"""Learn energy heads that are chosen by an atom's environment, and run
molecular dynamics with them.

A potential's heads are tables, one per species (Section 3.2 of the paper).
Here each species has a choice of heads, one of its own and some that all
species share: a router, a linear map of the descriptor, gives each atom the
weights (gates) of the heads its species may use.  The encoder stays as it is;
the heads and the router are fitted to reference energies per atom (those of
another potential, which stands in for first-principles data):

  descriptors -> route -> group -> heads -> squared error and balance loss
              <- route_backward <- heads' gradients             -> AdamW

and the fitted heads then give dE/dG to the force kernel in a velocity-Verlet
run.  All heads a species may use are mixed, so that energies are smooth.

    python examples/mixture_heads.py [--cells 8] [--steps 200] [--bits 8]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth
from paper_2608_16329_amd import AdamW, Learner, Potential, binding

ACC_PER_FORCE_MASS = 9.648533212e-3   # (eV/A)/amu -> A/fs^2
WIDTH = 64                            # hidden width of a head


def head_segments(width: int, hidden: int):
    """(values, inputs a value is drawn over, whether it is a matrix) of a head table, in its order."""
    return [(WIDTH * width, width, True), (WIDTH, width, False)] \
        + [(WIDTH * WIDTH, WIDTH, True), (WIDTH, WIDTH, False)] * (hidden - 1) \
        + [(WIDTH, WIDTH, True), (1, WIDTH, False)]


class MixtureHeads:
    """A router and heads over descriptors: energies, gradients, and one step of learning."""

    def __init__(self, n_species: int, shared: int, width: int, hidden: int, scale: float = 1.0, bits: int = 32, seed: int = 0):
        dev = torch.device("cuda")
        g = torch.Generator(device=dev).manual_seed(seed)
        self.learner = Learner()
        self.width, self.hidden, self.top_k = width, hidden, 1 + shared
        self.n_heads = n_species + shared
        # species s may use head s and the shared ones
        self.allowed = torch.cat([torch.eye(n_species), torch.ones(n_species, shared)], 1).to(dev, torch.uint8).contiguous()
        segments = head_segments(width, hidden)
        spread = torch.cat([torch.full((m,), fan ** -0.5) for m, fan, _ in segments]).to(dev)
        spread[:WIDTH * width] *= scale
        self.weights = torch.randn((self.n_heads, len(spread)), generator=g, device=dev) * spread
        self.router = 0.01 * scale * torch.randn((self.n_heads, width), generator=g, device=dev)
        self.dweights, self.drouter = torch.zeros_like(self.weights), torch.zeros_like(self.router)
        # one tensor per matrix and vector of every head, and the router
        params, grads, decay = [], [], []
        for e in range(self.n_heads):
            params += self.weights[e].split([m for m, _, _ in segments])
            grads += self.dweights[e].split([m for m, _, _ in segments])
            decay += [matrix for _, _, matrix in segments]
        self.opt = AdamW(params + [self.router], grads + [self.drouter], bits=bits, decay=decay + [False])
        self.steps = 0

    def _buffers(self, n: int) -> None:
        if getattr(self, "n", None) == n:
            return
        self.n = n
        f32, i32 = dict(device="cuda", dtype=torch.float32), dict(device="cuda", dtype=torch.int32)
        self.experts, self.gates = torch.empty((n, self.top_k), **i32), torch.empty((n, self.top_k), **f32)
        self.counts, self.loss = torch.empty(self.n_heads + 1, **i32), torch.empty(1, **f32)
        self.offsets, self.order = torch.empty(self.n_heads + 1, **i32), torch.empty(n * self.top_k, **i32)
        self.energy, self.dgates = torch.empty(n, **f32), torch.empty((n, self.top_k), **f32)
        self.dx, self.dlogits = torch.empty((n, self.width), **f32), torch.empty((n, self.n_heads), **f32)

    def _route(self, x, types) -> None:
        self._buffers(len(x))
        self.logits = x @ self.router.t()
        self.learner.route(self.logits, self.experts, self.gates, self.counts, self.loss, kinds=types, allowed=self.allowed)
        self.learner.group(self.experts, self.offsets, self.order)

    def _heads(self, x, **outputs) -> None:
        self.learner.heads(x, self.weights, self.offsets, self.order, hidden=self.hidden, top_k=self.top_k,
                           gates=self.gates, energy=self.energy, **outputs)

    def _route_backward(self, types, dloss=None) -> None:
        self.learner.route_backward(self.logits, self.experts, self.counts, self.dlogits, dgates=self.dgates, dloss=dloss,
                                    kinds=types, allowed=self.allowed)

    def energies(self, x, types):
        self._route(x, types)
        self._heads(x)
        return self.energy

    def energies_and_gradient(self, x, types):
        """Energies and dE/dx: through the heads, and through the gates."""
        self._route(x, types)
        self._heads(x, dx=self.dx, dgates=self.dgates)
        self._route_backward(types)
        self.dx.addmm_(self.dlogits, self.router)
        return self.energy, self.dx

    def learn(self, x, types, target, lr: float, balance: float = 1e-3):
        """One step on mean squared error + balance x balance loss; the squared error before it."""
        energy = self.energies(x, types)
        miss = energy - target
        error = miss.square().mean()
        self._heads(x, denergy=(2.0 / len(x)) * miss, dweights=self.dweights, dgates=self.dgates)
        self._route_backward(types, torch.full((1,), balance, device="cuda"))
        torch.mm(self.dlogits.t(), x, out=self.drouter)
        self.steps += 1
        self.opt.step(self.steps, lr=lr, beta2=0.99, weight_decay=1e-4, seed=self.steps)
        return error


class MixturePotential:
    """A potential's encoder with mixture heads: energies and forces of a structure."""

    def __init__(self, pot: Potential, heads: MixtureHeads, types):
        self.pot, self.heads, self.types = pot, heads, types
        self.rows = torch.empty((len(types), pot.width), device="cuda")

    def energy_forces(self, pos, forces):
        self.pot.descriptors(pos, self.rows)
        energy, gradient = self.heads.energies_and_gradient(self.rows, self.types)
        self.pot.forces_from_descriptors(pos, gradient, forces)
        return energy


def fit(cells: int = 8, steps: int = 200, bits: int = 32, shared: int = 2, seed: int = 0, say=print):
    """Fit on a six-component FCC crystal of 4 cells^3 atoms; the potential, its structure and errors on the way."""
    w = synth.make_workload("fcc-hea6-128", seed=seed, n=cells, energy_scale=synth.PHYSICAL_ENERGY_SCALE)
    teacher = Potential(w.hp, synth.random_weights(w.hp, seed + 50, energy_scale=synth.PHYSICAL_ENERGY_SCALE))
    pot = Potential(w.hp, w.weights)
    pos, types = torch.from_numpy(w.pos).cuda(), torch.from_numpy(w.types).cuda()
    forces = torch.empty_like(pos)
    reference = torch.empty(len(pos), dtype=torch.float64, device="cuda")
    for p in (teacher, pot):
        p.build_neighbors(pos, types, w.box)
    teacher.compute(pos, forces, reference)
    pot.set_fusion(binding.MLIP_FUSION_PARTIAL)
    rows = torch.empty((len(pos), pot.width), device="cuda")
    pot.descriptors(pos, rows)
    target = (reference - reference.mean()).float()
    target /= target.std()
    heads = MixtureHeads(w.hp.n_species, shared, pot.width, w.hp.reg_hidden, scale=1.0 / float(rows.square().mean().sqrt()),
                         bits=bits, seed=seed)
    errors = []
    for step in range(steps):
        lr = 2e-3 * min(1.0, (step + 1) / 20) * 0.5 * (1 + math.cos(math.pi * step / steps))
        errors.append(heads.learn(rows, types, target, lr))
        if step % 50 == 0 or step == steps - 1:
            say(f"step {step}: root mean square error {math.sqrt(float(errors[-1])):.4f}, balance loss "
                f"{float(heads.loss):.4f}, atoms per head {heads.counts[:-1].tolist()}")
    return MixturePotential(pot, heads, types), w, pos, [float(e) for e in errors]


def run(potential: MixturePotential, w, pos, steps: int = 50, dt: float = 1.0, energy_unit: float = 0.02, say=print):
    """Velocity Verlet with the fitted heads (energies in units of energy_unit eV); total energies."""
    masses = torch.from_numpy(w.masses).cuda()[potential.types.long()][:, None]
    vel = torch.from_numpy(w.vel).cuda()
    pos, forces = pos.clone(), torch.empty_like(pos)
    potential.pot.build_neighbors(pos, potential.types, w.box)
    energy = potential.energy_forces(pos, forces)
    totals = []
    for step in range(steps):
        vel += (0.5 * dt * ACC_PER_FORCE_MASS * energy_unit) * forces / masses
        pos += dt * vel
        if step % 10 == 9:
            potential.pot.build_neighbors(pos, potential.types, w.box)
        energy = potential.energy_forces(pos, forces)
        vel += (0.5 * dt * ACC_PER_FORCE_MASS * energy_unit) * forces / masses
        kinetic = 0.5 * (masses * vel.square()).sum() / ACC_PER_FORCE_MASS
        totals.append(float(energy.double().sum() * energy_unit + kinetic))
        if step % 10 == 0:
            say(f"MD step {step}: potential {float(energy.double().sum() * energy_unit):.4f} eV, kinetic "
                f"{float(kinetic):.4f} eV, total {totals[-1]:.4f} eV")
    return totals


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cells", type=int, default=8, help="edge of the crystal in cells of 4 atoms")
    ap.add_argument("--steps", type=int, default=200, help="learning steps")
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32), help="bits of the optimiser's moments")
    ap.add_argument("--md-steps", type=int, default=50)
    args = ap.parse_args()
    potential, workload, positions, _ = fit(args.cells, args.steps, args.bits)
    run(potential, workload, positions, args.md_steps)
