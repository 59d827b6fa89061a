"""Energy heads over rows grouped by head, with their gradients, against the
definition in 64 bits (autograd over float64 PyTorch operations).

Tolerances: every product is a float32 sum of at most 1024 (inputs), 64 (layers)
or the head's rows (weight gradients) terms, so relative to the largest value of
an output the error is a small multiple of 2^-24 sqrt(terms) per layer; over 9
layers and 10^4 rows that stays below 2e-5 of the largest value (1e-4 of it is
refused outright by a wrong term of any size that matters).  bf16 dx is rounded
once more, 2^-8 relative."""
import numpy as np
import pytest

import synth
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu


def values_of(D, H):
    return 64 * D + 64 + (H - 1) * (64 * 64 + 64) + 65


def inputs(n, D, H, E, K, dtype, spare, seed, absent=0.1, skew=False):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dev = torch.device("cuda:0")
    x = torch.full((n, D + spare), float("nan"), dtype=getattr(torch, dtype), device=dev)[:, :D]
    x.copy_(torch.randn((n, D), generator=g, device=dev).abs() * 0.7)
    scale = torch.cat([torch.full((m,), f ** -0.5) for m, f in [(64 * D, D), (64, D)] + [(4096, 64), (64, 64)] * (H - 1) + [(65, 64)]])
    w = torch.randn((E, values_of(D, H)), generator=g, device=dev) * scale.to(dev)
    ids = torch.randint(0, max(1, E // 3) if skew else E, (n, K), generator=g, device=dev, dtype=torch.int32)
    if absent:
        ids[torch.rand((n, K), generator=g, device=dev) < absent] = -1
        if n:
            ids[n // 2] = -1                                        # a row without any head
    gates = torch.rand((n, K), generator=g, device=dev)
    up = torch.randn((n,), generator=g, device=dev)
    return x, w, ids, gates, up


def definition(x, w, ids, gates, up, H):
    import torch
    n, D = x.shape
    x64 = x.double().clone().requires_grad_(True)
    w64 = w.double().clone().requires_grad_(True)
    g64 = (gates.double().clone() if gates is not None else torch.ones(ids.shape, dtype=torch.float64, device=x.device)).requires_grad_(True)
    energy = torch.zeros(n, dtype=torch.float64, device=x.device)
    for e in range(len(w)):
        for k in range(ids.shape[1]):
            rows = (ids[:, k] == e).nonzero()[:, 0]
            if not len(rows):
                continue
            t, at = w64[e], 0

            def take(*shape):
                nonlocal at
                m = int(np.prod(shape))
                at += m
                return t[at - m:at].view(*shape)
            y = torch.nn.functional.silu(x64[rows] @ take(64, D).t() + take(64))
            for _ in range(H - 1):
                y = y + torch.nn.functional.silu(y @ take(64, 64).t() + take(64))
            v = y @ take(64) + take(1)
            energy = energy.index_add(0, rows, g64[rows, k] * v)
    total = (energy * (up.double() if up is not None else 1.0)).sum()
    if total.requires_grad:
        grads = torch.autograd.grad(total, (x64, w64, g64), allow_unused=True)
    else:
        grads = (None, None, None)
    grads = [torch.zeros_like(s) if d is None else d for d, s in zip(grads, (x64, w64, g64))]
    return energy.detach(), *grads


def run(L, x, w, ids, gates, up, H, want=("energy", "dx", "dweights", "dgates")):
    import torch
    dev = x.device
    n, K = ids.shape
    offsets = torch.empty(len(w) + 1, dtype=torch.int32, device=dev)
    order = torch.empty(n * K, dtype=torch.int32, device=dev)
    L.group(ids, offsets, order)
    nan = float("nan")
    out = dict(energy=torch.full((n,), nan, device=dev), dx=torch.full(x.shape, nan, dtype=x.dtype, device=dev),
               dweights=torch.full_like(w, nan), dgates=torch.full((n, K), nan, device=dev))
    out = {k: v for k, v in out.items() if k in want}
    L.heads(x, w, offsets, order, hidden=H, top_k=K, gates=gates, denergy=up, **out)
    torch.cuda.synchronize()
    return out


def close(got, ref, name, scale=2e-5, rel=0.0):
    import torch
    assert got.shape == ref.shape
    if not ref.numel():
        return 0.0
    assert bool(torch.isfinite(got.float()).all()), name
    err = (got.double() - ref).abs()
    top = float(ref.abs().max())
    assert bool((err <= scale * top + rel * ref.abs()).all()), (name, float(err.max()), top)
    return float(err.max()) / top if top else 0.0


CASES = [  # rows, inputs, layers, heads, heads a row, spare
    (0, 16, 1, 2, 1, 0), (1, 128, 4, 6, 1, 0), (3, 1, 1, 1, 1, 0), (17, 2, 2, 3, 2, 1), (64, 3, 3, 2, 1, 0),
    (129, 5, 4, 4, 1, 3), (128, 64, 4, 1, 1, 0), (500, 65, 2, 7, 3, 2), (1000, 128, 4, 6, 1, 0), (777, 192, 4, 8, 2, 0),
    (300, 129, 5, 3, 1, 0), (900, 200, 6, 2, 1, 5), (257, 384, 8, 5, 1, 0), (640, 96, 7, 64, 4, 0), (400, 130, 1, 3, 2, 0),
    (300, 1024, 2, 2, 1, 0), (5000, 32, 3, 256, 1, 0), (40000, 128, 4, 2, 1, 0)]


@pytest.mark.parametrize("rows,width,hidden,experts,top_k,spare", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_heads_match_definition(rows, width, hidden, experts, top_k, spare, dtype):
    import torch
    from paper_2608_16329_amd import Learner
    x, w, ids, gates, up = inputs(rows, width, hidden, experts, top_k, dtype, spare, rows + width, skew=experts > 5)
    ref = dict(zip(("energy", "dx", "dweights", "dgates"), definition(x, w, ids, gates, up, hidden)))
    # the gradient of a gate whose entry has no head is 0 and the gate not used
    L = Learner()
    gates[ids < 0] = float("nan")
    got = run(L, x, w, ids, gates, up, hidden)
    rel = 2.0 ** -8 if dtype == "bfloat16" else 0.0
    errs = {k: close(got[k], ref[k], k, rel=rel if k == "dx" else 0.0) for k in ref}
    log(f"[heads] {rows}x{width} H{hidden} E{experts} k{top_k} {dtype}: " + " ".join(f"{k} {v:.1e}" for k, v in errs.items()))
    again = run(L, x, w, ids, gates, up, hidden)
    for k in got:
        assert torch.equal(got[k], again[k]), k                    # the same bits from run to run
    # the energies alone, and with the descriptors' gradient alone
    for want in (("energy",), ("energy", "dx"), ("dweights",), ("dx", "dgates")):
        part = run(L, x, w, ids, gates, up, hidden, want)
        for k in want:
            close(part[k], ref[k], k, rel=rel if k == "dx" else 0.0)
    L.close()


def test_species_heads_are_the_potentials():
    """Species as experts, no gates, no upstream gradient: energies and dE/dG of
    the head tables of a potential's blob."""
    import torch
    from oracle.model import Model
    from paper_2608_16329_amd import Learner
    hp = synth.HParams(n_species=3)
    blob = synth.random_weights(hp, 4)
    tables = blob[-3 * values_of(128, 4):].reshape(3, -1)
    rng = np.random.default_rng(1)
    n = 1234
    G = rng.normal(0, 1, (n, 128)) ** 2
    types = rng.integers(0, 3, n).astype(np.int32)
    x = torch.from_numpy(G).to("cuda:0", torch.float32)
    w = torch.from_numpy(tables).to("cuda:0", torch.float32)
    got = run(Learner(), x, w, torch.from_numpy(types).cuda()[:, None], None, None, 4, ("energy", "dx"))
    ref = definition(x, w, torch.from_numpy(types).cuda()[:, None], None, None, 4)
    close(got["energy"], ref[0], "energy")
    close(got["dx"], ref[1], "dx")
    assert Model(hp, blob) is not None


def test_gradients_against_differences():
    """Directional derivatives of the float64 definition by central differences,
    along random directions in descriptors, weights and gates."""
    import torch
    from paper_2608_16329_amd import Learner
    n, D, H, E, K = 60, 48, 4, 3, 2
    x, w, ids, gates, up = inputs(n, D, H, E, K, "float32", 0, 9)
    got = run(Learner(), x, w, ids, gates, up, H)
    g = torch.Generator(device="cuda:0").manual_seed(2)
    for name, at in (("dx", 0), ("dweights", 1), ("dgates", 3)):
        args = [x.double(), w.double(), ids, gates.double(), up.double()]
        v = torch.randn(args[at].shape, generator=g, device="cuda:0", dtype=torch.float64)
        h = 1e-5

        def total(s):
            a = list(args)
            a[at] = a[at] + s * h * v
            return float((definition(*a, H)[0] * up.double()).sum())
        fd = (total(1) - total(-1)) / (2 * h)
        an = float((got[name].double() * v).sum())
        size = float((got[name].double() * v).norm())
        assert abs(fd - an) <= 1e-4 * max(size, abs(fd)), (name, fd, an)


def test_a_nan_stays_with_its_row():
    import torch
    from paper_2608_16329_amd import Learner
    x, w, ids, gates, up = inputs(700, 128, 4, 2, 1, "float32", 0, 3, absent=0.0)
    x[77, 5] = float("nan")
    got = run(Learner(), x, w, ids, gates, up, 4, ("energy", "dx"))
    bad = torch.isnan(got["energy"])
    assert bool(bad[77]) and int(bad.sum()) == 1
    assert int(torch.isnan(got["dx"]).any(1).sum()) == 1


def test_long_head_and_short_heads():
    """One head with most of the rows beside many with one or none: sums of all
    work-groups of a head, and heads without rows."""
    from paper_2608_16329_amd import Learner
    import torch
    n, D, H, E = 70000, 64, 2, 40
    x, w, ids, gates, up = inputs(n, D, H, E, 1, "float32", 0, 5, absent=0.0)
    ids[:] = 20
    ids[:10, 0] = torch.arange(10, dtype=torch.int32) * 4
    got = run(Learner(), x, w, ids, gates, up, H)
    ref = dict(zip(("energy", "dx", "dweights", "dgates"), definition(x, w, ids, gates, up, H)))
    for k in ref:
        close(got[k], ref[k], k)
    assert float(got["dweights"][1].abs().max()) == 0.0


def test_refusals():
    import torch
    from paper_2608_16329_amd import Learner, MlipError
    L = Learner()
    x, w, ids, gates, up = inputs(20, 32, 2, 3, 2, "float32", 0, 1)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    order = torch.zeros(40, dtype=torch.int32, device="cuda:0")
    L.group(ids, offsets, order)
    e = torch.empty(20, device="cuda:0")
    L.heads(x, w, offsets, order, hidden=2, top_k=2, energy=e)
    with pytest.raises(MlipError, match="no output"):
        L.heads(x, w, offsets, order, hidden=2, top_k=2)
    with pytest.raises(ValueError, match="values a head"):
        L.heads(x, w, offsets, order, hidden=3, top_k=2, energy=e)
    with pytest.raises(MlipError, match="hidden"):
        L.heads(x, w, offsets, order, hidden=9, top_k=2, energy=e)
    with pytest.raises(ValueError, match="order"):
        L.heads(x, w, offsets, order[:30], hidden=2, top_k=2, energy=e)
    with pytest.raises(ValueError, match="offsets"):
        L.heads(x, w, offsets[:3], order, hidden=2, top_k=2, energy=e)
    with pytest.raises(ValueError, match="dx"):
        L.heads(x, w, offsets, order, hidden=2, top_k=2, dx=torch.empty((20, 32), dtype=torch.bfloat16, device="cuda:0"))
    with pytest.raises(ValueError, match="weights"):
        L.heads(x, w.double(), offsets, order, hidden=2, top_k=2, energy=e)
    with pytest.raises(ValueError, match="next to each other"):
        L.heads(torch.empty((32, 20), device="cuda:0").t(), w, offsets, order, hidden=2, top_k=2, energy=e)


@pytest.mark.parametrize("rows,width,heads,dtype", [((1 << 31) - 1, 1, 1, "bfloat16"), ((1 << 30) + 5, 2, 2, "float32")])
def test_as_many_rows_as_there_may_be(rows, width, heads, dtype):
    """Row numbers up to 2^31 - 2, more than 2^32 values that are copied to rows
    of four, and memory beyond 2^32 bytes from its start."""
    import torch
    from paper_2608_16329_amd import Learner
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GiB of free memory")
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(3)
    _, w, _, _, _ = inputs(1, width, 1, heads, 1, dtype, 0, 8)
    x = torch.empty((rows, width), dtype=getattr(torch, dtype), device=dev)
    ids = torch.zeros((rows, 1), dtype=torch.int32, device=dev)
    for at in range(0, rows, 1 << 27):
        x[at:at + (1 << 27)].copy_(torch.rand(x[at:at + (1 << 27)].shape, generator=g, device=dev))
        if heads > 1:
            ids[at:at + (1 << 27)].copy_(torch.randint(0, heads, ids[at:at + (1 << 27)].shape, generator=g, device=dev))
    L = Learner()
    offsets, order = torch.empty(heads + 1, dtype=torch.int32, device=dev), torch.empty(rows, dtype=torch.int32, device=dev)
    L.group(ids, offsets, order)
    energy = torch.full((rows,), float("nan"), device=dev)
    L.heads(x, w, offsets, order, hidden=1, energy=energy)
    torch.cuda.synchronize()
    assert int(offsets[heads]) == rows
    some = torch.cat([torch.arange(0, 500), torch.arange((1 << 30) - 250, (1 << 30) + 5), torch.arange(rows - 500, rows)]).to(dev)
    ref = definition(x[some], w, ids[some], torch.ones((len(some), 1), device=dev), None, 1)[0]
    close(energy[some], ref, "energy")
    del energy, order, ids, x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_far_apart(dtype):
    """Rows 2^26 values apart, memory beyond 2^32 values from its start: the same bits as rows side by side."""
    import torch
    from paper_2608_16329_amd import Learner
    n, D, H, E = 70, 36, 2, 3
    x, w, ids, gates, up = inputs(n, D, H, E, 1, dtype, 0, 6)
    far = torch.empty((n, 1 << 26), dtype=x.dtype, device=x.device)[:, 7:7 + D]
    far.copy_(x)
    L = Learner()
    a, b = run(L, x, w, ids, gates, up, H), run(L, far, w, ids, gates, up, H)
    for k in a:
        assert torch.equal(a[k], b[k]), k
