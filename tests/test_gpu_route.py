"""Routing to experts with its balance loss, its gradient, and the grouping of
entries by expert, against their definitions in 64 bits.

Tolerances: probabilities and gates are quotients of at most 256 float32
exponentials, each good to 2 ulp after an argument that is rounded once (error
of exp(z - top) up to |z - top| 2^-24 relative, |z - top| < 40 here); 1e-5
absolute covers both.  The loss sums float32 probabilities; gradients are
products of the above with sums of at most 256 terms of size O(1).  bf16
outputs are rounded once more, 2^-8 relative."""
import numpy as np
import pytest

from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu


def reference(z, k, kinds, allowed, gates_of, dgates, dloss):
    """z float64 [n, E]; everything in float64, row by row."""
    n, E = z.shape
    experts = -np.ones((n, k), np.int32)
    gates = np.zeros((n, k))
    p = np.zeros((n, E))
    live = np.zeros(n, bool)
    for i in range(n):
        use = z[i] != -np.inf
        if kinds is not None:
            use = use & (allowed[kinds[i]] != 0) if 0 <= kinds[i] < len(allowed) else np.zeros(E, bool)
        ids = np.flatnonzero(use)
        if not len(ids):
            continue
        live[i] = True
        e = np.exp(z[i, ids] - z[i, ids].max())
        p[i, ids] = e / e.sum()
        best = ids[np.argsort(-z[i, ids], kind="stable")][:k]
        experts[i, :len(best)] = best
        w = p[i, best]
        gates[i, :len(best)] = w / w.sum() if gates_of == "chosen" else w
    counts = np.array([(experts == e).sum() for e in range(E)] + [live.sum()], np.int32)
    rows, entries = live.sum(), counts[:E].sum()
    f = counts[:E] / max(entries, 1)
    loss = E * (f * p.sum(0)).sum() / max(rows, 1)
    d = np.zeros((n, E))
    for i in np.flatnonzero(live):
        h = dloss * E * f / rows
        there = experts[i] >= 0
        ids, g = experts[i][there], dgates[i][there]
        if gates_of == "all":
            h = h.copy()
            np.add.at(h, ids, g)
        d[i] = p[i] * (h - (p[i] * h).sum())
        if gates_of == "chosen":
            w = gates[i][there]
            d[i, ids] += w * (g - (w * g).sum())
    return experts, gates, counts, loss, d


def run(L, z, k, kinds, allowed, gates_of, dgates, dloss, dtype):
    import torch
    dev = torch.device("cuda:0")
    n, E = z.shape
    out = dict(experts=torch.full((n, k), 7, dtype=torch.int32, device=dev), gates=torch.full((n, k), np.nan, device=dev),
               counts=torch.full((E + 1,), -5, dtype=torch.int32, device=dev), loss=torch.full((1,), np.nan, device=dev),
               dlogits=torch.full((n, E), np.nan, dtype=dtype, device=dev))
    how = dict(kinds=kinds, allowed=allowed, gates_of=gates_of)
    L.route(z, out["experts"], out["gates"], out["counts"], out["loss"], **how)
    L.route_backward(z, out["experts"], out["counts"], out["dlogits"], dgates=dgates, dloss=dloss, **how)
    torch.cuda.synchronize()
    return {name: t.float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()
            for name, t in out.items()}


CASES = [  # rows, experts, top_k, kinds, spare columns
    (0, 3, 1, 0, 0), (1, 1, 1, 0, 0), (1, 256, 16, 0, 0), (7, 2, 2, 0, 1), (255, 4, 1, 2, 0), (256, 5, 5, 3, 2),
    (257, 16, 2, 0, 0), (300, 17, 16, 6, 0), (1000, 29, 3, 6, 3), (513, 64, 4, 16, 0), (777, 65, 7, 1, 5),
    (400, 128, 8, 0, 0), (333, 250, 3, 4, 1), (70001, 6, 2, 6, 0), (20011, 33, 2, 2, 7)]


@pytest.mark.parametrize("rows,experts,top_k,n_kinds,spare", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gates_of", ["chosen", "all"])
def test_route_matches_definition(rows, experts, top_k, n_kinds, spare, dtype, gates_of):
    import torch
    from paper_2608_16329_amd import Learner
    dev, dt = torch.device("cuda:0"), getattr(torch, dtype)
    rng = np.random.default_rng([rows, experts, top_k])
    wide = torch.full((rows, experts + spare), np.nan, dtype=dt, device=dev)
    z = wide[:, :experts]
    # in bf16 many logits are equal; quarter steps make some equal in float32 too
    z.copy_(torch.from_numpy(np.round(4 * rng.normal(0, 2, (rows, experts))) / 4 if experts > 64 else
                             rng.normal(0, 2, (rows, experts))))
    kinds = allowed = kinds_d = allowed_d = None
    if n_kinds:
        kinds = rng.integers(-1, n_kinds + 1, rows).astype(np.int32)      # some kinds have no row in the table
        allowed = (rng.random((n_kinds, experts)) < 0.5).astype(np.uint8)
        allowed[0] = 0                                                   # and one kind no expert
        kinds_d, allowed_d = torch.from_numpy(kinds).to(dev), torch.from_numpy(allowed).to(dev)
    if rows > 5:
        z[2] = -np.inf
        z[3, : experts - 1] = -np.inf
    ref_z = z.double().cpu().numpy()
    if rows and n_kinds:
        # what is masked may hold anything
        masked = ~((kinds >= 0) & (kinds < n_kinds))
        masked = masked[:, None] | (allowed[np.clip(kinds, 0, n_kinds - 1)] == 0)
        bad = torch.from_numpy(masked & (rng.random((rows, experts)) < 0.5)).to(dev)
        z[bad] = float("nan")
        z[torch.from_numpy(masked).to(dev) & ~bad] = float("inf")
    dgates = rng.normal(0, 1, (rows, top_k))
    dg = torch.from_numpy(dgates).to(dev, torch.float32)
    dl = torch.full((1,), 0.3, device=dev)
    L = Learner()
    got = run(L, z, top_k, kinds_d, allowed_d, gates_of, dg, dl, dt)
    again = run(L, z, top_k, kinds_d, allowed_d, gates_of, dg, dl, dt)
    ids, gates, counts, loss, d = reference(ref_z, top_k, kinds, allowed, gates_of, dg.double().cpu().numpy(), 0.3)
    assert np.array_equal(got["experts"], ids)
    assert np.array_equal(got["counts"], counts)
    np.testing.assert_allclose(got["gates"], gates, rtol=0, atol=1e-5)
    np.testing.assert_allclose(got["loss"], [loss], rtol=1e-5, atol=1e-7)
    np.testing.assert_allclose(got["dlogits"], d, rtol=2.0 ** -8 if dtype == "bfloat16" else 0, atol=2e-5)
    for name in got:
        assert np.array_equal(got[name], again[name]), name              # the same bits from run to run
    L.close()


def test_gradient_against_differences():
    """The gradient of the loss and gates by central differences of the float64
    definition, at fixed choices and shares (logits 0.02 apart, steps of 1e-5)."""
    import torch
    from paper_2608_16329_amd import Learner
    rng = np.random.default_rng(3)
    n, E, K = 5, 6, 3
    z = rng.permuted(np.tile(np.arange(E) * 0.4, (n, 1)), axis=1) + rng.uniform(-0.1, 0.1, (n, E))
    z32 = torch.from_numpy(z).to("cuda:0", torch.float32)
    z = z32.double().cpu().numpy()
    dg = rng.normal(0, 1, (n, K)).astype(np.float32)
    for gates_of in ("chosen", "all"):
        got = run(Learner(), z32, K, None, None, gates_of, torch.from_numpy(dg).cuda(), torch.full((1,), 0.7, device="cuda:0"),
                  torch.float32)
        ids = got["experts"]
        f = got["counts"][:E] / got["counts"][:E].sum()

        def value(y):
            e = np.exp(y)
            p = e / e.sum(1, keepdims=True)
            w = np.take_along_axis(p, ids, 1)
            if gates_of == "chosen":
                w = w / w.sum(1, keepdims=True)
            return (dg * w).sum() + 0.7 * E * (f * p.mean(0)).sum()

        for i in range(n):
            for e in range(E):
                h = np.zeros((n, E))
                h[i, e] = 1e-5
                fd = (value(z + h) - value(z - h)) / 2e-5
                assert abs(fd - got["dlogits"][i, e]) < 1e-5, (gates_of, i, e)


def test_nan_in_a_row_stays_in_the_row():
    import torch
    from paper_2608_16329_amd import Learner
    z = torch.zeros((300, 9), device="cuda:0")
    z[5, 3] = float("nan")
    z[6, 2] = float("inf")
    got = run(Learner(), z, 2, None, None, "chosen", torch.ones((300, 2), device="cuda:0"), None, torch.float32)
    bad = np.isnan(got["gates"]).any(1)
    assert bad[5] and bad[6] and bad.sum() == 2
    assert ((got["experts"] >= 0) & (got["experts"] < 9)).all()
    keep = np.ones(300, bool)
    keep[5:7] = False
    assert np.isfinite(got["dlogits"][keep]).all()


@pytest.mark.parametrize("m", [0, 1, 63, 64, 65, 1023, 1025, 8192, 8193, 50001, 4 * 1024 * 64 + 7])
@pytest.mark.parametrize("E", [1, 2, 7, 64, 256])
def test_group_is_a_stable_sort(m, E):
    import torch
    from paper_2608_16329_amd import Learner
    rng = np.random.default_rng([m, E])
    ids = rng.integers(-2, E + 2, m).astype(np.int32)
    if m > 100:
        ids[: m // 2] = rng.integers(0, max(1, E // 8), m // 2)      # some heads get most
    L = Learner()
    offsets = torch.full((E + 1,), -9, dtype=torch.int32, device="cuda:0")
    order = torch.full((m,), -9, dtype=torch.int32, device="cuda:0")
    L.group(torch.from_numpy(ids).cuda(), offsets, order)
    key = np.where((ids >= 0) & (ids < E), ids, E)
    assert np.array_equal(order.cpu().numpy(), np.argsort(key, kind="stable"))
    assert np.array_equal(offsets.cpu().numpy(), np.searchsorted(np.sort(key), np.arange(E + 1)))
    log(f"[group] {m} entries, {E} experts, workspace {L.memory_bytes()} bytes")


def test_other_stream():
    """Inputs made on one stream, the context on another, results used on the first."""
    import torch
    from paper_2608_16329_amd import Learner
    side = torch.cuda.Stream()
    L = Learner(side)
    n, E = 200000, 32
    first = None
    for _ in range(3):
        big = torch.randn((4096, 4096), device="cuda:0")
        z = (big @ big)[:, :E].repeat(49, 1)[:n].contiguous()
        z.normal_(generator=torch.Generator(device="cuda:0").manual_seed(1))
        experts = torch.empty((n, 1), dtype=torch.int32, device="cuda:0")
        gates, loss = torch.empty((n, 1), device="cuda:0"), torch.empty(1, device="cuda:0")
        counts = torch.empty(E + 1, dtype=torch.int32, device="cuda:0")
        L.route(z, experts, gates, counts, loss)
        same = (experts[:, 0] == z.argmax(1)).all()
        assert bool(same)
        first = counts.clone() if first is None else first
        assert torch.equal(first, counts)


def test_refusals():
    import torch
    from paper_2608_16329_amd import Learner, MlipError
    L = Learner()
    dev = torch.device("cuda:0")

    def args(n=4, E=8, k=2, dtype=torch.float32):
        return [torch.zeros((n, E), dtype=dtype, device=dev), torch.zeros((n, k), dtype=torch.int32, device=dev),
                torch.zeros((n, k), device=dev), torch.zeros(E + 1, dtype=torch.int32, device=dev),
                torch.zeros(1, device=dev)]

    L.route(*args())
    for bad in (dict(E=257), dict(E=20, k=17), dict(E=2, k=3), dict(k=0)):
        with pytest.raises(MlipError, match="ARG"):
            L.route(*args(**bad))
    with pytest.raises(ValueError, match="float16"):
        L.route(*args(dtype=torch.float16))
    for place, wrong in ((1, torch.zeros((4, 2), device=dev)), (2, torch.zeros((4, 3), device=dev)),
                         (3, torch.zeros(8, dtype=torch.int32, device=dev)), (4, torch.zeros(2, device=dev)),
                         (0, torch.zeros((4, 8))), (0, torch.zeros((8, 4), device=dev).t())):
        a = args()
        a[place] = wrong
        with pytest.raises(ValueError):
            L.route(*a)
    a = args()
    with pytest.raises(ValueError, match="together"):
        L.route(*a, kinds=torch.zeros(4, dtype=torch.int32, device=dev))
    with pytest.raises(ValueError, match="allowed"):
        L.route(*a, kinds=torch.zeros(4, dtype=torch.int32, device=dev), allowed=torch.zeros((1, 7), dtype=torch.uint8, device=dev))
    with pytest.raises(ValueError, match="gates_of"):
        L.route(*a, gates_of="none")
    with pytest.raises(ValueError, match="dlogits"):
        L.route_backward(a[0], a[1], a[3], torch.zeros((4, 8), dtype=torch.bfloat16, device=dev))
    with pytest.raises(MlipError, match="n_experts"):
        L.group(a[1], torch.zeros(300, dtype=torch.int32, device=dev), torch.zeros(8, dtype=torch.int32, device=dev))
    with pytest.raises(ValueError, match="order"):
        L.group(a[1], torch.zeros(9, dtype=torch.int32, device=dev), torch.zeros(7, dtype=torch.int32, device=dev))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("experts", [3, 8, 29])
def test_rows_far_apart(dtype, experts):
    """Rows 2^26 values apart, memory beyond 2^32 values from its start: the same bits as rows side by side."""
    import torch
    from paper_2608_16329_amd import Learner
    n, K, dev = 70, 2, torch.device("cuda:0")
    z = torch.randn((n, experts), generator=torch.Generator(device=dev).manual_seed(experts), device=dev).to(getattr(torch, dtype))
    far = torch.empty((n, 1 << 26), dtype=z.dtype, device=dev)[:, 5:5 + experts]
    far.copy_(z)
    dgates, one = torch.ones((n, K), device=dev).cumsum(0), torch.ones(1, device=dev)
    L, out = Learner(), []
    for logits in (z, far):
        ids, gates = torch.empty((n, K), dtype=torch.int32, device=dev), torch.empty((n, K), device=dev)
        counts, loss = torch.empty(experts + 1, dtype=torch.int32, device=dev), torch.empty(1, device=dev)
        dlogits = torch.empty((n, experts), dtype=z.dtype, device=dev)
        L.route(logits, ids, gates, counts, loss)
        L.route_backward(logits, ids, counts, dlogits, dgates=dgates, dloss=one)
        out.append((ids, gates, counts, loss, dlogits))
    for a, b in zip(*out):
        assert torch.equal(a, b)
