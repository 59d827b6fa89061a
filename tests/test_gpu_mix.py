"""Rows brought into the experts' order and back with weights, and the gradient,
against their definitions in 64 bits.

Copies are exact.  A sum of k products in float32: k roundings of partial sums no
larger than the sum of the sizes, k 2^-24 of it; a dot product of w terms added by
up to 64 lanes and then pairwise: (w / 8 + 10) 2^-24 at most.  bf16 results are
rounded once, 2^-8 of their size."""
import numpy as np
import pytest

from tests.layers_reference import groups

pytestmark = pytest.mark.gpu

CASES = [  # rows, width, top_k, experts, share without an expert, spare values between rows
    (1, 1, 1, 1, 0.0, 0), (1, 128, 2, 8, 0.0, 0), (5, 3, 3, 4, 0.4, 1), (64, 31, 1, 7, 0.0, 0), (100, 32, 2, 2, 0.1, 0), (77, 385, 3, 29, 0.03, 3),
    (40, 1024, 2, 16, 0.0, 0), (9, 1030, 16, 16, 0.3, 0), (300, 64, 1, 256, 0.5, 7), (33, 4097, 2, 3, 0.2, 1), (12, 256, 4, 6, 1.0, 0),
    (2, 65536, 2, 2, 0.0, 0), (5001, 20, 2, 9, 0.1, 0)]


def spaced(x, dtype, spare):
    import torch
    t = torch.full((x.shape[0], x.shape[1] + spare), float("nan"), dtype=dtype, device="cuda")
    t[:, :x.shape[1]] = torch.from_numpy(x).to(dtype).cuda()
    return t[:, :x.shape[1]]


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("n,w,k,E,empty,spare", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("weighted", [True, False])
def test_sort_combine_and_gradients(n, w, k, E, empty, spare, dtype, weighted):
    import torch
    from paper_2608_16329_amd import Learner
    rng, dtype = np.random.default_rng(n + 7 * w + k), getattr(torch, dtype)
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    _, offsets, order = groups(rng, n, k, E, empty)
    m, live = n * k, int(offsets[-1])
    x = spaced(rng.standard_normal((n, w)), dtype, spare)
    yv = rng.standard_normal((m, w))
    yv[live:] = np.nan                                       # nobody's rows are not looked at
    y, dout = spaced(yv, dtype, 2 * spare), spaced(rng.standard_normal((n, w)), dtype, spare)
    places_want = np.full(m, -1)
    places_want[order[:live]] = np.arange(live)
    gv = rng.random((n, k)).astype(np.float32) - 0.3
    gv.reshape(-1)[places_want < 0] = np.nan                 # nor are their gates
    gates = torch.from_numpy(gv).cuda() if weighted else None
    L = Learner()
    xs = torch.full((m, w), 5.0, dtype=dtype, device="cuda")
    places = torch.full((n, k), 77, dtype=torch.int32, device="cuda")
    L.sort(x, torch.from_numpy(offsets).cuda(), torch.from_numpy(order).cuda(), xs, places)
    assert np.array_equal(places.cpu().numpy().reshape(-1), places_want)
    want = host(x)[order // k]
    want[live:] = 5.0
    assert np.array_equal(host(xs), want)
    alone = torch.full((n, k), 77, dtype=torch.int32, device="cuda")
    L.sort(x, torch.from_numpy(offsets).cuda(), torch.from_numpy(order).cuda(), None, alone)
    assert torch.equal(alone, places)

    out = torch.full((n, w), np.nan, dtype=dtype, device="cuda")
    L.combine(y, places, out, gates=gates)
    g = np.where(places_want >= 0, gv.reshape(-1).astype(np.float64) if weighted else 1.0, 0.0)
    rows = np.where((places_want >= 0)[:, None], host(y)[np.maximum(places_want, 0)], 0.0)
    terms = (rows * g[:, None]).reshape(n, k, w)
    want = terms.sum(1)
    assert (np.abs(host(out) - want) <= k * 2.0 ** -24 * np.abs(terms).sum(1) + step * np.abs(want)).all()

    dy = torch.full((m, w), 6.0, dtype=dtype, device="cuda")
    dgates = torch.full((n, k), np.nan, device="cuda")
    L.combine_backward(dout, y, places, dy, gates=gates, dgates=dgates)
    want = np.full((m, w), 6.0)
    want[places_want[places_want >= 0]] = (np.repeat(host(dout), k, 0) * g[:, None])[places_want >= 0]
    assert (np.abs(host(dy) - want) <= step * np.abs(want)).all()
    terms = rows.reshape(n, k, w) * host(dout)[:, None, :]
    assert (np.abs(host(dgates) - terms.sum(2)) <= (w / 8 + 10) * 2.0 ** -24 * np.abs(terms).sum(2)).all()
    dy2 = torch.full((m, w), 6.0, dtype=dtype, device="cuda")
    L.combine_backward(dout, None, places, dy2, gates=gates)
    assert torch.equal(dy, dy2)

    # the gradient of sort: <dxs, sort(v)> = <combine(dxs), v>
    dx = torch.empty((n, w), dtype=dtype, device="cuda")
    L.combine(xs, places, dx)
    terms = np.where((places_want >= 0)[:, None], host(xs)[np.maximum(places_want, 0)], 0.0).reshape(n, k, w)
    assert (np.abs(host(dx) - terms.sum(1)) <= k * 2.0 ** -24 * np.abs(terms).sum(1) + step * np.abs(terms.sum(1))).all()
    L.close()


def test_combine_gradient_against_differences():
    """combine is linear in y and in the gates: a difference over any step is the derivative but for rounding."""
    import torch
    from paper_2608_16329_amd import Learner
    rng = np.random.default_rng(3)
    n, w, k, E = 6, 50, 2, 3
    _, offsets, order = groups(rng, n, k, E, 0.2)
    L = Learner()
    x = torch.randn((n, w), device="cuda")
    xs, places = torch.zeros((n * k, w), device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda")
    L.sort(x, torch.from_numpy(offsets).cuda(), torch.from_numpy(order).cuda(), xs, places)
    y, gates, dout = torch.randn((n * k, w), device="cuda"), torch.rand((n, k), device="cuda"), torch.randn((n, w), device="cuda")
    dy, dgates, out = torch.zeros_like(y), torch.empty_like(gates), torch.empty_like(x)
    L.combine_backward(dout, y, places, dy, gates=gates, dgates=dgates)

    def loss(y, gates):
        L.combine(y, places, out, gates=gates)
        return float((out.double() * dout.double()).sum())
    size = float((dout.abs().sum() * (y.abs().max() * 2)).double()) * 2.0 ** -22
    for i in range(n):
        for s in range(k):
            up = gates.clone()
            up[i, s] += 1.0
            assert abs(loss(y, up) - loss(y, gates) - float(dgates[i, s])) <= size
    for p in range(n * k):
        up = y.clone()
        up[p, p] += 1.0
        assert abs(loss(up, gates) - loss(y, gates) - float(dy[p, p])) <= size
    L.close()


def test_places_that_are_none():
    """Whatever is no place of a row is no entry: nothing is read or written there."""
    import torch
    from paper_2608_16329_amd import Learner
    L = Learner()
    y = torch.ones((4, 16), device="cuda")
    places = torch.tensor([[0, 4], [-5, 2147483647]], dtype=torch.int32, device="cuda")
    out = torch.empty((2, 16), device="cuda")
    L.combine(y, places, out)
    assert (out[0] == 1).all() and (out[1] == 0).all()
    dy, dg = torch.zeros_like(y), torch.full((2, 2), 9.0, device="cuda")
    L.combine_backward(out + 2, y, places, dy, dgates=dg)
    assert (dy[0] == 3).all() and (dy[1:] == 0).all() and dg.tolist() == [[48.0, 0.0], [0.0, 0.0]]
    offsets, order = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 3, 900], [3, -1, 77, 0]))
    xs = torch.zeros((4, 16), device="cuda")
    places.fill_(-9)
    L.sort(torch.ones((2, 16), device="cuda"), offsets, order, xs, places)
    assert xs.sum(1).tolist() == [16, 0, 0, 16] and places.tolist() == [[3, -9], [-9, 0]]
    L.close()


def test_more_than_2_to_the_32_bytes():
    """Rows whose place lies behind 2^32 values."""
    import torch
    from paper_2608_16329_amd import Learner
    n, w, k = 2200000, 1024, 2
    L = Learner()
    ids = torch.zeros((n, k), dtype=torch.int32, device="cuda")
    ids[:, 1] = 1
    offsets, order = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(n * k, dtype=torch.int32, device="cuda")
    L.group(ids, offsets, order)
    x = torch.zeros((n, w), dtype=torch.bfloat16, device="cuda")
    x[-8:] = torch.randn((8, w), device="cuda").to(torch.bfloat16)
    xs, places = torch.empty((n * k, w), dtype=torch.bfloat16, device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda")
    L.sort(x, offsets, order, xs, places)
    assert torch.equal(xs[-8:], x[-8:]) and torch.equal(xs[n - 8:n], x[-8:])
    out = torch.empty_like(x)
    L.combine(xs, places, out)
    assert torch.equal(out[-8:].float(), 2 * x[-8:].float()) and not out[:-8].any()
    L.combine_backward(x, xs, places, xs.zero_())
    assert torch.equal(xs[-8:], x[-8:]) and torch.equal(xs[n - 8:n], x[-8:])
    L.close()


@pytest.mark.parametrize("n,w,k,E,dtype", [(60001, 385, 3, 9, "float32"), (50003, 1030, 3, 70, "bfloat16"), (50003, 1031, 3, 8, "bfloat16"), (20001, 4096, 1, 2, "float32"), (600001, 30, 4, 5, "float32")])
def test_rows_larger_than_the_last_cache(n, w, k, E, dtype):
    import torch
    from paper_2608_16329_amd import Learner
    dtype, m = getattr(torch, dtype), n * k
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(n)
    x, y, dout = (torch.randn((r, w), generator=g, device="cuda").to(dtype) for r in (n, m, n))
    experts, gates = torch.randint(-1, E, (n, k), generator=g, device="cuda", dtype=torch.int32), torch.rand((n, k), generator=g, device="cuda")
    L = Learner()
    offsets, order = (torch.empty(s, dtype=torch.int32, device="cuda") for s in (E + 1, m))
    L.group(experts, offsets, order)
    live, places = int(offsets[-1]), torch.empty((n, k), dtype=torch.int32, device="cuda")
    xs, dy = torch.full((m, w), 5.0, dtype=dtype, device="cuda"), torch.full((m, w), 5.0, dtype=dtype, device="cuda")
    L.sort(x, offsets, order, xs, places)
    assert torch.equal(xs[:live], x[(order[:live] // k).long()]) and bool((xs[live:] == 5).all())
    out, dgates = torch.empty((n, w), dtype=dtype, device="cuda"), torch.empty((n, k), device="cuda")
    L.combine(y, places, out, gates=gates)
    L.combine_backward(dout, y, places, dy, gates=gates, dgates=dgates)
    for a in range(0, n, 10000):
        p, gt = places[a:a + 10000].long(), gates[a:a + 10000].double()
        terms = torch.where((p >= 0)[..., None], y[p.clamp(min=0)].double(), 0.0)
        weighted = terms * gt[..., None]
        want = weighted.sum(1)
        assert bool(((out[a:a + 10000].double() - want).abs() <= k * 2.0 ** -24 * weighted.abs().sum(1) + step * want.abs()).all())
        d = dout[a:a + 10000].double()
        dots = terms * d[:, None]
        assert bool(((dgates[a:a + 10000].double() - dots.sum(2)).abs() <= (w / 8 + 10) * 2.0 ** -24 * dots.abs().sum(2)).all())
        want = (d[:, None] * gt[..., None])[p >= 0]
        assert bool(((dy[p[p >= 0]].double() - want).abs() <= step * want.abs()).all())
    assert bool((dy[live:] == 5).all())
    L.close()
