"""A training step through two wide layers of experts, as it is put together:
routing, grouping, rows into 8 bits in the experts' order, products, an activation
that keeps its argument in 8 bits, and back, with all gradients; recorded in graphs;
on streams; and what the Python calls refuse.

Each link is held, from what the one before it wrote, to its definition in 64 bits
(tolerances as in test_gpu_rows8.py, test_gpu_mix.py and test_gpu_product8.py)."""
import numpy as np
import pytest

from tests.layers_reference import dsilu, held, silu

pytestmark = pytest.mark.gpu


def host(t):
    return t.double().cpu().numpy()


class Step:
    """One expert layer pair over n rows: D inputs, H hidden, R outputs, E experts, k of them a row."""

    def __init__(self, n, D, H, R, E, k, dtype, stream=None):
        import torch
        from paper_2608_16329_amd import Learner, Rows8, Weights8
        g = torch.Generator(device="cuda").manual_seed(n + D)
        m, f32, i32, dev = n * k, torch.float32, torch.int32, "cuda"

        def rand(*s, scale=1.0):
            return torch.randn(s, generator=g, device=dev) * scale
        self.k, self.L = k, Learner(stream=stream)
        self.x, self.logits, self.dout = rand(n, D).to(dtype), rand(n, E), rand(n, R).to(dtype)
        self.logits[::7, : E // 2] = -float("inf")
        self.logits[3::11] = -float("inf")                    # rows without any expert
        self.W1, self.b1 = rand(E, H, D, scale=D ** -0.5), rand(E, H)
        self.W2, self.b2 = rand(E, R, H, scale=H ** -0.5), rand(E, R)
        empty = lambda *s, dtype=f32: torch.zeros(s, dtype=dtype, device=dev)
        self.experts, self.gates = empty(n, k, dtype=i32), empty(n, k)
        self.counts, self.loss = empty(E + 1, dtype=i32), empty(1)
        self.offsets, self.order, self.places = empty(E + 1, dtype=i32), empty(m, dtype=i32), empty(n, k, dtype=i32)
        self.xs, self.dxs, self.dx = empty(m, D, dtype=dtype), empty(m, D, dtype=dtype), empty(n, D, dtype=dtype)
        self.z, self.dh = empty(m, H, dtype=dtype), empty(m, H, dtype=dtype)
        self.y, self.dy, self.out = empty(m, R, dtype=dtype), empty(m, R, dtype=dtype), empty(n, R, dtype=dtype)
        self.x8, self.h8, self.kept, self.dz8, self.dy8 = (Rows8(m, w) for w in (D, H, H, H, R))
        for r in (self.x8, self.h8, self.kept, self.dz8, self.dy8):
            r.codes.zero_(), r.exps.zero_()
        self.w1, self.w2 = Weights8(E, H, D), Weights8(E, R, H)
        self.dW1, self.db1, self.dW2, self.db2 = (torch.zeros_like(t) for t in (self.W1, self.b1, self.W2, self.b2))
        self.dgates, self.dlogits = empty(n, k), empty(n, E)

    def run(self):
        s, L = self, self.L
        L.pack8_weights(s.W1, s.w1)
        L.pack8_weights(s.W2, s.w2)
        L.route(s.logits, s.experts, s.gates, s.counts, s.loss)
        L.group(s.experts, s.offsets, s.order)
        L.sort(s.x, s.offsets, s.order, s.xs, s.places)
        L.pack8(s.x, s.x8, offsets=s.offsets, order=s.order, top_k=s.k)
        L.product8(s.x8, s.w1, s.z, offsets=s.offsets, bias=s.b1)
        L.activate8(s.z, s.kept, h8=s.h8)
        L.product8(s.h8, s.w2, s.y, offsets=s.offsets, bias=s.b2)
        L.combine(s.y, s.places, s.out, gates=s.gates)
        L.combine_backward(s.dout, s.y, s.places, s.dy, gates=s.gates, dgates=s.dgates)
        L.route_backward(s.logits, s.experts, s.counts, s.dlogits, dgates=s.dgates)
        L.pack8(s.dy, s.dy8)
        L.product8_weights(s.dy8, s.h8, s.dW2, offsets=s.offsets, dbias=s.db2)
        L.product8(s.dy8, s.w2, s.dh, offsets=s.offsets, transposed=True)
        L.activate8_backward(s.kept, s.dh, dz8=s.dz8)
        L.product8_weights(s.dz8, s.x8, s.dW1, offsets=s.offsets, dbias=s.db1)
        L.product8(s.dz8, s.w1, s.dxs, offsets=s.offsets, transposed=True)
        L.combine(s.dxs, s.places, s.dx)

    NAMES = ("out", "dx", "dW1", "db1", "dW2", "db2", "dgates", "dlogits", "xs", "y")

    def results(self):
        return {n: getattr(self, n).clone() for n in self.NAMES}

    def values(self, r):
        import torch
        v = torch.empty((r.rows, r.width), device="cuda")
        self.L.unpack8(r, v)
        return host(v)


@pytest.mark.parametrize("n,D,H,R,E,k", [(300, 96, 200, 64, 5, 2), (2000, 193, 320, 130, 8, 1), (9, 40, 33, 7, 4, 4)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_step(n, D, H, R, E, k, dtype):
    import torch
    dtype = getattr(torch, dtype)
    s = Step(n, D, H, R, E, k, dtype)
    s.run()
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    offsets, order, places = (t.cpu().numpy() for t in (s.offsets, s.order, s.places))
    live = offsets[-1]
    assert 0 < live < n * k
    x8, h8, kept, dz8, dy8 = (s.values(r) for r in (s.x8, s.h8, s.kept, s.dz8, s.dy8))
    rows = order[:live] // k
    assert np.array_equal(host(s.xs)[:live], host(s.x)[rows]) and np.array_equal(x8[:live], held(host(s.x))[rows])
    z = host(s.z)[:live]
    assert np.array_equal(kept[:live], held(z))
    # h8: one rounding of 2^-4, or 2^-10 of the block's unit, at most 2^-8 of its largest, from silu(z) and its rounding to dtype
    h = silu(z)
    top = np.concatenate([np.repeat(np.abs(h[:, j:j + 128]).max(1, keepdims=True), min(128, H - j), 1) for j in range(0, H, 128)], 1)
    assert (np.abs(h8[:live] - h) <= (2.0 ** -4 + 2 * step + 2.0 ** -20) * np.abs(h) + 2.0 ** -15 * top).all()
    g = host(s.gates).reshape(-1)[order[:live]]
    dout = host(s.dout)[rows]
    assert (np.abs(host(s.dy)[:live] - g[:, None] * dout) <= (step + 2.0 ** -23) * np.abs(g[:, None] * dout)).all()
    assert np.array_equal(dy8[:live], held(host(s.dy)[:live]))
    dh = host(s.dh)[:live]
    dz = dh * dsilu(kept[:live])
    sg = 1 / (1 + np.exp(-kept[:live]))
    top = np.concatenate([np.repeat(np.abs(dz[:, j:j + 128]).max(1, keepdims=True), min(128, H - j), 1) for j in range(0, H, 128)], 1)
    err = np.abs(dh) * sg * (1 + np.abs(kept[:live])) * (16 + 8 * np.abs(kept[:live])) * 2.0 ** -24
    assert (np.abs(dz8[:live] - dz) <= (2.0 ** -4 + 2 * step) * np.abs(dz) + 2 * err + 2.0 ** -15 * top).all()
    # products, from what was packed
    w1, w2 = held(host(s.W1), matrix=True), held(host(s.W2), matrix=True)
    cut = 7 * 2.0 ** -13 if dtype == torch.bfloat16 else 0.0
    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        for got, a, w, bias in ((s.z, x8, w1[e], s.b1), (s.y, h8, w2[e], s.b2), (s.dh, dy8, w2[e].T, None), (s.dxs, dz8, w1[e].T, None)):
            want, size = a[r] @ w.T, np.abs(a[r]) @ np.abs(w).T
            if bias is not None:
                want, size = want + host(bias)[e], size + np.abs(host(bias)[e])
            bound = (w.shape[1] / 32 + 5) * 2.0 ** -23 * size + step * np.abs(want) + cut * size
            assert (np.abs(host(got)[r] - want) <= bound).all()
        for got, own, a, b in ((s.dW2, s.db2, dy8, h8), (s.dW1, s.db1, dz8, x8)):
            m = offsets[e + 1] - offsets[e]
            bound = (m / 32 + 4 + m / 256) * 2.0 ** -23
            assert (np.abs(host(got)[e] - a[r].T @ b[r]) <= bound * (np.abs(a[r]).T @ np.abs(b[r]))).all()
            assert (np.abs(host(own)[e] - a[r].sum(0)) <= (bound + m / 32 * 2.0 ** -23) * np.abs(a[r]).sum(0)).all()
    there = places >= 0
    y = np.where(there[..., None], host(s.y)[np.maximum(places, 0)], 0) * np.where(there, host(s.gates), 0)[..., None]
    assert (np.abs(host(s.out) - y.sum(1)) <= k * 2.0 ** -24 * np.abs(y).sum(1) + step * np.abs(y.sum(1))).all()
    assert not host(s.out)[~there.any(1)].any() and not host(s.dx)[~there.any(1)].any()
    dots = np.where(there[..., None], host(s.y)[np.maximum(places, 0)], 0) * host(s.dout)[:, None]
    assert (np.abs(host(s.dgates) - dots.sum(2)) <= (R / 8 + 10) * 2.0 ** -24 * np.abs(dots).sum(2)).all()
    s.L.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_recorded_step(dtype):
    """Two steps recorded in graphs, replayed in turn with other inputs between eager calls: the bits of eager calls."""
    import torch
    dtype = getattr(torch, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = Step(700, 96, 256, 64, 6, 2, dtype, stream=side), Step(150, 200, 130, 33, 3, 1, dtype, stream=side)
    b.L.close()
    b.L = a.L                                                 # one context, one workspace
    eager = [Step(700, 96, 256, 64, 6, 2, dtype), Step(150, 200, 130, 33, 3, 1, dtype)]
    torch.cuda.synchronize()
    graphs = []
    with torch.cuda.stream(side):
        a.run()
        b.run()
    side.synchronize()
    for s in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.run()
        graphs.append(graph)
    for turn in range(4):
        for s, e in zip((a, b), eager):
            for t in (s, e):
                t.x.copy_(torch.roll(t.x, turn, 0) * (1 + turn))
                t.logits.copy_(torch.roll(t.logits, 2 * turn, 0))
                t.W1.copy_(torch.roll(t.W1, turn, 1))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for graph in graphs if turn % 2 else graphs[::-1]:
                graph.replay()
        torch.cuda.synchronize()
        for s, e in zip((a, b), eager):
            e.run()
            got, want = s.results(), e.results()
            for name in Step.NAMES:
                assert torch.equal(got[name], want[name]), (turn, name)
            s.out.zero_(), s.dx.zero_(), s.dW1.zero_()
        torch.cuda.synchronize()
    a.L.close()


def test_step_on_another_stream():
    """Inputs written late on the current stream, the step on one of its own: the bits of one stream."""
    import torch
    one, two = Step(500, 64, 128, 32, 4, 2, torch.bfloat16), Step(500, 64, 128, 32, 4, 2, torch.bfloat16, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    for turn in range(3):
        big = torch.randn((4096, 4096), device="cuda")
        late = (big @ big)[0, 0].tanh()
        for s in (two, one):
            s.x.mul_(1 + 0.1 * late.to(s.x.dtype))
            s.run()
        got, want = two.results(), one.results()
        for name in Step.NAMES:
            assert torch.equal(got[name], want[name]), (turn, name)
    one.L.close()
    two.L.close()


def test_refusals_in_python():
    import torch
    from paper_2608_16329_amd import Learner, MlipError, Rows8, Weights8
    L = Learner()
    f = lambda *s, dtype=torch.float32, device="cuda": torch.zeros(s, dtype=dtype, device=device)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    x, xs, places, offsets, order = f(4, 8), f(8, 8), i(4, 2), i(4), i(8)
    r, w = Rows8(4, 8), Weights8(3, 5, 8, transposed=False)
    refused = [
        lambda: L.sort(x.cpu(), offsets, order, xs, places), lambda: L.sort(x.half(), offsets, order, xs, places),
        lambda: L.sort(x, offsets.long(), order, xs, places), lambda: L.sort(x, offsets, i(7), xs, places),
        lambda: L.sort(x, offsets, order, f(7, 8), places), lambda: L.sort(x, offsets, order, xs, i(8)),
        lambda: L.sort(x, offsets, order, xs.bfloat16(), places), lambda: L.sort(x.t(), offsets, order, xs, places),
        lambda: L.combine(xs, places, f(5, 8)), lambda: L.combine(f(9, 8), places, x), lambda: L.combine(xs, places, x, gates=f(4, 3)),
        lambda: L.combine(xs, places.long(), x), lambda: L.combine_backward(x, None, places, xs, dgates=f(4, 2)),
        lambda: L.combine_backward(x, xs.bfloat16(), places, xs, dgates=f(4, 2)), lambda: L.combine_backward(f(5, 8), xs, places, xs),
        lambda: L.pack8(f(5, 8), r), lambda: L.pack8(f(4, 9), r), lambda: L.pack8(x, r, top_k=2), lambda: L.pack8(x, r, order=order),
        lambda: L.pack8(x, Rows8(4, 8, device="cpu")), lambda: L.unpack8(r, f(4, 9)), lambda: L.unpack8(r, x.half()),
        lambda: L.pack8_weights(f(3, 5, 9), w), lambda: L.pack8_weights(f(3, 5, 8).half(), w),
        lambda: L.product8(r, w, f(4, 5)), lambda: L.product8(r, w, f(4, 6), offsets=i(4)), lambda: L.product8(r, w, f(4, 5), offsets=i(3)),
        lambda: L.product8(r, w, f(4, 5), offsets=i(4), bias=f(3, 6)), lambda: L.product8(Rows8(4, 5), w, x, offsets=i(4), transposed=True),
        lambda: L.product8_weights(r, Rows8(5, 8), f(1, 8, 8)), lambda: L.product8_weights(r, r, f(3, 8, 8)),
        lambda: L.product8_weights(r, r, f(1, 8, 8), dbias=f(8)), lambda: L.activate8(x, Rows8(4, 9)), lambda: L.activate8(x, r, f(4, 9)),
        lambda: L.activate8(x, r, x, residual=x.bfloat16()), lambda: L.activate8_backward(Rows8(3, 8), x, x), lambda: L.activate8(x[0], r)]
    for k, call in enumerate(refused):
        with pytest.raises((ValueError, AttributeError)):
            call()
            pytest.fail(f"call {k} was not refused")
    for call in (lambda: L.activate8(x), lambda: L.activate8_backward(r, x), lambda: L.sort(f(4, 0), offsets, order, f(8, 0), places),
                 lambda: L.combine(f(4 * 17, 8), i(4, 17), x)):
        with pytest.raises(MlipError) as e:
            call()
        assert e.value.status == -1 and str(e.value)
    # nothing to do is fine
    L.sort(f(0, 8), offsets, i(0), f(0, 8), i(0, 2))
    L.combine(f(0, 8), i(0, 2), f(0, 8))
    L.pack8(f(0, 8), Rows8(0, 8))
    L.unpack8(Rows8(0, 8), f(0, 8))
    L.activate8(f(0, 8), Rows8(0, 8), f(0, 8))
    L.product8(Rows8(0, 8), w, f(0, 5), offsets=i(4))
    dw, db = torch.ones((3, 5, 8), device="cuda"), torch.ones((3, 5), device="cuda")
    L.product8_weights(Rows8(0, 5), Rows8(0, 8), dw, offsets=i(4), dbias=db)
    assert not dw.any() and not db.any()
    L.close()
