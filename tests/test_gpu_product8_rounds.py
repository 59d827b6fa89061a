"""Products of rows in 8 bits where work-groups take several tiles each, full and
partial ones, of one to many blocks of inputs: every result against a product in 64
bits (tolerances as in test_gpu_product8.py; the part that bfloat16 results may lose
in an instruction is bounded with the largest product of a row's block of 128, which
is at least that of any eight)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,K,N,E", [(70000, 128, 512, 3), (70001, 200, 520, 2), (40000, 640, 1024, 1), (33000, 1300, 777, 4), (200000, 60, 260, 16),
                                     (40001, 300, 2100, 3), (131149, 640, 1024, 5), (30011, 100, 1029, 2), (131149, 70, 1031, 2)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_tiles(m, K, N, E, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn((m, K), generator=g, device="cuda") * torch.exp(torch.randn((m, 1), generator=g, device="cuda"))
    w, c = torch.randn((E, N, K), generator=g, device="cuda"), torch.randn((E, N), generator=g, device="cuda")
    cuts = torch.sort(torch.randint(0, m - 5, (E - 1,), generator=g, device="cuda")).values.tolist()
    ends = [0] + cuts + [m - 5]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    L, x8, w8 = Learner(), Rows8(m, K), Weights8(E, N, K, transposed=False)
    L.pack8(x, x8)
    L.pack8_weights(w, w8)
    kind = getattr(torch, dtype)
    y = torch.full((m, N), 3.0, dtype=kind, device="cuda")
    xv, again = torch.empty_like(x), torch.full((m, N), 4.0, dtype=kind, device="cuda")
    L.unpack8(x8, xv)
    rows = Rows8(E * N, K, codes=w8.codes.reshape(E * N, -1),
                 exps=w8.exps.repeat_interleave(128, 1)[:, :N].reshape(E * N, -1).contiguous())
    wv = torch.empty((E * N, K), device="cuda")
    L.unpack8(rows, wv)
    wv = wv.view(E, N, K)
    for _ in range(3):                                        # one after another, the same bits each
        L.product8(x8, w8, y, offsets=off, bias=c)
        L.product8(x8, w8, again, offsets=off, bias=c)
        assert torch.equal(y[:m - 5], again[:m - 5])
    assert (y[m - 5:] == 3).all()
    pad = (-K) % 128
    for e in range(E):
        for a in range(ends[e], ends[e + 1], 16384):
            b = min(ends[e + 1], a + 16384)
            xd, wd = xv[a:b].double(), wv[e].double()
            want = xd @ wd.t().contiguous() + c[e].double()
            size = xd.abs() @ wd.abs().t().contiguous() + c[e].double().abs()
            bound = (K / 32 + 5) * 2.0 ** -23 * size
            if dtype == "bfloat16":
                xt = torch.nn.functional.pad(xd.abs(), (0, pad)).view(b - a, -1, 128).amax(2)
                wt = torch.nn.functional.pad(wd.abs(), (0, pad)).view(N, -1, 128).amax(2)
                bound = bound + 2.0 ** -8 * want.abs() + 7 * 16 * 2.0 ** -13 * (xt @ wt.t().contiguous())
            assert bool(((y[a:b].double() - want).abs() <= bound).all()), (e, a)
    L.close()


@pytest.mark.parametrize("m,K,N,E", [(20011, 512, 512, 3), (5003, 2048, 2048, 4), (17009, 500, 512, 70), (33333, 1000, 700, 1), (16411, 256, 2300, 9)])
def test_gradients_in_large_tiles(m, K, N, E):
    """Matrices whose gradients have tiles of 256 x 256, experts whose rows end within a step, NaN behind the last."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    g = torch.Generator(device="cuda").manual_seed(m)
    x, dy = torch.randn((m, K), generator=g, device="cuda"), torch.randn((m, N), generator=g, device="cuda")
    x[m - 7:], dy[m - 7:] = float("nan"), float("nan")
    cuts = torch.sort(torch.randint(0, m - 7, (E - 1,), generator=g, device="cuda")).values.tolist()
    ends = [0] + cuts + [m - 7]
    if E > 2:
        ends[1] = ends[2]                                     # one without rows
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    L, x8, dy8 = Learner(), Rows8(m, K), Rows8(m, N)
    L.pack8(x, x8)
    L.pack8(dy, dy8)
    xv, dv = torch.empty_like(x), torch.empty_like(dy)
    L.unpack8(x8, xv)
    L.unpack8(dy8, dv)
    dw, db = torch.full((E, N, K), 3.0, device="cuda"), torch.full((E, N), 3.0, device="cuda")
    L.product8_weights(dy8, x8, dw, offsets=off, dbias=db)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        xd, dd = xv[a:b].double(), dv[a:b].double()
        bound = ((b - a) / 32 + 4 + (b - a) / 256) * 2.0 ** -23
        want, size = dd.t().contiguous() @ xd, dd.abs().t().contiguous() @ xd.abs()
        assert bool(((dw[e].double() - want).abs() <= bound * size).all()), e
        assert bool(((db[e].double() - dd.sum(0)).abs() <= (bound + (b - a) / 32 * 2.0 ** -23) * dd.abs().sum(0)).all()), e
    again = torch.full((E, N, K), 4.0, device="cuda")
    L.product8_weights(dy8, x8, again, offsets=off)
    assert torch.equal(dw, again)
    L.close()
