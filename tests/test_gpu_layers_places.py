"""Wide layers where their data stands otherwise than in the other tests: expert 0's
rows not the first ones, and tensors that start at the alignment of one value.
Tolerances of the products as in test_gpu_product8.py, with the largest product of a
row's block of 128 for that of eight neighbours."""
import pytest

pytestmark = pytest.mark.gpu


def odd(fill, dtype, *shape):
    """A contiguous tensor one value behind an allocation's start."""
    import torch
    n = 1
    for s in shape:
        n *= s
    return torch.full((n + 1,), fill, dtype=dtype, device="cuda")[1:].view(shape)


# few rows, tiles, more experts than a wavefront has lanes; gradients with and without slices
@pytest.mark.parametrize("m,K,N,E,first", [(50, 130, 40, 2, 20), (3000, 200, 130, 5, 1000), (40000, 640, 300, 256, 777), (70000, 300, 520, 3, 33333)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_products_behind_the_first_rows(m, K, N, E, first, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    g, kind = torch.Generator(device="cuda").manual_seed(m), getattr(torch, dtype)
    last = m - 3
    x, dy, w = (torch.randn(s, generator=g, device="cuda") for s in ((m, K), (m, N), (E, N, K)))
    for t in (x, dy):
        t[:first], t[last:] = float("nan"), float("nan")     # nobody's rows
    cuts = torch.sort(torch.randint(first, last, (E - 1,), generator=g, device="cuda")).values.tolist()
    ends = [first] + cuts + [last]
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    L, x8, dy8, w8 = Learner(), Rows8(m, K), Rows8(m, N), Weights8(E, N, K)
    L.pack8(x, x8)
    L.pack8(dy, dy8)
    L.pack8_weights(w, w8)
    c = odd(0.0, torch.float32, E, N)
    c.copy_(torch.randn((E, N), generator=g, device="cuda"))
    y, dx, dw, db = odd(3.0, kind, m, N), odd(3.0, kind, m, K), odd(3.0, torch.float32, E, N, K), odd(3.0, torch.float32, E, N)
    L.product8(x8, w8, y, offsets=off, bias=c)
    L.product8(dy8, w8, dx, offsets=off, transposed=True)
    L.product8_weights(dy8, x8, dw, offsets=off, dbias=db)

    def held(r):
        v = torch.empty((r.rows, r.width), device="cuda")
        L.unpack8(r, v)
        return v.double()
    xv, dv = held(x8), held(dy8)
    wv = held(Rows8(E * N, K, codes=w8.codes.reshape(E * N, -1),
                    exps=w8.exps.repeat_interleave(128, 1)[:, :N].reshape(E * N, -1).contiguous())).view(E, N, K)
    for t in (y, dx):
        assert bool((t[:first] == 3).all()) and bool((t[last:] == 3).all())

    def tops(t):
        pad = (-t.shape[1]) % 128
        return torch.nn.functional.pad(t.abs(), (0, pad)).view(t.shape[0], (t.shape[1] + pad) // 128, 128).amax(2)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        n = b - a
        for got, of, mat, add in ((y, xv, wv[e], c[e].double()), (dx, dv, wv[e].t().contiguous(), None)):
            of, mt = of[a:b], mat.t().contiguous()
            want, size = of @ mt, of.abs() @ mt.abs()
            if add is not None:
                want, size = want + add, size + add.abs()
            bound = (mat.shape[1] / 32 + 5) * 2.0 ** -23 * size
            if dtype == "bfloat16":
                bound = bound + 2.0 ** -8 * want.abs() + 7 * 16 * 2.0 ** -13 * (tops(of) @ tops(mat).t().contiguous())
            assert bool(((got[a:b].double() - want).abs() <= bound).all()), e
        bound = (n / 32 + 4 + n / 256) * 2.0 ** -23
        dt = dv[a:b].t().contiguous()
        assert bool(((dw[e].double() - dt @ xv[a:b]).abs() <= bound * (dt.abs() @ xv[a:b].abs())).all()), e
        assert bool(((db[e].double() - dt.sum(1)).abs() <= (bound + n / 32 * 2.0 ** -23) * dt.abs().sum(1)).all()), e
    L.close()


@pytest.mark.parametrize("w", [130, 512])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_at_one_values_alignment(w, dtype):
    """The bits of tensors that start at an allocation's."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    n, k, E, kind = 700, 3, 7, getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(w)
    L = Learner()
    offsets, order = (torch.empty(s, dtype=torch.int32, device="cuda") for s in (E + 1, n * k))
    L.group(torch.randint(-1, E, (n, k), generator=g, device="cuda", dtype=torch.int32), offsets, order)
    rows, matrices = torch.randn((n, w), generator=g, device="cuda"), torch.randn((2, 200, w), generator=g, device="cuda")
    results = []
    for place in (odd, lambda fill, dtype, *s: torch.full(s, fill, dtype=dtype, device="cuda")):
        x, m = place(0.0, kind, n, w), place(0.0, kind, 2, 200, w)
        x.copy_(rows), m.copy_(matrices)
        xs, dy, out, h, dz, back = (place(5.0, kind, r, w) for r in (n * k, n * k, n, n, n, n))
        places, dgates = torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda")
        kept, w8 = Rows8(n, w), Weights8(2, 200, w)
        L.sort(x, offsets, order, xs, places)
        L.combine(xs, places, out)
        L.combine_backward(x, xs, places, dy, dgates=dgates)
        L.activate8(x, kept, h)
        L.activate8_backward(kept, x, dz)
        L.unpack8(kept, back)
        L.pack8_weights(m, w8)
        results.append((xs, dy, out, h, dz, back, places, dgates, kept.codes, kept.exps, w8.codes, w8.t_codes, w8.exps, w8.t_exps))
    for i, (one, other) in enumerate(zip(*results)):
        assert torch.equal(one, other), i
    L.close()
