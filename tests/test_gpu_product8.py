"""Products of rows and matrices in 8 bits over grouped rows, and the gradients of
the matrices, against products of the packed values in 64 bits.

Products of two codes are exact in float32.  float32 results: instructions of 32
products each, whose own sums are good to 4 x 2^-23 of the sum of the sizes, and
K / 32 additions of partial sums no larger than that, each off by at most one unit
in the last place, 2^-23: (K / 32 + 4) 2^-23 of it, the bias one more, and one
for each of the slices' sums of a gradient.  The bias's gradient: four sums of a
quarter of the rows each, two rows an instruction, n / 8 roundings of half a unit:
n / 16 of 2^-23 for n / 32.  bfloat16 results: an instruction adds
eight neighbouring products with their bits below 2^-13 of the largest one's power
of two cut off, 7 x 2^-13 of it for every eight; the rest as above; and half a
step of the result, 2^-8."""
import numpy as np
import pytest

from tests.layers_reference import held

pytestmark = pytest.mark.gpu

CASES = [  # rows, inputs, outputs, experts, rows without an expert, experts without rows
    (1, 1, 1, 1, 0, ()), (1, 1024, 1024, 1, 0, ()), (3, 130, 5, 1, 0, ()), (16, 128, 16, 1, 0, ()), (17, 129, 33, 2, 1, ()), (40, 640, 260, 4, 3, (1,)),
    (64, 384, 128, 8, 0, (0, 7)), (100, 100, 100, 1, 0, ()), (129, 257, 129, 1, 2, ()), (300, 385, 321, 3, 7, (2,)), (700, 1, 200, 2, 0, ()),
    (500, 200, 1, 2, 5, ()), (1000, 1024, 130, 5, 9, (0, 3)), (513, 128, 512, 256, 4, ()), (2000, 64, 64, 70, 0, (69,)), (257, 1153, 384, 1, 0, ())]


def rows(rng, n, w):
    x = rng.standard_normal((n, w)) * np.exp(rng.standard_normal((n, 1)))
    x[rng.random(n) < 0.05] = 0
    return x


def make(seed, m, K, N, E, spare, skip):
    import torch
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, E, m - spare)
    for e in skip:
        ids[ids == e] = next(f for f in range(E) if f not in skip)
    counts = np.bincount(ids, minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    x, w = rows(rng, m, K).astype(np.float32), rng.standard_normal((E, N, K)).astype(np.float32) / np.float32(np.sqrt(K))
    dy, bias = rows(rng, m, N).astype(np.float32), rng.standard_normal((E, N)).astype(np.float32)
    x[offsets[-1]:], dy[offsets[-1]:] = np.nan, np.nan        # nobody's rows
    return offsets, *(torch.from_numpy(v).cuda() for v in (x, w, dy, bias))


def host(t):
    return t.double().cpu().numpy()


def cut(x, w, K):
    """7 x 2^-13 of the largest product's power of two of every eight neighbours, added up: rows, outputs."""
    pad = (-K) % 8
    t = np.abs(np.pad(x, ((0, 0), (0, pad)))[:, None, :] * np.pad(w, ((0, 0), (0, pad)))[None])
    top = t.reshape(*t.shape[:2], -1, 8).max(3)
    return 7 * 2.0 ** -13 * np.where(top > 0, np.exp2(np.floor(np.log2(np.where(top > 0, top, 1)))), 0).sum(2)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:4])))
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bias", [True, False])
def test_product_and_gradient_in_x(case, dtype, bias):
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    m, K, N, E, spare, skip = case
    offsets, x, w, dy, c = make(m + K, *case)
    f32, dtype = dtype == "float32", getattr(torch, dtype)
    L, w8, x8, dy8 = Learner(), Weights8(E, N, K), Rows8(m, K), Rows8(m, N)
    L.pack8_weights(w, w8)
    L.pack8(x, x8)
    L.pack8(dy, dy8)
    off = torch.from_numpy(offsets).cuda() if E > 1 or spare else None
    y = torch.full((m, N), 3.0, dtype=dtype, device="cuda")
    dx = torch.full((m, K), 3.0, dtype=dtype, device="cuda")
    L.product8(x8, w8, y, offsets=off, bias=c if bias else None)
    L.product8(dy8, w8, dx, offsets=off, transposed=True)
    wv = held(host(w), matrix=True)
    for got, of, mat, add, inner in ((host(y), held(host(x)), wv, host(c) if bias else None, K),
                                     (host(dx), held(host(dy)), wv.transpose(0, 2, 1), None, N)):
        assert (got[offsets[-1]:] == 3.0).all()
        for e in range(E):
            a, b = offsets[e], offsets[e + 1]
            if a == b:
                continue
            want, size = of[a:b] @ mat[e].T, np.abs(of[a:b]) @ np.abs(mat[e]).T
            if add is not None:
                want, size = want + add[e], size + np.abs(add[e])
            bound = (inner / 32 + 5) * 2.0 ** -23 * size
            if not f32:
                bound = bound + 2.0 ** -8 * np.abs(want) + cut(of[a:b], mat[e], inner)
            assert (np.abs(got[a:b] - want) <= bound).all()
    L.close()


@pytest.mark.parametrize("case", CASES + [(5000, 100, 60, 1, 3, ()), (20000, 130, 140, 3, 100, (1,)), (9000, 257, 64, 40, 0, (5, 6))],
                         ids=lambda c: "-".join(map(str, c[:4])))
def test_gradients_of_the_matrices(case):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    m, K, N, E, spare, skip = case
    offsets, x, w, dy, c = make(m * 3 + K, *case)
    L, x8, dy8 = Learner(), Rows8(m, K), Rows8(m, N)
    L.pack8(x, x8)
    L.pack8(dy, dy8)
    off = torch.from_numpy(offsets).cuda() if E > 1 or spare else None
    dw, db = torch.full((E, N, K), 3.0, device="cuda"), torch.full((E, N), 3.0, device="cuda")
    L.product8_weights(dy8, x8, dw, offsets=off, dbias=db)
    xv, dv = held(host(x)), held(host(dy))
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        n = b - a
        bound = (n / 32 + 4 + n / 256) * 2.0 ** -23
        assert (np.abs(host(dw)[e] - dv[a:b].T @ xv[a:b]) <= bound * (np.abs(dv[a:b]).T @ np.abs(xv[a:b]))).all()
        assert (np.abs(host(db)[e] - dv[a:b].sum(0)) <= (bound + n / 32 * 2.0 ** -23) * np.abs(dv[a:b]).sum(0)).all()
    again = torch.full((E, N, K), 4.0, device="cuda")
    L.product8_weights(dy8, x8, again, offsets=off)
    assert torch.equal(dw, again)                             # the same bits, with and without dbias
    L.close()


@pytest.mark.parametrize("m,K,N", [(40, 300, 200), (8, 300, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_nan_stays_in_its_row(m, K, N, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    x, w = torch.randn((m, K), device="cuda"), torch.randn((1, N, K), device="cuda")
    x[3, 7], w[0, 5, 2], x[0, 9] = float("nan"), float("nan"), float("inf")
    L, x8, w8 = Learner(), Rows8(m, K), Weights8(1, N, K)
    L.pack8(x, x8)
    L.pack8_weights(w, w8)
    y = torch.zeros((m, N), dtype=getattr(torch, dtype), device="cuda")
    L.product8(x8, w8, y)
    nan = np.isnan(host(y))
    want = np.zeros((m, N), bool)
    want[3], want[0], want[:, 5] = True, True, True
    assert np.array_equal(nan, want)
    dw, db, dy8 = torch.zeros((1, N, K), device="cuda"), torch.zeros((1, N), device="cuda"), Rows8(m, N)
    dy = torch.randn((m, N), device="cuda")
    dy[2, 11] = float("nan")
    L.pack8(dy, dy8)
    L.product8_weights(dy8, x8, dw, dbias=db)
    want = np.zeros((N, K), bool)
    want[11], want[:, 7], want[:, 9] = True, True, True
    assert np.array_equal(np.isnan(host(dw)[0]), want) and np.flatnonzero(np.isnan(host(db)[0])).tolist() == [11]
    L.close()


def test_gradients_against_differences():
    """y is linear in the packed rows and matrices: differences of the loss <dy, y> over steps that 8 bits hold."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    g = torch.Generator(device="cuda").manual_seed(2)
    m, K, N = 24, 136, 20
    pick = torch.tensor([-1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5], device="cuda")

    def some(*shape):
        return pick[torch.randint(0, 7, shape, generator=g, device="cuda")]
    x, w, dy = some(m, K), some(1, N, K), some(m, N)
    x[:, 0], x[:, -1], w[0, 0, 0], w[0, 0, -1], dy[:, 0] = 1.5, 1.5, 1.5, 1.5, 1.5
    L, x8, w8, dy8 = Learner(), Rows8(m, K), Weights8(1, N, K), Rows8(m, N)
    y, dx, dw = torch.empty((m, N), device="cuda"), torch.empty((m, K), device="cuda"), torch.empty((1, N, K), device="cuda")

    def loss(x, w):
        L.pack8(x, x8)
        L.pack8_weights(w, w8)
        L.product8(x8, w8, y)
        return float((y.double() * dy.double()).sum())
    base = loss(x, w)                                         # all sums are of small multiples of 1/4: exact
    L.pack8(dy, dy8)
    L.product8(dy8, w8, dx, transposed=True)
    L.product8_weights(dy8, x8, dw)
    for i, k in ((0, 3), (5, 127), (23, 130), (11, 135)):
        up = x.clone()
        up[i, k] += 0.5 if up[i, k] < 1 else -0.5
        assert (loss(up, w) - base) / float(up[i, k] - x[i, k]) == float(dx[i, k])
    for n, k in ((1, 0), (7, 127), (19, 129)):
        up = w.clone()
        up[0, n, k] += 0.5 if up[0, n, k] < 1 else -0.5
        assert (loss(x, up) - base) / float(up[0, n, k] - w[0, n, k]) == float(dw[0, n, k])
    L.close()


def test_codes_behind_2_to_the_32():
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    m, K, N = 4300000, 1000, 33
    L, x8, w8 = Learner(), Rows8(m, K), Weights8(2, N, K)
    x8.codes.zero_(), x8.exps.fill_(127)
    x, w = torch.randn((200, K), device="cuda"), torch.randn((2, N, K), device="cuda")
    one = Rows8(200, K)
    L.pack8(x, one)
    x8.codes[-200:], x8.exps[-200:] = one.codes, one.exps
    L.pack8_weights(w, w8)
    off = torch.tensor([0, m - 150, m], dtype=torch.int32, device="cuda")
    off2 = torch.tensor([0, 50, 200], dtype=torch.int32, device="cuda")
    xv, wv = torch.empty((200, K), device="cuda"), held(host(w), matrix=True)
    L.unpack8(one, xv)
    for dtype in (torch.float32, torch.bfloat16):
        y, few = torch.empty((m, N), dtype=dtype, device="cuda"), torch.empty((200, N), dtype=dtype, device="cuda")
        L.product8(x8, w8, y, offsets=off)
        L.product8(one, w8, few, offsets=off2)
        assert not y[:-200].any()
        for e, (a, b) in enumerate(((0, 50), (50, 200))):     # the few rows and the many may be added up in another order
            want, size = host(xv)[a:b] @ wv[e].T, np.abs(host(xv)[a:b]) @ np.abs(wv[e]).T
            bound = (K / 32 + 5) * 2.0 ** -23 * size
            if dtype == torch.bfloat16:
                bound = bound + 2.0 ** -8 * np.abs(want) + cut(host(xv)[a:b], wv[e], K)
            for got in (host(y[m - 200 + a:m - 200 + b]), host(few[a:b])):
                assert (np.abs(got - want) <= bound).all()
    dy8, dyone = Rows8(m, N), Rows8(200, N)
    dy8.codes.zero_(), dy8.exps.fill_(127)
    L.pack8(torch.randn((200, N), device="cuda"), dyone)
    dy8.codes[-200:], dy8.exps[-200:] = dyone.codes, dyone.exps
    dw, few = torch.empty((2, N, K), device="cuda"), torch.empty((2, N, K), device="cuda")
    L.product8_weights(dy8, x8, dw, offsets=off)
    L.product8_weights(dyone, one, few, offsets=off2)
    # the same 150 and 50 rows in other tiles: both are within the tolerance of the exact sums
    dv = torch.empty((200, N), device="cuda")
    L.unpack8(dyone, dv)
    for e, (a, b) in enumerate(((0, 50), (50, 200))):
        want, size = host(dv)[a:b].T @ host(xv)[a:b], np.abs(host(dv)[a:b]).T @ np.abs(host(xv)[a:b])
        # rows of zeros add nothing, wherever they are
        for got in (dw, few):
            assert (np.abs(host(got)[e] - want) <= 12 * 2.0 ** -23 * size).all()
    L.close()
