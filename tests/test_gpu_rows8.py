"""Rows and matrices in 8 bits, and activations that keep them, against their
definitions in 64 bits.

Packing has no tolerance: exponents are read off the values' bits, a value times
a power of two is exact (or far below the smallest code), and one rounding to
nearest even follows.  Activations: exp is good to 2 ulp of its value, the sum
1 + exp to one more rounding, the quotient to 2, so a sigmoid s is off by 5 x 2^-24
relative; silu is one product more, the derivative s (1 + z (1 - s)) adds 1 - s
(error 5 x 2^-24 s + 2^-24) times |z|, and three roundings: (16 + 8 |z|) 2^-24 of
the largest of its terms, 1 + |z|, times s.  bf16 outputs are rounded once more,
2^-8 of their size."""
import numpy as np
import pytest

from tests.layers_reference import dsilu, groups, held, silu

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 0), (3, 7, 1), (5, 8, 0), (2, 127, 0), (17, 128, 0), (4, 129, 3), (9, 255, 0), (6, 256, 5), (33, 257, 0), (70, 384, 1),
          (5, 513, 0), (300, 1024, 0), (3, 4097, 2), (1, 65536, 0), (2049, 65, 0)]


def values(rng, n, w):
    """Rows of very different sizes, zeros, blocks of zeros, ties and values at the borders of the rule."""
    x = rng.standard_normal((n, w)) * np.exp(rng.standard_normal((n, 1)) * 3)
    x[rng.random((n, w)) < 0.1] = 0
    x[rng.random(n) < 0.1] = 0
    x[:, ::5] = np.rint(x[:, ::5] * 16) / 16
    x[n // 2, 0] = 1.75 * 2.0 ** rng.integers(-20, 20)
    x[n // 3, -1] = 1.875 * 2.0 ** rng.integers(5, 20)
    return x


def tensor(x, dtype, spare=0):
    """x on the GPU in rows `spare` values further apart than they are long, NaN between them."""
    import torch
    t = torch.full((x.shape[0], x.shape[1] + spare), float("nan"), dtype=dtype, device="cuda")
    t[:, :x.shape[1]] = torch.from_numpy(x).to(dtype).cuda()
    return t[:, :x.shape[1]]


def host(t):
    return t.double().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


@pytest.mark.parametrize("n,w,spare", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_pack_unpack(n, w, spare, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    rng, dtype = np.random.default_rng(n * 1000 + w), getattr(torch, dtype)
    x = tensor(values(rng, n, w), dtype, spare)
    L, r = Learner(), Rows8(n, w)
    r.codes.fill_(0x55), r.exps.fill_(0x55)
    L.pack8(x, r)
    want = held(host(x))
    for out in (torch.float32, torch.bfloat16):
        got = torch.full((n, w), 7.0, dtype=out, device="cuda")
        L.unpack8(r, got)
        assert same(host(got), want)
    codes, exps = r.codes.cpu().numpy(), r.exps.cpu().numpy()
    assert not codes[:, w:].any() and not exps[:, (w + 127) // 128:].any()
    L.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_pack_of_what_is_not_finite_and_of_extremes(dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    dtype = getattr(torch, dtype)
    big = torch.finfo(dtype).max
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 300))
    x[0, 3], x[1, 130], x[2, 299], x[3, :] = np.nan, np.inf, -np.inf, np.nan
    x[4] *= 1e-30
    x[5] *= 2.0 ** -110
    x[6] *= 2.0 ** -126
    x[7, :] = 2.0 ** -126
    x[8, 5] = big
    x[9, :] = big
    x[10, :] = -0.0
    x[11, 0], x[11, 1:] = 448.0, 464.0 / 2 ** 9
    x[12, :], x[12, 17] = np.inf, 1.5
    t = tensor(x, dtype)
    L, r = Learner(), Rows8(40, 300)
    L.pack8(t, r)
    got = torch.empty((40, 300), device="cuda")
    L.unpack8(r, got)
    assert same(host(got), held(host(t)))
    L.close()


@pytest.mark.parametrize("n,w,k,E,empty", [(1, 128, 1, 1, 0.0), (50, 200, 2, 5, 0.2), (333, 128, 3, 29, 0.1), (64, 600, 1, 256, 0.0),
                                           (20, 130, 16, 20, 0.5), (40, 64, 2, 3, 1.0)])
def test_pack_in_the_experts_order(n, w, k, E, empty):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    rng = np.random.default_rng(n)
    _, offsets, order = groups(rng, n, k, E, empty)
    x = tensor(values(rng, n, w), torch.float32, 3)
    L, r = Learner(), Rows8(n * k, w)
    r.codes.fill_(0x38), r.exps.fill_(127)
    L.pack8(x, r, offsets=torch.from_numpy(offsets).cuda(), order=torch.from_numpy(order).cuda(), top_k=k)
    got = torch.empty((n * k, w), device="cuda")
    L.unpack8(r, got)
    want = held(host(x))[order // k]
    want[offsets[-1]:] = 1.0                                  # left as they were
    assert same(host(got), want)
    assert (r.codes.cpu().numpy()[offsets[-1]:] == 0x38).all()
    L.close()


@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (2, 3, 130), (1, 128, 128), (3, 129, 127), (2, 300, 257), (1, 64, 1024), (1, 513, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_pack_weights(E, N, K, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8, Weights8
    rng, dtype = np.random.default_rng(N), getattr(torch, dtype)
    w = torch.from_numpy(rng.standard_normal((E, N, K)) * np.exp(rng.standard_normal((E, N, 1)) * 2)).to(dtype).cuda()
    if N * K > 4:
        w[0, N // 2, K // 2] = float("inf")
    want = held(host(w), matrix=True)
    L, w8 = Learner(), Weights8(E, N, K)
    for t in (w8.codes, w8.exps, w8.t_codes, w8.t_exps):
        t.fill_(0x55)
    L.pack8_weights(w, w8)

    def read(codes, exps, width):
        """Values by the rows' reader: a matrix' exponents for each of its rows."""
        rows = codes.shape[1]
        r = Rows8(E * rows, width, codes=codes.reshape(E * rows, -1),
                  exps=exps.repeat_interleave(128, 1)[:, :rows].reshape(E * rows, -1).contiguous())
        got = torch.empty((E * rows, width), device="cuda")
        L.unpack8(r, got)
        return host(got).reshape(E, rows, width)
    assert same(read(w8.codes, w8.exps, K), want)
    assert same(read(w8.t_codes, w8.t_exps, N), want.transpose(0, 2, 1))
    assert not w8.codes.cpu().numpy()[..., K:].any() and not w8.exps.cpu().numpy()[..., (K + 127) // 128:].any()
    assert not w8.t_codes.cpu().numpy()[..., N:].any() and not w8.t_exps.cpu().numpy()[..., (N + 127) // 128:].any()
    alone = Weights8(E, N, K, transposed=False)
    L.pack8_weights(w, alone)
    assert torch.equal(alone.codes, w8.codes) and torch.equal(alone.exps, w8.exps)
    L.close()


@pytest.mark.parametrize("n,w,spare", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_activation(n, w, spare, residual, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    rng, dtype = np.random.default_rng(n + w), getattr(torch, dtype)
    z = rng.standard_normal((n, w)) * 3
    z.reshape(-1)[::7] *= 20
    z = tensor(z, dtype, spare)
    r = tensor(rng.standard_normal((n, w)), dtype, 2 * spare) if residual else None
    dh = tensor(rng.standard_normal((n, w)), dtype, spare)
    L = Learner()
    kept, h8, dz8, again = (Rows8(n, w) for _ in range(4))
    h, dz = (torch.full((n, w), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    L.activate8(z, kept, h, h8=h8, residual=r)
    L.activate8_backward(kept, dh, dz, dz8=dz8)
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    zd, want = host(z), silu(host(z)) + (host(r) if residual else 0)
    assert (np.abs(host(h) - want) <= 8 * 2.0 ** -24 * np.abs(silu(zd)) + step * np.abs(want) + 1e-37).all()
    zk = held(zd)
    want, s = host(dh) * dsilu(zk), 1 / (1 + np.exp(-zk))
    bound = np.abs(host(dh)) * s * (1 + np.abs(zk)) * (16 + 8 * np.abs(zk)) * 2.0 ** -24
    assert (np.abs(host(dz) - want) <= bound + step * np.abs(want) + 1e-37).all()
    # kept and packed outputs are what packing gives
    for packed, of in ((kept, z), (h8, h), (dz8, dz)):
        L.pack8(of, again)
        assert torch.equal(packed.codes, again.codes) and torch.equal(packed.exps, again.exps)
    # each output alone
    one = Rows8(n, w)
    L.activate8(z, None, None, h8=one, residual=r)
    assert torch.equal(one.codes, h8.codes)
    L.activate8_backward(kept, dh, None, dz8=one)
    assert torch.equal(one.codes, dz8.codes)
    L.close()


def test_activation_gradient_against_differences():
    """silu's difference quotient at values that 8 bits hold: curvature |silu''| <= 1/2, step 2^-6, both sides in float32."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    z = torch.arange(-64, 64, device="cuda").reshape(2, 64).float() / 8      # up to 8, in eighths: below 4 all held
    z = z.clamp(-1.875, 1.875) * torch.where(z.abs() < 2, 1.0, 2.0)
    L, kept = Learner(), Rows8(2, 64)
    dz, up, down = torch.empty_like(z), torch.empty_like(z), torch.empty_like(z)
    L.activate8(z, kept, up)
    held_z = torch.empty_like(z)
    L.unpack8(kept, held_z)
    L.activate8_backward(kept, torch.ones_like(z), dz)
    step = 2.0 ** -6
    L.activate8(held_z + step, None, up)
    L.activate8(held_z - step, None, down)
    # the third derivative of silu is below 1, so a central quotient is off by step^2 / 6; sizes up to 4, 2^-22 of them over 2 step
    assert float((((up - down) / (2 * step)) - dz).abs().max()) <= step ** 2 / 6 + 4 * 2.0 ** -22 / (2 * step)
    L.close()


def test_activation_of_large_and_not_finite():
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    z = torch.tensor([[-1000.0, 1000.0, float("nan"), float("inf"), 0.0, -0.0, -87.0, -104.0]], device="cuda").repeat(2, 1)
    z[1, 2:4] = 1.0
    L, kept, h, dz = Learner(), Rows8(2, 8), torch.empty_like(z), torch.empty_like(z)
    L.activate8(z, kept, h)
    L.activate8_backward(kept, torch.ones_like(z), dz)
    h, dz = host(h), host(dz)
    assert np.isnan(h[0, 2]) and np.isinf(h[0, 3]) and np.isnan(dz[0, 2:4]).all()
    assert h[1, 1] == 1000 and abs(h[1, 0]) == 0 and dz[1, 1] == 1 and dz[1, 0] == 0 and dz[1, 4] == 0.5
    assert np.isfinite(h[1]).all() and np.isfinite(dz[1]).all()
    L.close()


def test_more_than_2_to_the_32_values():
    """Rows behind the 2^32nd code and the 2^31st value: the first and last rows are looked at."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    n, w = 4200000, 1024
    x = torch.zeros((n, w), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((64, w), device="cuda").to(torch.bfloat16)
    x[:64], x[-64:] = tail.flip(0), tail
    L, r = Learner(), Rows8(n, w)
    L.pack8(x, r)
    back = torch.empty_like(x)
    L.unpack8(r, back)
    assert same(host(back[-64:]), held(host(tail))) and same(host(back[:64]), held(host(tail.flip(0))))
    h = torch.empty_like(x)
    L.activate8(x, r, h)
    L.activate8_backward(r, x, back)
    one, kept = torch.empty_like(tail), Rows8(64, w)
    L.activate8(tail, kept, one)
    assert torch.equal(one, h[-64:])
    L.activate8_backward(kept, tail, one)
    assert torch.equal(one, back[-64:])
    L.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,w", [(3, 7), (40, 129), (70, 515)])
def test_activation_in_place(n, w, dtype):
    """h over z or over the residual, dz over dh: bit for bit what other places get."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    rng, dtype = np.random.default_rng(w), getattr(torch, dtype)
    z, r, dh = (tensor(values(rng, n, w), dtype) for _ in range(3))
    L, kept, again = Learner(), Rows8(n, w), Rows8(n, w)
    h, dz = torch.empty_like(z), torch.empty_like(z)
    L.activate8(z, kept, h, residual=r)
    L.activate8_backward(kept, dh, dz)
    over_z, over_r, over_dh = z.clone(), r.clone(), dh.clone()
    L.activate8(over_z, again, over_z, residual=r)
    L.activate8(z, None, over_r, residual=over_r)
    L.activate8_backward(again, over_dh, over_dh)
    assert torch.equal(over_z, h) and torch.equal(over_r, h) and torch.equal(over_dh, dz)
    assert torch.equal(again.codes, kept.codes) and torch.equal(again.exps, kept.exps)
    L.close()


@pytest.mark.parametrize("n,w,dtype", [(300001, 257, "float32"), (40003, 3500, "bfloat16"), (1100001, 65, "float32"), (70001, 2050, "bfloat16"), (70001, 2051, "bfloat16")])
def test_values_larger_than_the_last_cache(n, w, dtype):
    """All rows at once and in parts that the cache holds: the same bits."""
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    g, dtype = torch.Generator(device="cuda").manual_seed(n), getattr(torch, dtype)
    z, r, dh = (torch.randn((n, w), generator=g, device="cuda").to(dtype) for _ in range(3))
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    offsets = torch.tensor([0, n - 3], dtype=torch.int32, device="cuda")
    L, packed, sorted8, kept, h8, dz8 = Learner(), *(Rows8(n, w) for _ in range(5))
    h, dz, back = (torch.empty_like(z) for _ in range(3))
    L.pack8(z, packed)
    L.pack8(z, sorted8, offsets=offsets, order=order)
    L.unpack8(packed, back)
    L.activate8(z, kept, h, h8=h8, residual=r)
    L.activate8_backward(kept, dh, dz, dz8=dz8)
    for a in range(0, n, 30000):
        s = slice(a, min(n, a + 30000))
        m = s.stop - a
        one, two, three = (Rows8(m, w) for _ in range(3))
        u, v = torch.empty((m, w), dtype=dtype, device="cuda"), torch.empty((m, w), dtype=dtype, device="cuda")

        def same_as(part, whole):
            return torch.equal(part.codes, whole.codes[s]) and torch.equal(part.exps, whole.exps[s])
        L.pack8(z[s], one)
        L.unpack8(one, u)
        assert same_as(one, packed) and torch.equal(u, back[s])
        L.activate8(z[s], one, u, h8=two, residual=r[s])
        L.activate8_backward(one, dh[s], v, dz8=three)
        assert same_as(one, kept) and same_as(two, h8) and same_as(three, dz8) and torch.equal(u, h[s]) and torch.equal(v, dz[s])
    at = order[:n - 3].long()
    assert torch.equal(sorted8.codes[:n - 3], packed.codes[at]) and torch.equal(sorted8.exps[:n - 3], packed.exps[at])
    L.close()
