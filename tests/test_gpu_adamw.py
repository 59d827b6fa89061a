"""AdamW over many tensors with moments in 32 and in 8 bits.

Tolerances: a moment is two float32 products and a sum (2 units in the last
place, 2^-23 of the larger term); the update is a quotient with a square root,
six roundings, 1e-6 of its size, added to the parameter (half a unit).  bf16
parameters are rounded once more (2^-9).  8-bit codes are compared exactly with
the definition's float32 operations done one by one in NumPy, and their values
with the unrounded moment: at most one code apart."""
import math

import numpy as np
import pytest

from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
f32 = np.float32


def pow2(e):
    return np.ldexp(f32(1), e).astype(f32)


def dice(seed, at):
    h = (at.astype(np.uint64) * 0x9E3779B1 + seed) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
    h = ((h ^ (h >> 12)) * 0x297A2D39) & 0xFFFFFFFF
    return h ^ (h >> 15)


def decode(code, e, mant):
    """Values of codes from the header's definition, float64."""
    c = code.astype(int)
    sign = np.where(c > 127, -1.0, 1.0) if mant == 3 else 1.0
    c = c & 127 if mant == 3 else c
    E, f = c >> mant, (c & (2 ** mant - 1)) / 2 ** mant
    v = np.where(E > 0, (1 + f) * 2.0 ** (E - 15), f * 2.0 ** -14) * 2.0 ** e
    return np.where(c == (127 if mant == 3 else 255), np.nan, sign * v)


def encode(x, mant, up):
    """One block: exponent and codes, in float32 as the definition's operations."""
    size = np.abs(x).astype(f32)
    fine = np.isfinite(size)
    top = size[fine].max(initial=0)
    e = int(np.clip((np.array([top], f32).view(np.int32)[0] >> 23) - 126, -126, 126))
    y = np.where(fine, size, 0).astype(f32) * pow2(-e)
    ey = np.maximum((y.view(np.int32) >> 23) - 127, -14)
    whole = np.floor(((y * pow2(mant - ey)).astype(f32) + up.astype(f32)).astype(f32)).astype(int)
    code = np.minimum(((ey + 14) << mant) + whole, 126 if mant == 3 else 254)
    if mant == 4:
        code = np.where((size > 0) & (code == 0), 1, code)
    code = np.where(fine, code, 127 if mant == 3 else 255)
    if mant == 3:
        code = np.where(fine & (x < 0), code | 128, code)
    return e, code.astype(np.uint8)


SETS = {"one": [1], "odd": [1, 255, 256, 257, 3, 0, 64, 513], "ends": [4096, 4097, 8191, 2048, 2049, 65],
        "tables": [128, 128, 16384, 128, 16384, 128, 4096, 32] * 9 + [8192, 64, 4096, 64, 64, 1] * 3, "long": [1000003]}


def make(sizes, ptype, gtype, seed, shift=1):
    """Tensors back to back from an odd place, as in a blob: not aligned."""
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    n = sum(sizes)

    def flat(dtype, scale):
        t = torch.full((n + shift,), float("nan"), dtype=getattr(torch, dtype), device="cuda:0")[shift:]
        t.copy_(torch.randn(n, generator=g, device="cuda:0") * scale)
        return t
    return flat(ptype, 0.3), flat(gtype, 0.02)


@pytest.mark.parametrize("sizes", SETS, ids=list(SETS))
@pytest.mark.parametrize("ptype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_match_definition(sizes, ptype, gtype, bits):
    import torch
    from paper_2608_16329_amd import AdamW
    sizes = SETS[sizes]
    n = sum(sizes)
    param, grad = make(sizes, ptype, gtype, n)
    decay = [k % 3 != 1 for k in range(len(sizes))]
    opt = AdamW(param.split(sizes), grad.split(sizes), bits=bits, decay=decay)
    start = np.cumsum([0] + sizes)
    lr, b1, b2, eps, wd, gs = 3e-3, 0.9, 0.98, 1e-8, 0.05, 0.5
    keep = np.repeat(np.where(decay, f32(1 - lr * wd), f32(1)), sizes).astype(f32)
    m = np.zeros(n, f32)
    v = np.zeros(n, f32)
    for step in (1, 2, 3, 4):
        grad.mul_(-0.7 if step == 3 else 0.9)
        p = param.float().cpu().numpy().astype(np.float64)
        opt.step(step, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, grad_scale=gs, seed=77 * step)
        torch.cuda.synchronize()
        gr = grad.float().cpu().numpy().astype(f32) * f32(gs)
        m = m * f32(b1) + gr * f32(1 - b1)
        v = v * f32(b2) + (gr * gr) * f32(1 - b2)
        up = lr / (1 - b1 ** step) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) / math.sqrt(1 - b2 ** step) + eps)
        want = p * keep - up
        got = param.float().cpu().numpy()
        tol = 1e-6 * np.abs(up) + 2.0 ** -23 * np.abs(p) + (2.0 ** -8 * np.abs(want) if ptype == "bfloat16" else 0)
        assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()
        if bits == 32:
            assert np.array_equal(opt.m.cpu().numpy(), m)
            assert np.array_equal(opt.v.cpu().numpy(), v)
            continue
        r = dice(77 * step, np.arange(n))
        codes_m, codes_v = opt.m.cpu().numpy(), opt.v.cpu().numpy()
        em, ev = opt.m_exp.cpu().numpy(), opt.v_exp.cpu().numpy()
        block = 0
        for a, z in zip(start, sizes):
            for b in range(0, z, 256):
                at = slice(a + b, a + min(b + 256, z))
                for x, mant, u, codes, exps in ((m, 3, r & 0xFFFF, codes_m, em), (v, 4, r >> 16, codes_v, ev)):
                    e, c = encode(x[at], mant, u[at].astype(f32) * f32(2.0 ** -16))
                    assert exps[block] == e + 127 and np.array_equal(codes[at], c), (step, a, b, mant)
                    near = decode(c, e, mant)
                    size = np.abs(x[at].astype(np.float64))
                    gap = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(size, 1e-300))) - e, -14) - mant) * 2.0 ** e
                    assert (np.abs(near - x[at]) <= gap * 1.0001).all()
                    x[at] = near
                block += 1
        vals = [torch.empty(n, device="cuda:0") for _ in range(2)]
        opt.moments(*vals)
        assert np.array_equal(vals[0].cpu().numpy(), m) and np.array_equal(vals[1].cpu().numpy(), v)
    opt.close()


def test_rounding_is_unbiased():
    """The mean of many roundings of one value lies within five standard
    deviations (at most half a gap / sqrt(n) each) of it."""
    import torch
    from paper_2608_16329_amd import AdamW
    n = 256 * 400
    param, grad = torch.zeros(n, device="cuda:0"), torch.full((n,), 0.0371, device="cuda:0")
    grad[::256] = 0.05
    opt = AdamW([param], [grad], bits=8)
    opt.step(1, lr=0.0, seed=5)
    m, v = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    opt.moments(m, v)
    keep = torch.ones(n, dtype=torch.bool, device="cuda:0")
    keep[::256] = False
    for got, x, mant in ((m, 0.0371 * 0.1, 3), (v, 0.0371 ** 2 * 0.01, 4)):
        mean = float(got[keep].double().mean())
        gap = 2.0 ** (math.floor(math.log2(x)) - mant)
        assert len(got[keep].unique()) == 2
        assert abs(mean - x) <= 5 * 0.5 * gap / math.sqrt(n * 255 / 256) + 1e-6 * x, (mean, x, gap)


def test_not_finite_stays_where_it_is():
    import torch
    from paper_2608_16329_amd import AdamW
    for bits in (32, 8):
        param, grad = make([700], "float32", "float32", 3)
        grad[300], grad[10] = float("nan"), float("inf")
        opt = AdamW([param], [grad], bits=bits)
        for step in (1, 2):
            opt.step(step, lr=1e-3, seed=step)
        bad = ~torch.isfinite(param)
        assert bad.nonzero()[:, 0].tolist() == [10, 300]


def test_extreme_sizes():
    """Zeros, the smallest and the largest values: a moment of 0 stays 0, a v
    that is not 0 never becomes 0, nothing becomes infinite."""
    import torch
    from paper_2608_16329_amd import AdamW
    for size in (0.0, 1e-30, 1e-18, 1e10, 1e18):
        grad = torch.full((600,), size, device="cuda:0")
        grad[1::2] *= 1e-5
        param = torch.zeros(600, device="cuda:0")
        opt = AdamW([param], [grad], bits=8)
        for step in (1, 2, 3):
            opt.step(step, lr=1e-3, seed=step)
        m, v = torch.empty(600, device="cuda:0"), torch.empty(600, device="cuda:0")
        opt.moments(m, v)
        assert bool(torch.isfinite(param).all() and torch.isfinite(m).all() and torch.isfinite(v).all())
        if size == 0.0:
            assert not bool(m.any() or v.any() or param.any())
        if size >= 1e-15:
            assert bool((v > 0).all())
            assert float(param.abs().max()) < 3.5e-3     # three steps of at most about lr each


def test_into_leaves_the_start_alone():
    import torch
    from paper_2608_16329_amd import AdamW
    sizes = SETS["odd"]
    for bits in (32, 8):
        param, grad = make(sizes, "float32", "float32", 8)
        twin = param.clone()
        new = torch.empty_like(param)
        opt = AdamW(param.split(sizes), grad.split(sizes), bits=bits, into=new.split(sizes))
        ref = AdamW(twin.split(sizes), grad.split(sizes), bits=bits)
        held = param.clone()
        opt.step(1, lr=9.0, seed=3)                       # a step that is dropped
        assert torch.equal(param, held)
        for step in (1, 2, 3):
            opt.step(step, lr=1e-3, weight_decay=0.1, seed=step)
            opt.accept()
            ref.step(step, lr=1e-3, weight_decay=0.1, seed=step)
        assert torch.equal(new, twin)                     # an odd number of accepted steps: in the second set
        assert torch.equal(opt.m, ref.m) and torch.equal(opt.v, ref.v)


def test_moments_are_the_last_step_s():
    """What the last step wrote, before and after it is accepted: the moments of
    a plan that updates in place."""
    import torch
    from paper_2608_16329_amd import AdamW
    sizes = SETS["odd"]
    n = sum(sizes)
    param, grad = make(sizes, "float32", "float32", 9)
    twin, new = param.clone(), torch.empty_like(param)
    opt = AdamW(param.split(sizes), grad.split(sizes), bits=8, into=new.split(sizes))
    ref = AdamW(twin.split(sizes), grad.split(sizes), bits=8)

    def values(o):
        m, v = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
        o.moments(m, v)
        return m, v

    assert not any(bool(x.any()) for x in values(opt))
    for step in (1, 2, 3):
        opt.step(step, lr=1e-3, seed=step)
        ref.step(step, lr=1e-3, seed=step)
        want = values(ref)
        assert bool(want[0].any() and want[1].any())
        before = values(opt)
        opt.accept()
        for got in (before, values(opt)):
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_other_stream():
    import torch
    from paper_2608_16329_amd import AdamW
    param, grad = make([5000, 7], "float32", "float32", 4)
    twin = param.clone()
    opt = AdamW(param.split([5000, 7]), grad.split([5000, 7]), stream=torch.cuda.Stream())
    ref = AdamW(twin.split([5000, 7]), grad.split([5000, 7]))
    for step in (1, 2, 3):
        big = torch.randn((2048, 2048), device="cuda:0")
        grad.copy_((big @ big).flatten()[:5007])
        opt.step(step, lr=1e-2)
        ref.step(step, lr=1e-2)
        grad.zero_()
    assert torch.equal(param, twin)


def test_refusals():
    import torch
    from paper_2608_16329_amd import AdamW, MlipError
    p, g = torch.zeros((4, 4), device="cuda:0"), torch.zeros((4, 4), device="cuda:0")
    with pytest.raises(MlipError, match="no tensors"):
        AdamW([], [])
    with pytest.raises(ValueError, match="bits"):
        AdamW([p], [g], bits=16)
    with pytest.raises(ValueError, match="length"):
        AdamW([p], [g, g])
    with pytest.raises(ValueError, match="grads"):
        AdamW([p], [g[:2]])
    with pytest.raises(ValueError, match="float64"):
        AdamW([p.double()], [g])
    with pytest.raises(ValueError, match="contiguous"):
        AdamW([p.t()[:, :2]], [g[:, :2]])
    opt = AdamW([p], [g])
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan")), dict(grad_scale=float("inf"))):
        with pytest.raises(MlipError, match="ARG"):
            opt.step(**{"step": 1, "lr": 1e-3, **bad})
    with pytest.raises(ValueError, match="into"):
        opt.accept()
    with pytest.raises(MlipError, match="already"):
        opt.moments(torch.empty(16, device="cuda:0"), torch.empty(16, device="cuda:0"))
    log("[adamw] refusals answered")
