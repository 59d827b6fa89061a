"""8-bit moments of blocks whose gradients differ by orders of magnitude, and plans
of more pieces than work-groups."""
import math

import numpy as np
import pytest

from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu


def test_elements_far_below_their_blocks_largest():
    """Constant gradients of 0.76 and 10^-1 .. 10^-4 of it in blocks of 256, 300 steps, as include/mlip.h says: v below
    2^-18 2^e is held as that, and steps are shorter by the root of the ratio; larger ones are right on average.

    Tolerances: a rounding moves v by 0.41 of a gap between codes (root mean square), a gap is at most 7% of the values
    here, and v remembers 100 steps: 0.41 x 7% x sqrt(50) = 20% an element, 0.4% in the mean over 64 blocks of 50; m
    likewise 0.2%.  The mean of 1 / sqrt(v) is 3/8 of the spread's square off, 1.5%.  5% is asked of both means.  The
    largest v, 0.55 on average, stay between 1/2 and 1 (0.09 a rounding's memory), so that e is 0."""
    import torch
    from paper_2608_16329_amd import AdamW
    dev, blocks, steps, b1, b2, lr = torch.device("cuda:0"), 64, 300, 0.9, 0.99, 1e-3
    grad = torch.empty((blocks, 256), device=dev)
    share = torch.ones(256, device=dev)
    share[56:] = 10.0 ** -(1.0 + torch.arange(200, device=dev) // 50).float()
    grad[:] = 0.76 * share
    param, held = torch.zeros_like(grad), None
    opt = AdamW([param], [grad], bits=8)
    for step in range(1, steps + 1):
        held = param.clone() if step == steps else None
        opt.step(step, lr=lr, beta1=b1, beta2=b2, eps=1e-12, seed=step)
    m, v = torch.empty(grad.numel(), device=dev), torch.empty(grad.numel(), device=dev)
    opt.moments(m, v)
    v, moved = v.view(blocks, 256).double(), (held - param).double()
    assert opt.v_exp.unique().tolist() == [127]
    floor = 2.0 ** -18
    for k in range(1, 5):
        at = (share * 10 ** k - 1).abs() < 1e-3
        true = (0.76 * 10.0 ** -k) ** 2 * (1 - b2 ** steps)
        got, step_size = float(v[:, at].mean()), float(moved[:, at].mean())
        want = max(true, floor)
        log(f"[adamw] gradients 10^-{k} of the largest: v {got:.3e} of {true:.3e}, steps {step_size / lr:.4f} of lr")
        if true < floor:
            assert bool((v[:, at] == floor).all())
        assert abs(got / want - 1) <= 0.05
        # the update takes v before it is rounded
        used = b2 * want + (1 - b2) * (0.76 * 10.0 ** -k) ** 2
        assert abs(step_size / (lr * math.sqrt(true / used)) - 1) <= 0.05


def test_the_largest_sizes():
    """Sizes of 2^127 and more are held as the largest code of their block, smaller ones as everywhere."""
    import torch
    from paper_2608_16329_amd import AdamW
    param, grad = torch.zeros(256, device="cuda:0"), torch.ones(256, device="cuda:0")
    opt = AdamW([param], [grad], bits=8)
    # v' = 0.99 v + 0.01, v = 1.875 x 2^127
    opt.v.fill_(254)
    opt.v_exp.fill_(127 + 127)
    opt.step(1, lr=0.0, seed=1)
    m, v = torch.empty(256, device="cuda:0"), torch.empty(256, device="cuda:0")
    opt.moments(m, v)
    assert opt.v_exp.tolist() == [126 + 127]
    assert v.tolist() == [1.875 * 2.0 ** 126] * 256


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype", ["float32", "bfloat16"])
def test_more_pieces_than_work_groups(bits, gtype):
    """7,900 pieces for at most 2,048 work-groups: long tensors, thousands of one element, and odd ones.  Moments and codes
    exactly as float32 operations one by one give them; parameters as in test_gpu_adamw.py."""
    import torch
    from paper_2608_16329_amd import AdamW
    from tests.test_gpu_adamw import dice, f32, make, pow2
    sizes = [5000003] + [1] * 3000 + [257, 1025, 0, 255] + [1024] * 3
    n = sum(sizes)
    param, grad = make(sizes, "float32", gtype, 5)
    opt = AdamW(param.split(sizes), grad.split(sizes), bits=bits, decay=[k % 2 == 0 for k in range(len(sizes))])
    starts = np.cumsum([0] + sizes[:-1])
    first = np.concatenate([a + np.arange(0, z, 256) for a, z in zip(starts, sizes) if z])       # of every block
    block = np.repeat(np.arange(len(first)), np.diff(np.append(first, n)))
    lr, b1, b2, eps, wd = 1e-3, 0.9, 0.99, 1e-8, 0.05
    keep = np.repeat(np.where(np.arange(len(sizes)) % 2 == 0, f32(1 - lr * wd), f32(1)), sizes).astype(f32)
    m = v = np.zeros(n, f32)

    def held(x, mant, up):
        size = np.abs(x)
        e = np.clip((np.maximum.reduceat(size, first).view(np.int32) >> 23) - 126, -126, 126)
        y = size * pow2(-e)[block]
        ey = np.maximum((y.view(np.int32) >> 23) - 127, -14)
        code = ((ey + 14) << mant) + np.floor((y * pow2(mant - ey)) + up).astype(np.int32)
        code = np.minimum(code, 126 if mant == 3 else 254)
        if mant == 4:
            code = np.where((size > 0) & (code == 0), 1, code)
        ec = code >> mant
        near = ((code & (2 ** mant - 1)) + np.where(ec > 0, 2 ** mant, 0)).astype(f32) * pow2(np.maximum(ec, 1) - 15 - mant) * pow2(e)[block]
        return e + 127, np.where(x < 0, code | 128, code) if mant == 3 else code, np.where(x < 0, -near, near).astype(f32)

    for step in (1, 2, 3):
        p = param.cpu().numpy().astype(np.float64)
        opt.step(step, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, seed=step)
        torch.cuda.synchronize()
        gr = grad.float().cpu().numpy()
        m = m * f32(b1) + gr * f32(1 - b1)
        v = v * f32(b2) + (gr * gr) * f32(1 - b2)
        up = lr / (1 - b1 ** step) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) / math.sqrt(1 - b2 ** step) + eps)
        got = param.cpu().numpy()
        assert (np.abs(got - (p * keep - up)) <= 1e-6 * np.abs(up) + 2.0 ** -23 * np.abs(p)).all()
        if bits == 32:
            assert np.array_equal(opt.m.cpu().numpy(), m) and np.array_equal(opt.v.cpu().numpy(), v)
            continue
        r = dice(step, np.arange(n))
        for x, mant, bitsof, codes, exps in ((m, 3, r & 0xFFFF, opt.m, opt.m_exp), (v, 4, r >> 16, opt.v, opt.v_exp)):
            e, code, near = held(x, mant, bitsof.astype(f32) * f32(2.0 ** -16))
            assert np.array_equal(exps.cpu().numpy(), e) and np.array_equal(codes.cpu().numpy(), code)
            x[:] = near
        vals = [torch.empty(n, device="cuda:0") for _ in range(2)]
        opt.moments(*vals)
        assert np.array_equal(vals[0].cpu().numpy(), m) and np.array_equal(vals[1].cpu().numpy(), v)
    opt.close()
