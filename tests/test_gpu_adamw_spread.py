"""8-bit moments of blocks whose gradients differ by orders of magnitude, and plans
of more pieces than work-groups."""
import math

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
