"""Weight gradients of heads whose later layers outgrow the earlier ones.

They are compared layer by layer, each with its own largest value as the measure.
Tolerance: such heads are ill-conditioned (a z whose error is a part of a large sum
decides silu'), so the measure is what float32 operations lose on the same inputs,
computed beside the definition: eight times that, and 2e-6 for what both lose in
sums of other orders."""
import pytest

from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu


def tables(D, H, scales, E, g):
    """Heads with matrix t drawn at scales[t] / sqrt(inputs)."""
    import torch
    rows = []
    for _ in range(E):
        parts = []
        for t in range(H):
            fan = D if t == 0 else 64
            parts += [torch.randn(64 * fan, generator=g) * scales[t] * fan ** -0.5, torch.randn(64, generator=g) * fan ** -0.5]
        rows.append(torch.cat(parts + [torch.randn(65, generator=g) / 8]))
    return torch.stack(rows)


def layers(t, D, H):
    """Matrices and vectors of head tables [E, values], in their order."""
    sizes = [64 * D, 64] + [4096, 64] * (H - 1) + [64, 1]
    return t.split(sizes, dim=1)


def weights_gradient(x, w, ids, up, H, dtype):
    """From the formulas, in `dtype`, every y kept."""
    import torch
    D, out = x.shape[1], []
    for e in range(len(w)):
        rows = ids == e
        xe, ue = x[rows].to(dtype), up[rows].to(dtype)
        p = [q[0] for q in layers(w[e:e + 1].to(dtype), D, H)]
        A = [p[2 * t].view(64, -1) for t in range(H)]
        seen, z, y = [xe], [], 0.0
        for t in range(H):
            z.append(seen[-1] @ A[t].t() + p[2 * t + 1])
            y = y + z[-1] * torch.sigmoid(z[-1])
            seen.append(y)
        grads = [ue.sum().reshape(1), ue @ y]
        u = ue[:, None] * p[-2]
        for t in range(H - 1, -1, -1):
            s = torch.sigmoid(z[t])
            gz = u * (s * (1 + z[t] * (1 - s)))
            grads += [gz.sum(0), (gz.t() @ seen[t]).reshape(-1)]
            u = gz @ A[t] + (u if t else 0)
        out.append(torch.cat(grads[::-1]))
    return torch.stack(out)


@pytest.mark.parametrize("scales", [(0.1, 30, 30), (1, 30, 30, 30), (0.01, 30, 100, 100), (1, 1, 1, 1), (1,) + (30,) * 7],
                         ids=lambda s: "-".join(str(v) for v in s))
@pytest.mark.parametrize("rows", [600, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_layers_gradient_is_float32(scales, rows, dtype):
    import torch
    from paper_2608_16329_amd import Learner
    from tests.test_gpu_heads import run
    H, D, E = len(scales), 72, 2
    g = torch.Generator().manual_seed(rows + H)
    w = tables(D, H, scales, E, g)
    x = (torch.randn((rows, D), generator=g).abs() * 0.7).to(getattr(torch, dtype))
    up = torch.randn(rows, generator=g)
    ids = torch.randint(0, E, (rows, 1), generator=g, dtype=torch.int32)
    got = run(Learner(), x.cuda(), w.cuda(), ids.cuda(), None, up.cuda(), H, ("dweights",))["dweights"].cpu().double()
    ref = weights_gradient(x, w, ids[:, 0], up, H, torch.float64)
    plain = weights_gradient(x, w, ids[:, 0], up, H, torch.float32).double()
    worst = []
    for a, b, r in zip(layers(got, D, H), layers(plain, D, H), layers(ref, D, H)):
        top = float(r.abs().max())
        worst.append((float((a - r).abs().max()) / top, float((b - r).abs().max()) / top))
    log(f"[heads] layers {scales} {rows} rows {dtype}: " + " ".join(f"{a:.1e}/{b:.1e}" for a, b in worst))
    for k, (a, b) in enumerate(worst):
        assert a <= 8 * b + 2e-6, (k, a, b)
