"""Rows packed in the experts' order: entries that are none leave their rows as they
are, codes and exponents, as sorting leaves the rows of values."""
import pytest

pytestmark = pytest.mark.gpu


# widths: a row's exponents written by one of four, one of two, or all four groups of lanes, and in two words
@pytest.mark.parametrize("w", [64, 128, 200, 256, 300, 512, 640, 1100])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_entries_that_are_none(w, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    n, k = 6, 2
    x = torch.randn((n, w), device="cuda").to(getattr(torch, dtype))
    # the first, last and neighbouring rows of what a wavefront has; negative, one too many, the largest number
    order = torch.tensor([-1, 3, 12, 0, 2147483647, -2147483648, 5, 11, -5, 77, 1, 2], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 4, 10], dtype=torch.int32, device="cuda")
    L, r, rows = Learner(), Rows8(n * k, w), Rows8(n, w)
    r.codes.fill_(0x55), r.exps.fill_(0x66)
    L.pack8(x, r, offsets=offsets, order=order, top_k=k)
    L.pack8(x, rows)
    for p, entry in enumerate(order.tolist()):
        if p < 10 and 0 <= entry < n * k:
            assert torch.equal(r.codes[p], rows.codes[entry // k]) and torch.equal(r.exps[p], rows.exps[entry // k]), p
        else:
            assert bool((r.codes[p] == 0x55).all()) and bool((r.exps[p] == 0x66).all()), p
    L.close()
