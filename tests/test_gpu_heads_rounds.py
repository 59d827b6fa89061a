"""Weight gradients where a work-group has several tiles of a head: sums that go
on from tile to tile in registers and (inputs beyond 128) in memory, layers kept in
memory (5 and more), the next tile's rows under way.  Eight wavefronts up to 4
layers, four beyond.  Definition and tolerances as in test_gpu_heads.py, with
each layer's gradient measured by its own largest value."""
import pytest

from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu

CASES = [  # rows, inputs, layers, heads, heads a row, spare: 600 tiles and more for 256 work-groups
    (40000, 200, 4, 3, 2, 0), (80000, 130, 1, 2, 1, 1), (80000, 64, 2, 3, 1, 0), (40000, 130, 3, 5, 2, 3),
    (100000, 384, 4, 2, 1, 0), (40000, 192, 6, 4, 1, 0), (40000, 72, 5, 2, 1, 5), (20000, 320, 8, 3, 2, 0), (40000, 3, 7, 2, 1, 0)]


@pytest.mark.parametrize("rows,width,hidden,experts,top_k,spare", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_tiles_a_work_group(rows, width, hidden, experts, top_k, spare, dtype):
    import torch
    from paper_2608_16329_amd import Learner
    from tests.test_gpu_heads import close, definition, inputs, run
    from tests.test_gpu_heads_accuracy import layers
    x, w, ids, gates, up = inputs(rows, width, hidden, experts, top_k, dtype, spare, rows + width)
    ref = dict(zip(("energy", "dx", "dweights", "dgates"), definition(x, w, ids, gates, up, hidden)))
    L = Learner()
    gates[ids < 0] = float("nan")
    got = run(L, x, w, ids, gates, up, hidden)
    again = run(L, x, w, ids, gates, up, hidden)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    rel = 2.0 ** -8 if dtype == "bfloat16" else 0.0
    errs = {k: close(got[k], ref[k], k, rel=rel if k == "dx" else 0.0) for k in ("energy", "dx", "dgates")}
    for t, (a, b) in enumerate(zip(layers(got["dweights"], width, hidden), layers(ref["dweights"], width, hidden))):
        errs[f"dw{t}"] = close(a, b, f"dweights {t}")
    log(f"[heads] {rows}x{width} H{hidden} E{experts} k{top_k} {dtype}: " + " ".join(f"{k} {v:.1e}" for k, v in errs.items()))
    part = run(L, x, w, ids, gates, up, hidden, ("dweights",))
    assert torch.equal(part["dweights"], got["dweights"])
    L.close()
