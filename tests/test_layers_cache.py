"""When rows in 8 bits go past the last cache (csrc/layers.h), as a program for the CPU;
and that packing gives the same on both sides of that rule."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rule(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime.h")):
        pytest.skip("g++ and the HIP headers")
    exe = str(tmp_path / "layers_cache")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-o", exe,
                    os.path.join(ROOT, "tests", "layers_cache.cpp")], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and not res.stdout, res.stdout


# few rows for many experts, which stay in the cache, odd widths; the same rule's other side
@pytest.mark.gpu
@pytest.mark.parametrize("n,w,k,E,dtype", [(10240, 1024, 16, 64, "bfloat16"), (45001, 515, 3, 9, "float32"), (40003, 1001, 6, 16, "bfloat16"),
                                           (30011, 769, 5, 5, "float32")])
def test_packed_entries(n, w, k, E, dtype):
    import torch
    from paper_2608_16329_amd import Learner, Rows8
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((n, w), generator=g, device="cuda").to(getattr(torch, dtype))
    experts = torch.rand((n, E), generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
    experts[torch.rand((n, k), generator=g, device="cuda") < 0.05] = -1
    offsets, order = (torch.empty(s, dtype=torch.int32, device="cuda") for s in (E + 1, n * k))
    L, packed, rows = Learner(), Rows8(n * k, w), Rows8(n, w)
    L.group(experts, offsets, order)
    packed.codes.fill_(0x55), packed.exps.fill_(0x66)
    L.pack8(x, packed, offsets=offsets, order=order, top_k=k)
    L.pack8(x, rows)
    live = int(offsets[-1])
    assert 0 < live < n * k
    at = (order[:live] // k).long()
    assert torch.equal(packed.codes[:live], rows.codes[at]) and torch.equal(packed.exps[:live], rows.exps[at])
    assert bool((packed.codes[live:] == 0x55).all()) and bool((packed.exps[live:] == 0x66).all())
    L.close()
