"""What the entries of wide layers of experts refuse before anything touches a
device: the C entries (csrc/layers.cpp) with the HIP runtime replaced by counters,
the library's without a context, and the Python classes."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_c_entries(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime.h")):
        pytest.skip("g++ and the HIP headers")
    exe = str(tmp_path / "layers_refusals")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-o", exe,
                    os.path.join(ROOT, "tests", "layers_refusals.cpp"),
                    os.path.join(ROOT, "paper_2608_16329_amd", "csrc", "layers.cpp")], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and not res.stdout, res.stdout


def test_library_without_a_context():
    from paper_2608_16329_amd import binding as b
    p, q = b.mlip_rows_params(1, 1, 8, 0), b.mlip_product8_params(1, 8, 8, 0)
    lib, p, q = b._lib, ctypes.byref(p), ctypes.byref(q)
    assert lib.mlip_sort(None, p, 1, None, 8, None, None, None, None) == -1
    assert lib.mlip_combine(None, p, 1, None, 8, None, None, None) == -1
    assert lib.mlip_combine_backward(None, p, 1, None, 8, None, 8, None, None, None, None) == -1
    assert lib.mlip_pack8(None, p, 1, None, 8, None, None, None, None) == -1
    assert lib.mlip_unpack8(None, p, 1, None, None, None) == -1
    assert lib.mlip_activate8(None, p, 1, None, 8, None, 8, None, None, None, None, None) == -1
    assert lib.mlip_activate8_backward(None, p, 1, None, None, None, 8, None, None, None) == -1
    assert lib.mlip_pack8_weights(None, q, None, None, None, None, None) == -1
    assert lib.mlip_product8(None, q, 1, *[None] * 7) == -1
    assert lib.mlip_product8_weights(None, q, 1, *[None] * 7) == -1
    assert (b.mlip_row8_codes(129), b.mlip_row8_exps(129), b.mlip_row8_codes(-1)) == (256, 4, 0)


def test_places_in_python():
    import torch
    from paper_2608_16329_amd import Rows8, Weights8
    r = Rows8(3, 130, device="cpu")
    assert r.codes.shape == (3, 256) and r.exps.shape == (3, 4) and r.codes.dtype == torch.uint8
    assert Rows8(3, 130, codes=r.codes, exps=r.exps).codes is r.codes
    w = Weights8(2, 130, 600, device="cpu")
    assert w.codes.shape == (2, 130, 640) and w.exps.shape == (2, 2, 8)
    assert w.t_codes.shape == (2, 600, 256) and w.t_exps.shape == (2, 5, 4)
    assert Weights8(2, 130, 600, transposed=False, device="cpu").t_codes is None
    for bad in (lambda: Rows8(-1, 8, device="cpu"), lambda: Rows8(1, 0, device="cpu"), lambda: Rows8(1, 65537, device="cpu"),
                lambda: Rows8(3, 130, codes=r.codes), lambda: Rows8(4, 130, codes=r.codes, exps=r.exps),
                lambda: Rows8(3, 130, codes=r.codes.float(), exps=r.exps), lambda: Rows8(3, 130, codes=r.codes[:, ::2], exps=r.exps),
                lambda: Weights8(0, 1, 1, device="cpu"), lambda: Weights8(257, 1, 1, device="cpu"),
                lambda: Weights8(1, 0, 1, device="cpu"), lambda: Weights8(1, 1, 65537, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    for name in ("codes", "exps", "rows", "width"):           # checked once: not replaced afterwards
        with pytest.raises(AttributeError):
            setattr(r, name, r.codes)
