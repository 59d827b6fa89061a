"""The workspace of a learning context (csrc/learn.cpp) with the HIP runtime
replaced by counters: what a recorded graph uses stays allocated."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_graphs_workspace_stays(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime.h")):
        pytest.skip("g++ and the HIP headers")
    exe = str(tmp_path / "learn_workspace")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-o", exe,
                    os.path.join(ROOT, "tests", "learn_workspace.cpp"),
                    os.path.join(ROOT, "paper_2608_16329_amd", "csrc", "learn.cpp")], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and not res.stdout, res.stdout
