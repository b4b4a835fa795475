"""CPU check of the attention's plan over the sizes that its entry point lets
through: grids that a launch holds, ranges that cover the keys, stages that fit
the workspace (host code only, built with UndefinedBehaviorSanitizer)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_plans_fit_every_size(tmp_path):
    exe = str(tmp_path / "attn_plan")
    cmd = ["g++", "-std=c++17", "-O2", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "paper_2607_13332_amd", "csrc"),
           os.path.join(ROOT, "tests", "asan", "attn_plan_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "attention plans ok" in r.stdout
