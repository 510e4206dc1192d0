"""The plans of the attention's launches, on the host (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_launches_stay_below_the_limit_and_cover_every_tile(tmp_path):
    exe = str(tmp_path / "host_attention_plan_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-host-only", "-Wno-unused-command-line-argument", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-fno-gpu-sanitize",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2412_01034_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host_attention_plan_driver.cpp"), "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "plans: ok" in r.stdout, r.stdout[-4000:]
