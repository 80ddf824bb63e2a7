"""The rules that keep the adapters' and the 8-bit activations' kernels inside their buffers, walked on the CPU (no GPU) under
UndefinedBehaviorSanitizer: the header functions that launchers and kernels call.  And plans of transposed weights under both sanitizers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rules_keep_the_kernels_in_bounds(tmp_path):
    exe = str(tmp_path / "adapter_rules")
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2206_10620_amd", "csrc"),
           os.path.join(ROOT, "tests", "host_adapter_rules_main.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.stdout[-2000:], r.stderr[-2000:])


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_transposed_plans_run_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "transposed")
    csrc = os.path.join(ROOT, "paper_2206_10620_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "host_transposed_main.cpp"), os.path.join(csrc, "block_plan.cpp"),
           os.path.join(csrc, "plan.cpp"), "-pthread", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok "), (r.stdout[-2000:], r.stderr[-4000:])
