"""The orthogonalising call's host side on the CPU, under AddressSanitizer and UBSan: lists
of workgroups that cover every product once and stay inside the workspace."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1910_00643_amd", "csrc")


def test_lists_of_tiles(tmp_path):
    exe = str(tmp_path / "orth_plan")
    cmd = ["g++", "-O1", "-g", "-std=c++17", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-static-libasan", "-D__HIP_PLATFORM_AMD__", "-D_Float16=short", "-I/opt/rocm/include", "-I", CSRC, "-o", exe,
           os.path.join(ROOT, "tests", "orth_plan_driver.cpp")]
    build = subprocess.run(cmd, capture_output=True, text=True)
    if build.returncode != 0 and "asan" in (build.stderr + build.stdout).lower():
        pytest.skip("this toolchain has no static AddressSanitizer runtime")
    assert build.returncode == 0, build.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split()[-1] == "ok", r.stdout + r.stderr
