"""Every address that the MXFP4 product's tile kernels load from (tests/emu/emu_mx_loads.cpp, with the loader's own arithmetic): inside the operands' arrays, for all six forms, short
and long K, ragged last tiles, pitches from the smallest to the largest, parts of K."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


def test_no_load_leaves_its_array(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("ROCm clang not present")
    exe = str(tmp_path / "emu_mx_loads")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O2", "-pthread", "-I", os.path.join(ROOT, "tests", "emu"), "-o", exe, os.path.join(ROOT, "tests", "emu", "emu_mx_loads.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-2000:] + r.stderr[-2000:]
