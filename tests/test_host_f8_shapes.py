"""Every load of every tile that the 8-bit products and the gated block are made of (tests/emu/emu_f8_shapes.cpp): the shapes come from the list that the kernels take them from, so that none is left out."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


def test_every_load_of_every_tile(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("ROCm clang not present")
    exe = str(tmp_path / "emu_f8_shapes")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O2", "-pthread", "-I", os.path.join(ROOT, "tests", "emu"), "-o", exe, os.path.join(ROOT, "tests", "emu", "emu_f8_shapes.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-2000:] + r.stderr[-2000:]
