"""Every load of the 8-bit products' kernels (tests/emu/emu_f8_loads.cpp, with the loaders' own arithmetic): inside the operands' arrays, and every place of LDS gets what the kernels read there, for all tile
shapes, short and long K, ragged last tiles, both kinds of blocks, pitches from the smallest to the largest."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


def test_every_load_is_the_right_one(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("ROCm clang not present")
    exe = str(tmp_path / "emu_f8_loads")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O2", "-pthread", "-I", os.path.join(ROOT, "tests", "emu"), "-o", exe, os.path.join(ROOT, "tests", "emu", "emu_f8_loads.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-2000:] + r.stderr[-2000:]
