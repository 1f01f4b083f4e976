"""Matrices of one call of the 8-bit operators that share memory (tests/emu/f8_overlaps.cpp): what is written may share nothing with anything else, codes, scales and workspace alike."""
import os
import shutil
import subprocess

import pytest

from paper_2406_10707_amd import build
from tests.test_host_gemm_fence import HIPCC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not shutil.which(HIPCC):
        pytest.skip("hipcc not present")
    d = tmp_path_factory.mktemp("f8_overlaps")
    objects = []
    for f in [os.path.join(build.CSRC, f) for f in ("f8_quantize.hip", "f8_gemm.hip", "f8_gated.hip")] + [os.path.join(ROOT, "tests", "emu", "f8_overlaps.cpp")]:
        objects.append(str(d / (os.path.basename(f) + ".o")))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-c", f, "-o", objects[-1]] + build.HIPCC_FLAGS, check=True, capture_output=True)
    exe = str(d / "f8_overlaps")
    # the device code that the objects would register is not there, and not asked for
    subprocess.run(["g++", "-no-pie", "-Wl,--unresolved-symbols=ignore-all", "-o", exe] + objects, check=True)
    return exe


@pytest.mark.parametrize("what", ["calls", "rows", "marked"])
def test_overlaps(program, what):
    r = subprocess.run([program, what], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout[-3000:] + r.stderr
