"""The host side of the training operators (tests/emu/train_calls.cpp): their sources, compiled for the host alone, on a runtime of the test's own that records calls and launches."""
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
    d = tmp_path_factory.mktemp("train_calls")
    objects = []
    for f in [os.path.join(build.CSRC, f) for f in ("optim.hip", "mx_quantize.hip", "mx_gemm.hip")] + [os.path.join(ROOT, "tests", "emu", "train_calls.cpp")]:
        objects.append(str(d / (os.path.basename(f) + ".o")))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-c", f, "-o", objects[-1]] + build.HIPCC_FLAGS, check=True, capture_output=True)
    exe = str(d / "train_calls")
    # the device code that the objects would register is not there, and not asked for
    subprocess.run(["g++", "-no-pie", "-Wl,--unresolved-symbols=ignore-all", "-o", exe] + objects, check=True)
    return exe


@pytest.mark.parametrize("what", ["destroy", "grids"])
def test_calls(program, what):
    r = subprocess.run([program, what], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout + r.stderr
