"""The operators with 8-bit matrices under PyTorch: its memory, side streams, a captured graph whose replays equal eager calls, two steps on two streams. In a process of its own, as PyTorch has to be imported before the library."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_replays_and_streams_equal_eager_calls():
    print("captured 8-bit operators (subprocess)", flush=True)
    env = dict(os.environ, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "f8_graph_main.py")], capture_output=True, text=True, timeout=300, cwd=ROOT, env=env)
    assert r.returncode == 0 and "f8 graph ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
