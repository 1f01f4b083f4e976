"""The training operators under PyTorch: its memory, a side stream, a captured graph whose replays equal eager calls. In a process of its own, as PyTorch has to be imported before
the library."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_replays_equal_eager_calls():
    print("captured training operators (subprocess)", flush=True)
    env = dict(os.environ, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "train_graph_main.py")], capture_output=True, text=True, timeout=300, cwd=ROOT, env=env)
    assert r.returncode == 0 and "train graph ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
