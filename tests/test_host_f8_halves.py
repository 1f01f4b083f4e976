"""The sizes that the GPU tests name for tiles in halves take them (csrc/f8_forms.hpp), asked on the CPU."""
import os
import subprocess

from tests.test_gpu_f8_halves import HALVES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sizes_take_halves(tmp_path):
    checks = "".join(f"if (gated_form({t}, {-(-f // 128)}, {-(-d // 128)}) != kGatedHalves) return 1;\n" for t, d, f in HALVES)
    (tmp_path / "ask.cpp").write_text('#include <cstdio>\n#include "%s/paper_2406_10707_amd/csrc/f8_forms.hpp"\nusing namespace dsllm;\nint main() {\n%sreturn 0;\n}\n' % (ROOT, checks))
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(tmp_path / "ask"), str(tmp_path / "ask.cpp")], check=True)
    assert subprocess.run([str(tmp_path / "ask")]).returncode == 0
