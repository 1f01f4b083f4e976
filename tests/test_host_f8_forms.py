"""Which form a product of 8-bit matrices takes (csrc/f8_forms.hpp), asked on the CPU: the shapes that the GPU tests name for each form do take it, and parts of K cover it."""
import os
import subprocess

import pytest

from tests.test_gpu_f8_gemm import FORMS, PARTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "%s/paper_2406_10707_amd/csrc/f8_forms.hpp"
using namespace dsllm;
int main(int argc, char **argv) {
    const uint64_t m = atoll(argv[1]), n = atoll(argv[2]), k = atoll(argv[3]), ws = strtoull(argv[6], nullptr, 10);
    const F8Choice c = f8_choice(m, n, k, atoi(argv[4]), atoi(argv[5]), ws);
    const uint32_t steps = f8_steps(k), each = (steps + c.splits - 1) / c.splits;
    printf("%%s %%u %%d\n", kF8Forms[c.form].name, c.splits, uint64_t(each) * (c.splits - 1) < steps && f8_part_bytes(m, n) * (c.splits > 1 ? c.splits : 0) <= ws);
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("f8_forms")
    (d / "ask.cpp").write_text(PROGRAM % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "ask"), str(d / "ask.cpp")], check=True)

    def call(m, n, k, wide, rows, workspace):
        name, splits, fine = subprocess.run([str(d / "ask")] + [str(int(v)) for v in (m, n, k, wide, rows, workspace)], check=True, capture_output=True, text=True).stdout.split()
        assert fine == "1"
        return name, int(splits)
    return call


def test_every_form_has_shapes(ask):
    for form, shapes in FORMS.items():
        for m, n, k in shapes:
            for wide, rows in ((False, False), (True, False), (True, True), (False, True)):
                taken = ask(m, n, k, wide, rows, 0)
                if (wide, rows) == (False, False):
                    assert taken == (form, 1), (m, n, k, taken)
                assert (wide, rows) != (False, True) or taken[0] != "256x256"
    for wide, rows, shape, form in ((True, False, (8192, 8192, 8192), "256x256"), (False, True, (2048, 2560, 1024), "256x128"), (True, True, (8192, 8192, 8192), "256x256"), (True, False, (2048, 2560, 1024), "128x128")):
        assert ask(*shape, wide, rows, 0)[0] == form, (shape, wide, rows)


def test_parts(ask):
    for m, n, k in PARTS:
        assert ask(m, n, k, False, False, 2 ** 64 - 1)[1] > 1
    for m, n, k in [(17, 17, 200), (4096, 4096, 4096), (20, 1 << 30, 128), ((1 << 31) - 1, (1 << 31) - 1, 128), (100, 100, 1 << 23)]:
        for wide in (False, True):
            for rows in (False, True):
                ask(m, n, k, wide, rows, 2 ** 64 - 1)
                assert ask(m, n, k, wide, rows, 0)[1] == 1
