"""Which form the MXFP4 product takes (csrc/mx_gemm_forms.hpp), asked on the CPU: every form is some size's, grids count in 32 bits, and a form is
never far from the cheapest of the fitted costs."""
import os
import subprocess

import pytest

from tests.test_gpu_train_gemm import FORMS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = """#include <cstdio>
#include "mx_gemm_forms.hpp"
int main() {
    unsigned long long m, n, k, f32, ws;
    while (scanf("%llu %llu %llu %llu %llu", &m, &n, &k, &f32, &ws) == 5) {
        const dsllm::MxGemmChoice c = dsllm::mx_gemm_choice(m, n, k, f32, ws);
        if (c.form < 0) { printf("none,0,0\\n"); continue; }
        printf("%s,%llu,%u\\n", dsllm::kMxGemmForms[c.form].name, (unsigned long long)dsllm::kMxGemmForms[c.form].tiles(m, n), c.splits);
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("mxforms")
    (d / "main.cpp").write_text(MAIN)
    exe = str(d / "forms")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2406_10707_amd", "csrc"), "-o", exe, str(d / "main.cpp")], check=True)

    def f(shapes):
        out = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % (*s, 1 << 40)[:5] for s in shapes), capture_output=True, text=True, check=True).stdout
        return [(name, int(tiles), int(splits)) for name, tiles, splits in (x.rsplit(",", 2) for x in out.splitlines())]

    return f


def test_every_form_is_some_sizes(ask):
    sizes = [(8192, 8192, 8192, 0), (2048, 4096, 11008, 0), (2048, 2048, 2048, 0), (2304, 768, 8190, 1), (40, 11008, 4096, 0), (1000, 2304, 768, 0)]
    assert [name for name, _, _ in ask(sizes)] == ["256x256", "192x192", "128x128", "64x128", "64x64 four stages", "64x64 two stages"]


def test_the_forms_that_the_gpu_tests_stand_for(ask):
    for name, shapes in FORMS.items():
        for shape in shapes:
            assert [x[0] for x in ask([(*shape, 0, 0), (*shape, 1, 0)])] == [name] * 2, (name, shape)


def test_grids_count_in_32_bits(ask):
    shapes = [(m, n, k, 1) for m in (1, 65, 1 << 20, (1 << 31) - 1) for n in (1, 64, 1 << 12, 1 << 16) for k in (1, 8192) if m * n <= 1 << 37]
    for shape, (name, tiles, splits) in zip(shapes, ask(shapes)):
        assert name != "none" and tiles * splits * 256 < 1 << 32, (shape, name)


def test_long_axes_of_few_tiles_are_split_if_there_is_room(ask):
    shapes = [(64, 512, 16384, 0), (17, 64, 16384, 1), (30, 4096, 16384, 0)]
    for shape, (_, tiles, splits) in zip(shapes, ask(shapes)):
        m, n, k, _ = shape
        steps = -(-k // 256)
        each = -(-(-(-steps // splits)) // 4) * 4
        assert splits > 1 and each * (splits - 1) < steps, (shape, splits)      # no part without steps
        need = splits * m * n * 4
        assert ask([(*shape, need)])[0][2] == splits and ask([(*shape, need - 1)])[0][2] < splits and ask([(*shape, 0)])[0][2] == 1
