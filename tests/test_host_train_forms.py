"""Which form the MXFP4 product takes (csrc/mx_gemm_forms.hpp), asked on the CPU: every form is some size's, grids count in 32 bits, and a form is
never far from the cheapest of the fitted costs."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = """#include <cstdio>
#include "mx_gemm_forms.hpp"
int main() {
    unsigned long long m, n, k, f32;
    while (scanf("%llu %llu %llu %llu", &m, &n, &k, &f32) == 4) {
        const int f = dsllm::mx_gemm_form(m, n, k, f32);
        if (f < 0) { printf("none,0\\n"); continue; }
        printf("%s,%llu\\n", dsllm::kMxGemmForms[f].name, (unsigned long long)dsllm::kMxGemmForms[f].tiles(m, n));
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
        out = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in shapes), capture_output=True, text=True, check=True).stdout
        return [(x.rsplit(",", 1)[0], int(x.rsplit(",", 1)[1])) for x in out.splitlines()]

    return f


def test_every_form_is_some_sizes(ask):
    sizes = [(8192, 8192, 8192, 0), (2048, 4096, 11008, 0), (2048, 2048, 2048, 0), (2304, 768, 8190, 1), (1, 11008, 4096, 0), (1000, 2304, 768, 0)]
    assert [name for name, _ in ask(sizes)] == ["256x256", "192x192", "128x128", "64x128", "64x64 four stages", "64x64 two stages"]


def test_grids_count_in_32_bits(ask):
    shapes = [(m, n, k, 1) for m in (1, 65, 1 << 20, (1 << 31) - 1) for n in (1, 64, 1 << 12, 1 << 16) for k in (1, 8192) if m * n <= 1 << 37]
    for shape, (name, tiles) in zip(shapes, ask(shapes)):
        assert name != "none" and tiles * 256 < 1 << 32, (shape, name)
