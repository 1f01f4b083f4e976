"""Every product of 8-bit matrices takes a form that has a kernel (csrc/f8_forms.hpp), whatever the sizes, nothing to contract over among them."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "%s/paper_2406_10707_amd/csrc/f8_forms.hpp"
using namespace dsllm;
int main() {
    static_assert(!f8_form_has(0, false, true) && f8_form_has(0, true, true) && f8_form_has(1, false, true), "256 x 256 tiles of 8-bit sums with scales of single rows are the ones that there are not");
    std::mt19937_64 rng(1);
    auto size = [&](double most) { return uint64_t(std::exp(std::uniform_real_distribution<>(0, std::log(most))(rng))); };
    for (int turn = 0; turn < 300000; turn++) {
        const uint64_t m = size(2147483647.0), n = size(turn %% 2 ? 2147483647.0 : 70000.0), k = turn %% 3 ? size(1 << 23) : 0, workspace = turn %% 5 ? UINT64_MAX : size(1e9);
        for (int kind = 0; kind < 4; kind++) {
            const F8Choice c = f8_choice(m, n, k, kind & 1, kind >> 1, workspace);
            if (c.form < 0 || c.form >= kF8FormCount || !f8_form_has(c.form, kind & 1, kind >> 1) || c.splits < 1) {
                printf("%%llu x %%llu x %%llu, kind %%d: form %%d\n", (unsigned long long)m, (unsigned long long)n, (unsigned long long)k, kind, c.form);
                return 1;
            }
        }
    }
    printf("ok\n");
}
"""


def test_every_choice_has_a_kernel(tmp_path):
    (tmp_path / "choices.cpp").write_text("#include <cmath>\n" + PROGRAM % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O2", "-o", str(tmp_path / "choices"), str(tmp_path / "choices.cpp")], check=True)
    r = subprocess.run([str(tmp_path / "choices")], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
