// Which form a product of two MXFP4 matrices takes, by its sizes alone (host only).
#pragma once
#include <stdint.h>

namespace dsllm {

// A form's tile, how many of its blocks share a compute unit, and what it costs in us, fitted to 20 products from 1 x 11008 x 4096 to 8192^3 (mean 0.4 % over the
// best form of each, at most 4 %): a step of 256 values of K with 1, 2, 3 blocks on the unit, and what a block takes besides.
struct MxGemmForm {
    const char *name;
    uint32_t bm, bn, together;
    double step[3], block;
    uint64_t tiles(uint64_t m, uint64_t n) const { return (m + bm - 1) / bm * ((n + bn - 1) / bn); }
};
// What bounds a step: with 256 x 256 the matrix instructions and the power (1.73 GHz at 77 % of their cycles), with the others the panels' way into LDS, some 85 GB/s a unit; so
// large tiles are better wherever there are enough of them.
constexpr MxGemmForm kMxGemmForms[] = {
    {"256x256", 256, 256, 1, {1.3, 0, 0}, 9.0},
    {"192x192", 192, 192, 1, {0.82, 0, 0}, 6.5},
    {"128x128", 128, 128, 2, {0.5, 1.0, 0}, 4.2},
    {"64x128", 64, 128, 2, {0.37, 0.70, 0}, 3.0},
    {"64x64 four stages", 64, 64, 2, {0.22, 0.42, 0}, 2.4},
    {"64x64 two stages", 64, 64, 3, {0.37, 0.44, 0.58}, 2.4},
};
constexpr int kMxGemmFormCount = sizeof(kMxGemmForms) / sizeof(kMxGemmForms[0]);
constexpr uint32_t kComputeUnits = 256;

inline double mx_gemm_cost(const MxGemmForm &f, uint64_t m, uint64_t n, uint64_t k, bool f32_out) {
    const uint64_t tiles = f.tiles(m, n), at_once = kComputeUnits * f.together, full = tiles / at_once, rest = tiles % at_once;
    const double steps = double((k + 255) / 256), block = f.block * (f32_out ? 1.3 : 1.0);
    double t = double(full) * (steps * f.step[f.together - 1] + block);
    if (rest) t += steps * f.step[(rest + kComputeUnits - 1) / kComputeUnits - 1] + block;
    return t;
}

// The cheapest whose grid has fewer than 2^32 work-items; -1 if there is none.
inline int mx_gemm_form(uint64_t m, uint64_t n, uint64_t k, bool f32_out) {
    int best = -1;
    double least = 0;
    for (int f = 0; f < kMxGemmFormCount; f++) {
        if (kMxGemmForms[f].tiles(m, n) >= 1u << 24) continue;
        const double t = mx_gemm_cost(kMxGemmForms[f], m, n, k, f32_out);
        if (best < 0 || t < least) { best = f; least = t; }
    }
    return best;
}

}  // namespace dsllm
