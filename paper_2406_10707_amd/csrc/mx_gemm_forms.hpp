// Which form a product of two MXFP4 matrices takes, by its sizes alone (host only).
#pragma once
#include <stdint.h>

namespace dsllm {

// A form's tile, how many of its blocks share a compute unit, and what it costs, fitted to 20 products from 300 x 300 x 300 to 8192^3 so that the forms of each come out in their order (the choice is
// in the mean 0.4 % over the best form, at most 4 %): a step of 256 values of K with 1, 2, 3 blocks on the unit, and what a block takes besides. About microseconds, but no prediction of a time: 8192^3
// is 202 here and takes 226 to 254.
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
constexpr double kJoin = 4.5, kJoinBytes = 5e6;      // what the join costs besides; bytes a unit of cost

// `splits` blocks share a tile, each with a part of K.
inline double mx_gemm_cost(const MxGemmForm &f, uint64_t m, uint64_t n, uint64_t steps, uint32_t splits, bool f32_out) {
    const uint64_t blocks = f.tiles(m, n) * splits, at_once = kComputeUnits * f.together, full = blocks / at_once, rest = blocks % at_once;
    const double block = f.block * (f32_out || splits > 1 ? 1.3 : 1.0);
    double t = double(full) * (double(steps) * f.step[f.together - 1] + block);
    if (rest) t += double(steps) * f.step[(rest + kComputeUnits - 1) / kComputeUnits - 1] + block;
    return t;
}

// Parts of K lie one behind the other in the workspace, as f32 rows of whole 16 bytes; each has a multiple of four steps (a window of scales).
inline uint64_t mx_gemm_part_pitch(uint64_t n) { return (n + 3) / 4 * 4; }
inline uint64_t mx_gemm_part_bytes(uint64_t m, uint64_t n) { return m * mx_gemm_part_pitch(n) * 4; }
inline uint32_t mx_gemm_steps_a_split(uint32_t steps, uint32_t splits) { return ((steps + splits - 1) / splits + 3) / 4 * 4; }

// Up to sixteen rows of A have a kernel of their own: its waves for each 16 rows of B, 0 for other products. Two where K is up to 4096 (11008 x 4096 5.9 us, with four 6.4), else four (16384 x 16384
// 26.2, with two 27.9, with eight 29.5). However few rows B has: 16 x 64 x 16384 4.6 (the tiles in parts of K 9.0), 16 x 256 x 65536 13.1 (12.4), 1 x 16 x 65536 9.9 (10.6); only beyond do parts
// pay (1 x 16 x 262144 33.7, in parts 17.8).
inline uint32_t mx_gemm_few_waves(uint64_t m, uint32_t steps) { return m > 16 ? 0 : steps <= 16 ? 2 : 4; }

struct MxGemmChoice { int form; uint32_t splits; };

// The cheapest form and number of parts whose grid has fewer than 2^32 work-items and whose parts fit the workspace; form -1 if there is none. Joining the parts costs another launch and
// the way of the parts to memory and back.
inline MxGemmChoice mx_gemm_choice(uint64_t m, uint64_t n, uint64_t k, bool f32_out, uint64_t workspace) {
    const uint32_t steps = uint32_t((k + 255) / 256);
    MxGemmChoice best{-1, 1};
    double least = 0;
    for (int f = 0; f < kMxGemmFormCount; f++)
        for (uint32_t splits = 1; splits <= 16; splits *= 2) {
            const uint32_t each = mx_gemm_steps_a_split(steps, splits);
            if (splits > 1 && (uint64_t(each) * (splits - 1) >= steps || mx_gemm_part_bytes(m, n) > workspace / splits)) break;
            if (kMxGemmForms[f].tiles(m, n) * splits >= 1u << 24) break;
            double t = mx_gemm_cost(kMxGemmForms[f], m, n, splits > 1 ? each : steps, splits, f32_out);
            if (splits > 1) t += kJoin + double(mx_gemm_part_bytes(m, n)) * (2 * splits + 1) / kJoinBytes;
            if (best.form < 0 || t < least) { best = MxGemmChoice{f, splits}; least = t; }
        }
    return best;
}

}  // namespace dsllm
