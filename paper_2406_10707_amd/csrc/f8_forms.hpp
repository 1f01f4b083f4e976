// Which form a product of two 8-bit matrices with a scale for each block of 128 takes, by its sizes alone (host only).
#pragma once
#include <stdint.h>

namespace dsllm {

// A form's tile, how many of its blocks share a compute unit, and what it costs, about microseconds, fitted to 1500 times of 32 products from 300 x 2050 x 768 to 8192^3: a step of 128 values of K with blocks on every unit (and in
// every round but the last) or, of forms whose blocks share a unit, with one on it; what a block takes besides, with C in bf16 or in f32 (as which f16 counts). Steps for the two kinds of sums (8-bit instructions, bf16) and of B's scales (of 128 x 128,
// of single rows). The choice is in the mean 1 % over the best
// form, at most 8 %.
struct F8Form {
    const char *name;
    uint32_t bm, bn, together;
    double step[4][2], block[2];      // [2 wide + rows]: of the last round with up to one block a unit, of others
    uint64_t tiles(uint64_t m, uint64_t n) const { return (m + bm - 1) / bm * ((n + bn - 1) / bn); }
};
// Sums of the 8-bit instructions with scales of single rows do not fit the registers of a 64 x 128 wave (they spill: 8192^3 650 us, with 256 x 128 tiles 555).
constexpr double kF8Never = 1e9;
constexpr F8Form kF8Forms[] = {
    {"256x256", 256, 256, 1, {{1.13, 1.56}, {kF8Never, kF8Never}, {2.93, 3.34}, {3.26, 3.63}}, {8.9, 9.8}},
    {"256x128", 256, 128, 1, {{0.63, 0.89}, {0.84, 1.09}, {1.47, 1.69}, {1.65, 1.87}}, {5.7, 6.2}},
    {"128x128", 128, 128, 2, {{0.57, 0.96}, {0.63, 1.08}, {1.00, 1.69}, {1.19, 1.86}}, {4.1, 3.9}},
    {"64x64", 64, 64, 2, {{0.22, 0.38}, {0.27, 0.41}, {0.47, 0.65}, {0.52, 0.73}}, {2.8, 2.5}},
};
constexpr int kF8FormCount = sizeof(kF8Forms) / sizeof(kF8Forms[0]);
constexpr bool f8_form_has(int form, bool wide, bool rows) { return kF8Forms[form].step[2 * wide + rows][1] < kF8Never; }
constexpr uint32_t kF8Units = 256;
constexpr double kF8Join = 3.0, kF8JoinSplit = 0.45, kF8JoinBytes = 11.9e6;      // what joining parts of K costs besides, for each part, bytes a unit of cost
constexpr uint64_t kF8MostTiles = 1u << 22;              // of a launch

inline uint32_t f8_steps(uint64_t k) { return uint32_t((k + 127) / 128); }

inline double f8_cost(const F8Form &f, uint64_t m, uint64_t n, uint32_t steps, uint32_t splits, bool wide, bool rows) {
    const uint64_t blocks = f.tiles(m, n) * splits, at_once = kF8Units * f.together, full = blocks / at_once, rest = blocks % at_once;
    const double *step = f.step[2 * wide + rows], block = f.block[wide || splits > 1];
    double t = double(full) * (double(steps) * step[1] + block);
    if (rest) t += double(steps) * step[rest > kF8Units] + block;
    return t;
}

// Parts of K lie one behind the other in the workspace, as f32 rows of whole 16 bytes.
inline uint64_t f8_part_pitch(uint64_t n) { return (n + 3) / 4 * 4; }
inline uint64_t f8_part_bytes(uint64_t m, uint64_t n) { return m * f8_part_pitch(n) * 4; }

// Up to sixteen rows of A have a kernel of their own: its waves for each 16 rows of B. Two where K is up to 4096 and there is a block for every unit, else four: one row with 4096 x 4096 6.7 us (four 7.7), 1024 x 4096 4.2 (two 5.7),
// 4096 x 11008 12.8 (two 14.1, eight 13.0), 28672 x 8192 42.0 (44.5, 43.9); of both halves of the gated block 11008 x 4096 21.1 (22.9), 28672 x 8192 82 (87).
constexpr uint64_t kF8Few = 16;
inline uint32_t f8_few_waves(uint64_t n, uint32_t steps) { return steps <= 32 && n >= 16 * kF8Units ? 2 : 4; }

struct F8Choice { int form; uint32_t splits; };

// The cheapest form and number of parts whose parts fit the workspace. Joining the parts costs another launch and the way of the parts to memory and back.
inline F8Choice f8_choice(uint64_t m, uint64_t n, uint64_t k, bool wide, bool rows, uint64_t workspace) {
    const uint32_t steps = f8_steps(k);
    F8Choice best{-1, 1};
    double least = 0;
    for (int f = 0; f < kF8FormCount; f++)
        for (uint32_t splits = 1; splits <= 16 && f8_form_has(f, wide, rows); splits *= 2) {
            const uint32_t each = (steps + splits - 1) / splits;
            if (splits > 1 && (uint64_t(each) * (splits - 1) >= steps || f8_part_bytes(m, n) > workspace / splits || kF8Forms[f].tiles(m, n) > kF8MostTiles || m * f8_part_pitch(n) >> 33)) break;      // one launch for the tiles, one of 2^31 threads at most that joins them
            double t = f8_cost(kF8Forms[f], m, n, each, splits, wide, rows);
            if (splits > 1) t += kF8Join + kF8JoinSplit * splits + double(f8_part_bytes(m, n)) * (2 * splits + 1) / kF8JoinBytes;
            if (best.form < 0 || t < least) { best = F8Choice{f, splits}; least = t; }
        }
    return best;
}

// The gated block's forward pass: tiles of 256, 128 or 64 tokens by 128 columns of gate and of up, a block a unit, or (kGatedHalves) of 256 with the last round's in halves. By what a round of them costs, about microseconds: 4096 to 11008 columns
// 64 tokens 38 us (60 by tiles of 128, 99 of 256), 256 tokens 65 (78 by 64, 98 by 256), 512 tokens 104 (122, 116), 1024 tokens 163 with halves (204 without, 185 by 128).
constexpr int kGatedHalves = 3;
// 17 to 64 tokens: tiles of 32 columns, whose values a second launch rounds, where they are at least half as many as the units and at most one round of two a unit. 4096 to 11008 columns 30 to 32 us (36 to 37 in one launch), 2048 to 8192 14 to 16 (21 to
// 22), 8192 to 16384 72 to 77 (90), 768 to 4097, the fewest tiles, 12.4 to 13.5 (12.3 to 15); 8192 to 28672, 896 tiles, 127 (113).
inline bool gated_values_first(uint64_t tokens, uint64_t ffn) { return tokens > kF8Few && tokens <= 64 && ffn > 32 * (kF8Units / 2 - 1) && ffn <= 32 * 2 * kF8Units; }
inline int gated_form(uint64_t tokens, uint64_t across, uint32_t steps) {
    constexpr uint64_t rows[] = {256, 128, 64};
    constexpr double step[] = {2.75, 1.62, 0.97}, block[] = {10.6, 7.7, 6.9};
    auto round = [&](int f) { return step[f] * steps + block[f]; };
    int best = 0;
    double least = 0;
    for (int f = 0; f < 3; f++) {
        const double t = double(((tokens + rows[f] - 1) / rows[f] * across + kF8Units - 1) / kF8Units) * round(f);
        if (f == 0 || t < least) { best = f; least = t; }
    }
    const uint64_t count = (tokens + 255) / 256 * across, rest = count % kF8Units;
    return count > kF8Units && rest && 2 * rest <= kF8Units && double(count / kF8Units) * round(0) + round(1) < least ? kGatedHalves : best;
}

}  // namespace dsllm
