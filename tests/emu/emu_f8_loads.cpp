// Every load of the 8-bit products' kernels, with the loaders' own arithmetic, lane by lane on the CPU: all bytes lie inside the operand's arrays and inside what a descriptor names, go to the wave's own part of LDS, and
// every place of a stage gets the row, the sixteen bytes and the scale that the kernels read there. Prints the number of loads, or the first one that is wrong.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <utility>

using std::min;

struct Descriptor { const unsigned char *base; unsigned records; };
#define __amdgpu_buffer_rsrc_t Descriptor
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, records, flags) Descriptor{p, records}
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, to, bytes, voffset, soffset, imm, aux) buffer_loaded(rsrc, (unsigned char *)(to), bytes, voffset, soffset)
#define __builtin_amdgcn_global_load_lds(from, to, bytes, offset, aux) loaded((const unsigned char *)(from), (unsigned char *)(to), bytes)
void buffer_loaded(const Descriptor &from, const unsigned char *to, unsigned bytes, unsigned voffset, unsigned soffset);
void loaded(const unsigned char *from, const unsigned char *to, unsigned bytes);

#include "../../paper_2406_10707_amd/csrc/f8_loader.hpp"

ssize_t emu_pwrite(int fd, const void *buf, size_t n, off_t off) { return pwrite64(fd, buf, n, off); }

using namespace dsllm;

namespace {

unsigned long long count;
unsigned char lds[160 << 10];
struct Array { uint64_t base, bytes; } codes[3], scales[3];      // of A, B and the second B, at made-up addresses, far from one another: nothing is read
uint32_t lds_first, lds_end, lane_of_load;
std::map<uint32_t, uint64_t> landed;      // where in LDS, from where
char what[200];

void fail(const char *why) {
    printf("%s: %s\n", what, why);
    exit(1);
}

}  // namespace

void loaded(const unsigned char *from, const unsigned char *to, unsigned bytes) {
    count++;
    const uint64_t at = uint64_t(from);
    bool inside = false;
    for (int i = 0; i < 3; i++)
        for (const Array &a : {codes[i], scales[i]}) inside |= at >= a.base && at + bytes <= a.base + a.bytes;
    if (!inside) fail("outside the operands");
    const uint64_t place = to - lds + uint64_t(lane_of_load) * bytes;      // LDS is written in lane order
    if (to < lds || uint64_t(to - lds) < lds_first || uint64_t(to - lds) + 64 * bytes > lds_end) fail("outside LDS");
    landed[uint32_t(place)] = at;
}
void buffer_loaded(const Descriptor &from, const unsigned char *to, unsigned bytes, unsigned voffset, unsigned soffset) {
    if (uint64_t(voffset) + soffset + bytes > from.records) fail("outside the descriptor");
    loaded(from.base + uint64_t(voffset) + soffset, to, bytes);
}

namespace {

F8Side side(int i, uint64_t rows, uint64_t k, uint64_t wider, uint32_t shift) {
    F8Side s{};
    s.pitch = (k + 127) / 128 * 128 + 16 * wider;
    s.scale_pitch = (rows + (1u << shift) - 1 >> shift) + wider;
    s.rows = int64_t(rows);
    s.shift = shift;
    codes[i] = Array{uint64_t(2 * i + 1) << 44, (rows - 1) * s.pitch + (k + 127) / 128 * 128};
    scales[i] = Array{uint64_t(2 * i + 2) << 44, 4 * (((k + 127) / 128 - 1) * s.scale_pitch + (rows + (1u << shift) - 1 >> shift))};
    s.codes = reinterpret_cast<const uint8_t *>(codes[i].base);
    s.scales = reinterpret_cast<const float *>(scales[i].base);
    return s;
}

uint64_t code_at(const F8Side &s, int64_t row, uint32_t step, int piece) { return uint64_t(s.codes) + min(row, s.rows - 1) * s.pitch + 128ull * step + 16 * piece; }
uint64_t scale_at(const F8Side &s, int64_t row, uint32_t step) { return uint64_t(s.scales) + 4 * (step * s.scale_pitch + (min(row, s.rows - 1) >> s.shift)); }

template <class S>
void tile(const F8Side &a, const F8Side &b, const F8Side &b2, uint32_t steps, int64_t row, int64_t col) {
    for (uint32_t step = 0; step < steps; step++) {
        if (step >= 2 && step + 2 < steps) continue;      // the middle is like its neighbours
        landed.clear();
        lds_first = 0;
        lds_end = S::STAGE;
        for (uint32_t wave = 0; wave < S::NW; wave++)
            for (lane_of_load = 0; lane_of_load < 64; lane_of_load++) {
                const F8Loader<S> load(a, b, b2, steps, row, col, lane_of_load, wave);
                load.issue(lds, step);
            }
        // as f8_sums reads them
        for (int lane = 0; lane < 64; lane++) {
            const int q = lane >> 4, ar = lane & 15, swizzle = f8_rotated((ar >> 1) & 7);
            for (int wm = 0; wm < S::WM; wm++)
                for (int i = 0; i < S::TM; i++) {
                    const int64_t r = row + 16 * S::TM * wm + S::TM * ar + i;
                    for (int h = 0; h < 2; h++)
                        if (landed[wm * S::TM * 2048 + 2048 * i + ar * 128 + 16 * ((2 * q + h) ^ swizzle)] != code_at(a, r, step, 2 * q + h)) fail("A's codes");
                    if (landed[S::CODES + 4 * (16 * S::TM * wm + S::TM * ar + i)] != scale_at(a, r, step)) fail("A's scales");
                }
            for (int wn = 0; wn < S::WN; wn++)
                for (int j = 0; j < S::TN; j++) {
                    const int group = 16 * S::TN * wn + 16 * S::TNG * (j / S::TNG);
                    auto expected = [&](int in_group, const F8Side **of) {      // the row of B that is column `in_group` of a lane's group
                        const int n = group + in_group;
                        *of = S::PAIR && (n / (16 * S::TNG)) % 2 ? &b2 : &b;
                        return col + (S::PAIR ? n / (32 * S::TNG) * (16 * S::TNG) + n % (16 * S::TNG) : n);
                    };
                    const F8Side *of;
                    const int64_t r = expected(4 * S::TNG * (ar / 4) + 4 * (j % S::TNG) + ar % 4, &of);      // what the instruction gives to e = ar % 4 of the lanes with q = ar / 4
                    for (int h = 0; h < 2; h++)
                        if (landed[S::BM * 128 + wn * S::TN * 2048 + 2048 * j + ar * 128 + 16 * ((2 * q + h) ^ swizzle)] != code_at(*of, r, step, 2 * q + h)) fail("B's codes");
                    for (int e = 0; e < 4; e++) {
                        const int64_t c = expected(4 * S::TNG * q + 4 * (j % S::TNG) + e, &of);
                        if (landed[S::CODES + 4 * (S::BM + group + 4 * S::TNG * q + 4 * (j % S::TNG) + e)] != scale_at(*of, c, step)) fail("B's scales");
                    }
                    // one scale for a group where blocks have 128 rows
                    if (b.shift && landed[S::CODES + 4 * (S::BM + group)] != scale_at(*of, expected(4 * S::TNG * q + 4 * (j % S::TNG) + 3, &of), step)) fail("B's scale of a group");
                }
        }
    }
}

template <class S>
void tiles(const char *name) {
    const uint64_t sizes[][3] = {{1, 1, 1}, {1, 300, 128}, {17, 200, 129}, {256, 256, 256}, {257, 511, 1000}, {100, 129, 4096}, {300, 65, 8000}, {40, 1000, 300}};
    for (const auto &s : sizes)
        for (uint32_t shifts = 0; shifts < 4; shifts++)
            for (uint64_t wider : {0, 3}) {
                const uint64_t n = S::PAIR ? (s[1] + 1) / 2 : s[1];
                snprintf(what, sizeof what, "%s %llu x %llu x %llu shifts %u wider %llu", name, (unsigned long long)s[0], (unsigned long long)n, (unsigned long long)s[2], shifts, (unsigned long long)wider);
                const F8Side a = side(0, s[0], s[2], wider, 7 * (shifts & 1)), b = side(1, n, s[2], wider, 7 * (shifts >> 1)), b2 = side(2, n, s[2], 2 * wider, 7 * (shifts >> 1));
                for (int64_t row = 0; row < a.rows; row += S::BM)
                    for (int64_t col = 0; col < b.rows; col += S::PAIR ? S::BN / 2 : S::BN) tile<S>(a, b, b2, uint32_t((s[2] + 127) / 128), row, col);
            }
    // the longest rows that are allowed
    snprintf(what, sizeof what, "%s, rows of 2^23", name);
    const F8Side a = side(0, 300, 1 << 23, 0, 0), b = side(1, 300, 1 << 23, 0, 7), b2 = side(2, 300, 1 << 23, 0, 7);
    tile<S>(a, b, b2, 1 << 16, 0, 0);
    tile<S>(a, b, b2, 1 << 16, 256 / S::BM * S::BM, 256);
}

template <int MATRICES, bool EIGHT>
void few() {
    typedef F8FewLoader<MATRICES, EIGHT> L;
    for (uint64_t m : {1, 2, 7, EIGHT ? 8 : 16})
        for (uint64_t n : {1, 5, 16, 17, 300})
            for (uint64_t k : {1, 128, 129, 512, 1300, 5000})
                for (uint32_t shift : {0, 7}) {
                    snprintf(what, sizeof what, "few %llu x %llu x %llu", (unsigned long long)m, (unsigned long long)n, (unsigned long long)k);
                    const F8Side a = side(0, m, k, 0, 0), b = side(1, n, k, 1, shift), b2 = side(2, n, k, 2, shift);
                    const uint32_t steps = uint32_t((k + 127) / 128);
                    for (int64_t n0 = 0; n0 < b.rows; n0 += 16)
                        for (uint32_t window = 0; window < (steps + 3) / 4; window++) {
                            landed.clear();
                            for (lane_of_load = 0; lane_of_load < 64; lane_of_load++) {
                                const L load(a, b, b2, steps, n0, lane_of_load);
                                lds_first = 4 * L::STEP + (window & 1) * L::SCALES;
                                lds_end = lds_first + L::SCALES;
                                load.issue_scales(lds, window, window);
                                for (int s = 0; s < 4; s++) {
                                    lds_first = s * L::STEP;
                                    lds_end = lds_first + L::STEP;
                                    load.issue_step(lds, window, s);
                                }
                            }
                            for (uint32_t s = 0; s < 4 && 4 * window + s < steps; s++)
                                for (int x = 0; x < L::SIDES; x++)
                                    for (int r = 0; r < 16; r++) {
                                        const bool held = x || !EIGHT || r < 8;
                                        const F8Side &of = x == 0 ? a : x == 1 ? b : b2;
                                        const int64_t row = (x ? n0 : 0) + r;
                                        for (int piece = 0; piece < 8; piece++)
                                            if (held && landed[s * L::STEP + (x ? L::A_PLACES + 2048 * (x - 1) : 0) + 128 * r + 16 * (piece ^ f8_rotated((r >> 1) & 7))] != code_at(of, row, 4 * window + s, piece)) fail("codes");
                                        if (landed[4 * L::STEP + (window & 1) * L::SCALES + 4 * (16 * L::SIDES * s + 16 * x + r)] != scale_at(of, row, 4 * window + s)) fail("scales");
                                    }
                        }
                }
}

}  // namespace

int main() {
    tiles<F8Shape<4, 2, 4, 8, 4, 2, false>>("256x256");
    tiles<F8Shape<2, 2, 4, 4, 4, 2, false>>("128x128");
    tiles<F8Shape<2, 2, 2, 2, 2, 4, false>>("64x64");
    tiles<F8Shape<4, 2, 4, 8, 4, 2, true>>("pair 256x256");
    tiles<F8Shape<4, 2, 2, 8, 4, 2, true>>("pair 128x256");
    tiles<F8Shape<2, 4, 2, 4, 2, 2, true>>("pair 64x256");
    tiles<F8Shape<2, 2, 2, 2, 1, 4, true>>("pair 64x64");
    few<1, false>();
    few<1, true>();
    few<2, false>();
    few<2, true>();
    printf("ok %llu loads\n", count);
}
