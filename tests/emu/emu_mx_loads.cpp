// Every load of the MXFP4 product's tile kernels, with the loader's own arithmetic, lane by lane on the CPU: all sixteen bytes lie inside the operand's array and inside what the
// descriptor names, whatever the descriptor's own check makes of the scalar offset, and go to the block's own LDS. Prints the number of loads, or the first one that does not.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <utility>

using std::min;

struct Descriptor { const unsigned char *base; unsigned records; };
#define __amdgpu_buffer_rsrc_t Descriptor
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, records, flags) Descriptor{p, records}
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, to, bytes, voffset, soffset, imm, aux) loaded(rsrc, (unsigned char *)(to), bytes, voffset, soffset)
void loaded(const Descriptor &from, const unsigned char *to, unsigned bytes, unsigned voffset, unsigned soffset);

#include "../../paper_2406_10707_amd/csrc/mx_gemm_loader.hpp"

ssize_t emu_pwrite(int fd, const void *buf, size_t n, off_t off) { return pwrite64(fd, buf, n, off); }

using namespace dsllm;

namespace {

unsigned long long count;
unsigned char lds[160 << 10];
struct Array { const uint8_t *base; uint64_t bytes; } arrays[4];      // at made-up addresses, far from one another: nothing is read
uint32_t lds_bytes;
char what[200];

}  // namespace

void loaded(const Descriptor &from, const unsigned char *to, unsigned bytes, unsigned voffset, unsigned soffset) {
    count++;
    const uint64_t at = uint64_t(voffset) + soffset;
    bool inside = at + bytes <= from.records && to >= lds && uint64_t(to - lds) + 64 * bytes <= lds_bytes;
    bool of_one = false;
    for (const Array &a : arrays) of_one |= from.base >= a.base && from.base + at + bytes <= a.base + a.bytes;
    if (inside && of_one) return;
    printf("%s: offset %llu + %u of a descriptor of %u bytes\n", what, (unsigned long long)at, bytes, from.records);
    exit(1);
}

namespace {

template <int BM, int BN, int STAGES>
void walk(const GemmArgs &p, int64_t row, int64_t col, uint32_t first, uint32_t steps) {
    typedef StepLoader<BM, BN, 4, STAGES> Loader;
    lds_bytes = Loader::BYTES;
    for (int wave = 0; wave < 4; wave++)
        for (int lane = 0; lane < 64; lane++) {
            const Loader load(p, row, col, lane, wave);
            load.issue_first(lds, first, steps);
            for (uint32_t step = 0; step < steps; step++) {
                if (step >= 8 && step + 8 < steps) continue;      // the middle is like its neighbours
                auto turn = [&](auto t) {
                    if (step % 4 != t) return;
                    for (int i = 0; i < Loader::loads_of(t); i++) load.template issue<t>(lds, first, steps, step / 4, i);
                };
                for_each_of(turn, std::make_integer_sequence<int, 4>{});
            }
        }
}

template <int BM, int BN, int STAGES>
void check(uint64_t rows_a, uint64_t rows_b, uint64_t k, uint64_t wider, uint64_t wider_scales, uint32_t splits) {
    const uint64_t code_pitch = (k + 255) / 256 * 128 + 128 * wider, scale_pitch = std::max((k + 511) / 512 * 16, code_pitch / 16 / 16 * 16 + (code_pitch / 16 % 16 ? 16 : 0)) + 16 * wider_scales;
    for (int i = 0; i < 4; i++) arrays[i] = Array{reinterpret_cast<const uint8_t *>(uint64_t(i + 1) << 44), (i & 1 ? rows_b : rows_a) * (i < 2 ? code_pitch : scale_pitch)};
    GemmArgs p{};
    p.a = arrays[0].base;
    p.b = arrays[1].base;
    p.a_scale = arrays[2].base;
    p.b_scale = arrays[3].base;
    p.a_pitch = p.b_pitch = code_pitch;
    p.a_scale_pitch = p.b_scale_pitch = scale_pitch;
    p.m = rows_a;
    p.n = rows_b;
    p.steps = (k + 255) / 256;
    p.steps_a_split = splits > 1 ? mx_gemm_steps_a_split(p.steps, splits) : p.steps;
    snprintf(what, sizeof what, "%d x %d, %d stages: %llu x %llu x %llu, pitches %llu and %llu, %u parts", BM, BN, STAGES, (unsigned long long)rows_a, (unsigned long long)rows_b,
             (unsigned long long)k, (unsigned long long)code_pitch, (unsigned long long)scale_pitch, splits);
    for (uint32_t first = 0; first < p.steps; first += p.steps_a_split)
        for (int64_t row : {int64_t(0), int64_t((rows_a - 1) / BM * BM)})
            for (int64_t col : {int64_t(0), int64_t((rows_b - 1) / BN * BN)}) walk<BM, BN, STAGES>(p, row, col, first, std::min(p.steps - first, p.steps_a_split));
}

template <int BM, int BN, int STAGES>
void form() {
    const uint64_t rows[][2] = {{1, 1}, {17, 3}, {BM, BN}, {BM + 1, BN + 2}, {2 * BM - 1, 2 * BN - 3}};
    for (uint64_t k : {1, 256, 257, 512, 513, 1000, 1024, 1025, 1536, 2048, 2049, 8190, 8192, 131072})
        for (const auto &r : rows)
            for (uint32_t splits : {1, 4}) {
                if (splits > 1 && uint64_t(mx_gemm_steps_a_split((k + 255) / 256, splits)) * (splits - 1) >= (k + 255) / 256) continue;
                if (k == 131072 && splits == 1 && r[0] > BM) continue;
                check<BM, BN, STAGES>(r[0], r[1], k, 0, 0, splits);
                if (k < 3000) {
                    check<BM, BN, STAGES>(r[0], r[1], k, 1, 0, splits);
                    check<BM, BN, STAGES>(r[0], r[1], k, 0, 3, splits);
                    check<BM, BN, STAGES>(r[0], r[1], k, (8u << 20) / 128 - (k + 255) / 256, 0, splits);      // the longest rows these kernels take
                }
            }
}

}  // namespace

int main() {
    form<256, 256, 2>();
    form<192, 192, 2>();
    form<128, 128, 2>();
    form<64, 128, 2>();
    form<64, 64, 4>();
    form<64, 64, 2>();
    printf("ok %llu loads\n", count);
}
