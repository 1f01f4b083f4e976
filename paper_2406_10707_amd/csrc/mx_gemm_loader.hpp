// What a product of two MXFP4 matrices loads, and to which places of LDS (mx_gemm.hip).
#pragma once
#include "gemm_tile.hpp"
#include "kernel_util.hpp"
#include "mx_gemm_forms.hpp"

namespace dsllm {

struct GemmArgs {
    const uint8_t *a, *b, *a_scale, *b_scale;
    uint64_t a_pitch, b_pitch, a_scale_pitch, b_scale_pitch;
    void *c;
    int64_t ldc;
    int64_t m, n;
    uint32_t steps;        // of 256 values
    uint32_t steps_a_split;
    int64_t c_split;       // elements of C from one part of K to the next
    int accumulate, vector;
};

// The panels of a step of K (256 values, 128 bytes of codes a row) and the scales of four steps (32 bytes a row: pieces of 8 bytes, a step's, would take as
// many requests as the panels) go from memory to LDS without passing through registers. Rows past the end of a matrix are its last row again.
//
// LDS layout of a panel: eight 16-byte pieces (blocks of 32 values) a row; row r keeps piece p at place p ^ f(r), so that the rows that a fragment read
// touches lie in different banks. The loads write LDS in lane order, so the permutation is made on the global side. A fragments hold 16
// consecutive rows, f(r) = bits 1..3 of r, rotated; B fragments come in pairs that hold 32 rows as 8 (lane / 4) + lane % 4 and that + 4, f(r) = bits 1, 3, 4,
// rotated: with B as the first operand a lane ends up with eight consecutive columns of one row of C.
// Half h of a step takes piece 2 q + h in the lanes 16 q to 16 q + 15 (any order of K will do that both sides share): a lane's two scales of a step are
// then neighbours, in the upper or the lower half of an aligned word.
// LDS layout of the scales: of eight rows the first two steps' 16 bytes one behind the other, then the other two steps' (every other eight rows the other way round).
[[maybe_unused]] __device__ __forceinline__ uint32_t rotated(uint32_t three_bits) { return ((three_bits << 1) & 7) | (three_bits >> 2); }

template <int BM, int BN, int NW, int STAGES>
struct StepLoader {
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, PANELS = LA + LB;
    static constexpr int PANEL = (BM + BN) * 128, SCALES = (BM + BN) * 32, GROUPS = (BM + BN) / 32, BYTES = STAGES * PANEL + 2 * SCALES;
    static_assert(LA * 8 * NW == BM && LB * 8 * NW == BN && NW == 4 && BM % 32 == 0 && BN % 32 == 0, "panels divide among the waves");
    static constexpr int PARTS = (GROUPS + NW - 1) / NW;      // loads of a wave that a window of scales takes; at most one a step
    static_assert(STAGES == 2 ? PARTS <= 4 : STAGES == 4 && PARTS <= 2, "a step has one of them, and all are out before the panels that come with them");
    // which part goes out ahead of the panels in a window's step `turn`, of the next window or, in the last step, the next but one
    static constexpr int part_of(int turn) { return turn == 3 ? 0 : turn + 1; }
    static constexpr int scales_of(int turn) { return part_of(turn) < PARTS ? 1 : 0; }
    static constexpr int loads_of(int turn) { return scales_of(turn & 3) + PANELS; }
    __amdgpu_buffer_rsrc_t ra, rb, rs[PARTS];
    uint32_t off[LA + LB], scale_row[PARTS], scale_half, last_scales[PARTS], scale_place[PARTS], wave;

    __device__ __forceinline__ StepLoader(const GemmArgs &p, int64_t row, int64_t col, int lane, int wave_) : wave(wave_) {
        const uint32_t last_a = uint32_t(min(p.m - row, int64_t(BM)) - 1), last_b = uint32_t(min(p.n - col, int64_t(BN)) - 1);
        ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.a + row * p.a_pitch), 0, (last_a + 1) * uint32_t(p.a_pitch), 0x00020000);
        rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.b + col * p.b_pitch), 0, (last_b + 1) * uint32_t(p.b_pitch), 0x00020000);
        const uint32_t row0 = (lane >> 3) + 8 * wave, piece = lane & 7;
        const uint32_t fa = rotated(((lane >> 4) & 3) | ((wave & 1) << 2)), fb = rotated(((lane >> 4) & 1) | ((wave & 3) << 1));      // f of row0, and of every 32nd row from it
#pragma unroll
        for (int i = 0; i < LA + LB; i++) {
            const uint32_t r = row0 + 8 * NW * (i < LA ? i : i - LA);
            off[i] = (i < LA ? min(r, last_a) * uint32_t(p.a_pitch) : min(r, last_b) * uint32_t(p.b_pitch)) + 16 * (piece ^ (i < LA ? fa : fb));
        }
        scale_half = 16 * (((lane >> 3) ^ (lane >> 4)) & 1);
#pragma unroll
        for (int i = 0; i < PARTS; i++) {
            // rows of A, then of B; of each 32 of B first the sixteen of the pair's first fragment
            const uint32_t group = (i * NW + wave) % GROUPS, place = 8 * (lane >> 4) + (lane & 7);
            const bool of_a = 32 * group < BM;
            const uint32_t r = 32 * group + (of_a ? place : 8 * ((place & 15) >> 2) + (place & 3) + 4 * (place >> 4));
            scale_place[i] = STAGES * PANEL + 1024 * group;
            scale_row[i] = of_a ? min(r, last_a) * uint32_t(p.a_scale_pitch) : min(r - BM, last_b) * uint32_t(p.b_scale_pitch);
            last_scales[i] = uint32_t(of_a ? p.a_scale_pitch : p.b_scale_pitch) - 16;
            const uint8_t *base = of_a ? p.a_scale + row * p.a_scale_pitch : p.b_scale + col * p.b_scale_pitch;
            rs[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, of_a ? (last_a + 1) * uint32_t(p.a_scale_pitch) : (last_b + 1) * uint32_t(p.b_scale_pitch), 0x00020000);
        }
    }
    // where the 16 bytes of the window's first two steps of the row in place r lie; those of the other two: that ^ 128
    static __device__ __forceinline__ int scale_at(int r) { return STAGES * PANEL + (r >> 3) * 256 + ((r >> 3) & 1) * 128 + (r & 7) * 16; }
    // Part of a window of scales (four steps), which goes to the place of even or odd ones. What a row has behind its end is not used, and not read: its last sixteen bytes are taken
    // again (the window would be the load's scalar offset, of which its range check cannot be relied on).
    __device__ __forceinline__ void issue_scales(uint8_t *lds, uint32_t window, uint32_t odd, int part) const {
        const uint32_t at = scale_row[part] + min(32 * window + scale_half, last_scales[part]);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs[part], (DSLLM_LDS void *)(lds + scale_place[part] + (odd & 1) * SCALES), 16, at, 0, 0, 0);
    }
    // instruction j of a step's panels into stage `stage`
    __device__ __forceinline__ void issue_panels(uint8_t *lds, int stage, uint32_t step, int j) const {
        uint8_t *place = lds + stage * PANEL + (j < LA ? j : j - LA) * 1024 * NW + 1024 * wave + (j < LA ? 0 : BM * 128);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(j < LA ? ra : rb, (DSLLM_LDS void *)place, 16, off[j], 128 * step, 0, 0);
    }
    // Steps are counted from the part of K's first, which is a multiple of 4. Past the end the last step is loaded again, into a stage nothing reads.
    // What is on its way before the first step: (STAGES - 1) * PANELS + 1 loads behind the first window of scales and the first step
    __device__ __forceinline__ void issue_first(uint8_t *lds, uint32_t first, uint32_t steps) const {
#pragma unroll
        for (int i = 0; i < PARTS; i++) issue_scales(lds, first / 4, 0, i);
#pragma unroll
        for (int s = 0; s < STAGES; s++) {
            if (s == STAGES - 1) issue_scales(lds, first / 4 + 1, 1, 0);
#pragma unroll
            for (int i = 0; i < PANELS; i++) issue_panels(lds, s, first + min(uint32_t(s), steps - 1), i);
        }
    }
    // load i of those that go out in step 4 window + TURN: one of a later window of scales (not in every step), then the panels of the step STAGES later
    template <int TURN>
    __device__ __forceinline__ void issue(uint8_t *lds, uint32_t first, uint32_t steps, uint32_t window, int i) const {
        constexpr int part = part_of(TURN), scales = scales_of(TURN);
        if (scales && i == 0) issue_scales(lds, first / 4 + window + 1 + (TURN + 1) / 4, window + 1 + (TURN + 1) / 4, part);
        else issue_panels(lds, TURN % STAGES, first + min(4 * window + TURN + STAGES, steps - 1), i - scales);
    }
};

}  // namespace dsllm
