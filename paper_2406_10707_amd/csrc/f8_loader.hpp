// What products of 8-bit matrices with a scale for each block of 128 load, and to which places of LDS (f8_tile.hpp).
#pragma once
#include "gemm_tile.hpp"
#include "kernel_util.hpp"

namespace dsllm {

struct F8Side {
    const uint8_t *codes;
    const float *scales;
    uint64_t pitch, scale_pitch;
    int64_t rows;
    uint32_t shift;      // rows to a scale: 2^shift
};
// WM x WN waves, each computing (16 TM) x (16 TN) of the block's tile. TNG: fragments of B whose columns a lane holds one behind the other. STAGES steps of 128 values in LDS. PAIR: B's rows are those of two matrices, in turn
// groups of 16 TNG rows of the one and of the other.
//
// LDS of a stage: a place of 128 bytes for each row of A and of B, in the order in which fragments read them: fragment i of a wave takes places 16 i to 16 i + 15 of the wave's, lane ar = lane mod 16 the place ar, which holds
// row TM ar + i of A's wave tile, or row 4 TNG (ar / 4) + 4 j + ar mod 4 of a group of TNG fragments of B. Of place p, piece x (16 bytes) lies at x ^ f(p), f(p) = bits 1 to 3 of p, rotated: reads of neighbouring
// places lie in different banks. The loads write LDS in lane order; both orders are made on the global side. Then a scale for each row of A and of B.
template <int WM_, int WN_, int TM_, int TN_, int TNG_, int STAGES_, bool PAIR_>
struct F8Shape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, TNG = TNG_, STAGES = STAGES_;
    static constexpr bool PAIR = PAIR_;
    static constexpr int NW = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN, THREADS = 64 * NW;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LOADS = LA + LB + 1;      // a wave's loads of a step
    static constexpr int CODES = (BM + BN) * 128, STAGE = CODES + 256 * NW, BYTES = STAGES * STAGE;
    static_assert(LA * 8 * NW == BM && LB * 8 * NW == BN && TN % TNG == 0 && NW * 64 >= BM + BN && BM % 64 == 0, "loads divide among the waves");
    static_assert(!PAIR || TN == 2 * TNG, "a wave has a group of each");
};

// The product's, in the order of kF8Forms
template <int FORM> struct F8GemmShape;
template <> struct F8GemmShape<0> { typedef F8Shape<4, 2, 4, 8, 4, 2, false> type; };
template <> struct F8GemmShape<1> { typedef F8Shape<4, 2, 4, 4, 4, 3, false> type; };
template <> struct F8GemmShape<2> { typedef F8Shape<2, 2, 4, 4, 4, 2, false> type; };
template <> struct F8GemmShape<3> { typedef F8Shape<2, 2, 2, 2, 2, 4, false> type; };
// Those of the gated block's forward pass, in the order of gated_form; of its values first, and of the backward pass
template <int FORM> struct F8GatedShape;
template <> struct F8GatedShape<0> { typedef F8Shape<4, 2, 4, 8, 4, 2, true> type; };
template <> struct F8GatedShape<1> { typedef F8Shape<4, 2, 2, 8, 4, 2, true> type; };
template <> struct F8GatedShape<2> { typedef F8Shape<2, 4, 2, 4, 2, 2, true> type; };
typedef F8Shape<2, 2, 2, 2, 1, 4, true> F8GatedValuesShape;
typedef F8Shape<2, 2, 4, 4, 4, 2, false> F8BackwardShape;

__device__ __forceinline__ uint32_t f8_rotated(uint32_t three_bits) { return ((three_bits << 1) & 7) | (three_bits >> 2); }

// Rows past the end of a matrix are its last row again.
template <class S>
struct F8Loader {
    __amdgpu_buffer_rsrc_t ra, rb[2];
    uint32_t pitch_a, pitch_b[2], row_a, row_b, last_a, last_b, piece, wave;      // this lane's rows with the wave's first load, and what part of a row
    const float *scale;
    uint64_t scale_pitch;

    static constexpr uint32_t row_of_place_a(uint32_t place) { return place / (16 * S::TM) * (16 * S::TM) + S::TM * (place % 16) + place / 16 % S::TM; }
    static constexpr uint32_t row_of_place_b(uint32_t place) { return place / (16 * S::TNG) * (16 * S::TNG) + 4 * S::TNG * (place % 16 / 4) + 4 * (place / 16 % S::TNG) + place % 4; }
    // which of the two matrices, and which row behind the tile's first, the tile's row n of B is
    static constexpr uint32_t matrix_of(uint32_t n) { return S::PAIR ? n / (16 * S::TNG) & 1 : 0; }
    static constexpr uint32_t row_of(uint32_t n) { return S::PAIR ? n / (32 * S::TNG) * (16 * S::TNG) + n % (16 * S::TNG) : n; }

    __device__ __forceinline__ F8Loader(const F8Side a, const F8Side b, const F8Side b2, uint32_t steps, int64_t row, int64_t col, int lane, uint32_t wave_) : wave(wave_) {
        constexpr int ROWS_B = S::PAIR ? S::BN / 2 : S::BN;
        last_a = uint32_t(min(a.rows - row, int64_t(S::BM)) - 1);
        last_b = uint32_t(min(b.rows - col, int64_t(ROWS_B)) - 1);
        // a load's places are those of the first load and a multiple of 8 NW: sizes are powers of two, so that its rows are the sum of both places' rows
        const uint32_t place = 8 * wave + (lane >> 3);
        row_a = row_of_place_a(place);
        row_b = row_of(row_of_place_b(place));
        piece = 16 * ((lane & 7) ^ f8_rotated(((lane >> 4) & 3) | ((wave & 1) << 2)));
        auto descriptor = [&](const F8Side &side, int64_t first, uint32_t last) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(side.codes + first * side.pitch), 0, last * uint32_t(side.pitch) + 128 * steps, 0x00020000);
        };
        ra = descriptor(a, row, last_a);
        rb[0] = descriptor(b, col, last_b);
        rb[1] = S::PAIR ? descriptor(b2, col, last_b) : rb[0];
        pitch_a = uint32_t(a.pitch);
        pitch_b[0] = uint32_t(b.pitch);
        pitch_b[1] = uint32_t(b2.pitch);
        if (S::PAIR && matrix_of(8 * wave)) {      // this wave's loads begin with the second
            const auto r = rb[0];
            rb[0] = rb[1];
            rb[1] = r;
            const uint32_t p = pitch_b[0];
            pitch_b[0] = pitch_b[1];
            pitch_b[1] = p;
        }
        const uint32_t slot = 64 * wave;      // of the wave's first lane: a wave's scales are all A's or all B's
        if (slot < S::BM) {
            scale = a.scales + ((row + min(slot + lane, last_a)) >> a.shift);
            scale_pitch = a.scale_pitch;
        } else {
            const uint32_t n = min(slot - S::BM + lane, uint32_t(S::BN - 1));
            scale = b.scales;
            scale_pitch = b.scale_pitch;
            if (S::PAIR && matrix_of(n)) { scale = b2.scales; scale_pitch = b2.scale_pitch; }
            scale += (col + min(row_of(n), last_b)) >> b.shift;
        }
    }
    // all loads of a step into a stage
    __device__ __forceinline__ void issue(uint8_t *stage, uint32_t step) const {
#pragma unroll
        for (int c = 0; c < S::LOADS; c++) issue(stage, step, c);
    }
    __device__ __forceinline__ void issue(uint8_t *stage, uint32_t step, int c) const {
        if (c < S::LA) {
            const uint32_t at = min(row_a + row_of_place_a(8 * S::NW * c), last_a) * pitch_a + piece;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (DSLLM_LDS void *)(stage + 1024 * (S::NW * c + wave)), 16, at, 128 * step, 0, 0);
        } else if (c < S::LA + S::LB) {
            const uint32_t first = 8 * S::NW * (c - S::LA), which = matrix_of(first), at = min(row_b + row_of(row_of_place_b(first)), last_b) * pitch_b[which] + piece;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb[which], (DSLLM_LDS void *)(stage + S::BM * 128 + 1024 * (S::NW * (c - S::LA) + wave)), 16, at, 128 * step, 0, 0);
        } else __builtin_amdgcn_global_load_lds((const DSLLM_GLB void *)(scale + step * scale_pitch), (DSLLM_LDS void *)(stage + S::CODES + 256 * wave), 4, 0, 0);
    }
};

// What a wave of a product of up to sixteen rows of A (EIGHT: up to eight) loads: 16 (8) rows of A and 16 of each of MATRICES, 128 bytes a row and step, four steps to a window. LDS of a wave: the places of four steps, of each A's, then the others'; then two windows'
// scales, for each step 16 of A and 16 of each matrix. Rows past the end are the last row again; pieces of a place are permuted as in the tiles.
template <int MATRICES, bool EIGHT>
struct F8FewLoader {
    static constexpr int SIDES = 1 + MATRICES, A_PLACES = EIGHT ? 1024 : 2048, STEP = A_PLACES + MATRICES * 2048, SCALES = 4 * SIDES * 64, STEP_LOADS = STEP / 1024, SCALE_LOADS = SIDES, WAVE = 4 * STEP + 2 * SCALES;
    const uint8_t *from[STEP_LOADS];      // this lane's piece of the rows lane / 8 and, if there are so many, that + 8 of each side
    const float *scale_from[SCALE_LOADS];
    uint32_t scale_step[SCALE_LOADS], steps;
    uint64_t scale_pitch[SCALE_LOADS];

    __device__ __forceinline__ F8FewLoader(const F8Side &a, const F8Side &b, const F8Side &b2, uint32_t steps_, int64_t n0, int lane) : steps(steps_) {
#pragma unroll
        for (int i = 0; i < STEP_LOADS; i++) {
            constexpr int OF_A = A_PLACES / 1024;
            const int r = 8 * (i < OF_A ? i : (i - OF_A) & 1) + (lane >> 3);
            const F8Side &side = i < OF_A ? a : i < OF_A + 2 ? b : b2;
            from[i] = side.codes + min((i < OF_A ? 0 : n0) + r, side.rows - 1) * side.pitch + 16 * ((lane & 7) ^ f8_rotated((r >> 1) & 7));
        }
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; i++) {      // scale 64 i + lane of a window: step, then side, then row
            const uint32_t at = 64 * i + lane, which = at / 16 % SIDES;
            const F8Side &side = which == 0 ? a : which == 1 ? b : b2;
            scale_step[i] = at / (16 * SIDES);
            scale_from[i] = side.scales + (min((which ? n0 : 0) + int64_t(at % 16), side.rows - 1) >> side.shift);
            scale_pitch[i] = side.scale_pitch;
        }
    }
    // steps past the end are the last again
    __device__ __forceinline__ void issue_scales(uint8_t *mine, uint32_t window, uint32_t odd) const {
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; i++)
            __builtin_amdgcn_global_load_lds((const DSLLM_GLB void *)(scale_from[i] + min(4 * window + scale_step[i], steps - 1) * scale_pitch[i]), (DSLLM_LDS void *)(mine + 4 * STEP + (odd & 1) * SCALES + 256 * i), 4, 0, 0);
    }
    __device__ __forceinline__ void issue_step(uint8_t *mine, uint32_t window, int s) const {
        const uint64_t at = 128 * uint64_t(min(4 * window + s, steps - 1));
#pragma unroll
        for (int i = 0; i < STEP_LOADS; i++) __builtin_amdgcn_global_load_lds((const DSLLM_GLB void *)(from[i] + at), (DSLLM_LDS void *)(mine + s * STEP + 1024 * i), 16, 0, 0);
    }
};

}  // namespace dsllm
