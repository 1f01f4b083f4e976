// Tiles of products of 8-bit matrices with a scale for each block of 128: the sums that a block forms of what f8_loader.hpp loads. Used by the product (f8_gemm.hip) and by the gated
// block (f8_gated.hip).
//
// A block's products are summed by the matrix instructions, from zero; the vector units add the sum, times the two scales, to the f32 sums: four multiply-adds for 16 x 16 elements of C a lane. Sums therefore lie in ordinary
// registers, not in accumulation registers, which the vector units cannot read. There are two ways to a block's sum:
//   * v_mfma_f32_16x16x128_f8f6f4 takes the codes: 128 is a block. It adds eight products at a time in a window of 14 bits below the largest of them (measured: 2^16 + 2^2 loses the 2^2, 2^16 + 2^3 does not; between eights nothing
//     is lost), so that a sum is off by 1.5e-5 of its size in the mean over normally distributed data, at most some 2^-16 of the sum of magnitudes. For results in 16 bits, whose rounding is 2^-9 (2^-12).
//   * WIDE: v_mfma_f32_16x16x32_bf16, four times, of the codes as bf16, which holds them: half the rate, and sums as f32 gives them (1e-8). For results in f32, and for those that are rounded to 8 bits, whose scales are f32.
//
// B goes first: a lane then holds four consecutive columns of one row of C. Fragments of rows of A and B hold rows in an order of their own (below), so that a lane ends up with 4 TNG consecutive columns of TM consecutive rows.
#pragma once
#include <type_traits>

#include "f8_loader.hpp"
#include "f8_util.hpp"

namespace dsllm {

inline F8Side f8_side(const ckpt_f8_matrix *m) {
    return F8Side{static_cast<const uint8_t *>(m->codes), m->scales, m->code_pitch, m->scale_pitch, m->rows, f8_row_shift(*m)};
}
// 256 rows are addressed with 32 bits.
constexpr int64_t kF8LongestRow = 1 << 23;
inline const char *wrong_f8_contraction(const ckpt_f8_matrix *m) {
    return m->cols > kF8LongestRow || (m->rows && m->cols && m->code_pitch > uint64_t(kF8LongestRow)) ? "a product contracts over at most 2^23 elements, and takes pitches up to that" : nullptr;
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int FA, int FB>      // 0: E4M3, 1: E5M2
__device__ __forceinline__ f32x4 mfma_f8(i32x8 b, i32x8 a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, f32x4{0, 0, 0, 0}, FB, FA, 0, 0, 0, 0);
}
// Eight codes as bf16, which holds the values of both formats.
template <int FORMAT>
__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t hi) {
    u32x4 r;
    if constexpr (FORMAT == 0) {
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    } else {
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, false));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, true));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, false));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, true));
    }
    return __builtin_bit_cast(bf16x8, r);
}
// What a fragment is to the matrix instructions: a lane's 32 codes of a step, or those as bf16. Any order of K will do that both sides share.
template <bool WIDE, int FORMAT> struct F8Fragment {
    i32x8 codes;
    __device__ __forceinline__ void set(u32x4 lo, u32x4 hi) { codes = i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)}; }
};
template <int FORMAT> struct F8Fragment<true, FORMAT> {
    bf16x8 eights[4];
    __device__ __forceinline__ void set(u32x4 lo, u32x4 hi) {
        eights[0] = widened<FORMAT>(lo.x, lo.y);
        eights[1] = widened<FORMAT>(lo.z, lo.w);
        eights[2] = widened<FORMAT>(hi.x, hi.y);
        eights[3] = widened<FORMAT>(hi.z, hi.w);
    }
};

// The sums over steps [first, first + steps) of K. SQUARE: B's scales are those of 128 x 128, one for a group of columns. acc[i][j][e]: row 16 TM wm + TM ar + i, column 16 TN wn + 16 TNG (j / TNG) + 4 TNG q + 4 (j mod TNG) + e.
template <class S, bool SQUARE, bool WIDE, int FA, int FB>
__device__ __forceinline__ void f8_sums(f32x4 (&acc)[S::TM][S::TN], uint8_t *lds, const F8Loader<S> &load, uint32_t first, uint32_t steps, int lane, int wm, int wn) {
    const int q = lane >> 4, ar = lane & 15;
#pragma unroll
    for (int i = 0; i < S::TM; i++)
#pragma unroll
        for (int j = 0; j < S::TN; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    if (!steps) return;
#pragma unroll
    for (int s = 0; s < S::STAGES; s++) load.issue(lds + s * S::STAGE, first + min(uint32_t(s), steps - 1));
    const int swizzle = f8_rotated((ar >> 1) & 7), x0 = ar * 128 + 16 * ((2 * q) ^ swizzle), x1 = ar * 128 + 16 * ((2 * q + 1) ^ swizzle);
    const int base_a = wm * S::TM * 2048, base_b = S::BM * 128 + wn * S::TN * 2048;
    const int scales_a = S::CODES + 4 * (16 * S::TM * wm + S::TM * ar), scales_b = S::CODES + 4 * (S::BM + 16 * S::TN * wn);
    uint32_t at = 0;      // the stage's place
    for (uint32_t s = 0; s < steps; s++) {
        uint8_t *stage = lds + at;
        at = at + S::STAGE == S::BYTES ? 0 : at + S::STAGE;
        wait_loads_and_meet<(S::STAGES - 1) * S::LOADS>();
        auto read = [&](auto &f, int base) { f.set(*reinterpret_cast<const u32x4 *>(stage + base + x0), *reinterpret_cast<const u32x4 *>(stage + base + x1)); };
        float sa[S::TM];
#pragma unroll
        for (int i = 0; i < S::TM; i++) sa[i] = *reinterpret_cast<const float *>(stage + scales_a + 4 * i);
        F8Fragment<WIDE, FA> fa[S::TM];
#pragma unroll
        for (int i = 0; i < S::TM; i++) read(fa[i], base_a + 2048 * i);
#pragma unroll
        for (int j = 0; j < S::TN; j++) {
            F8Fragment<WIDE, FB> fb;
            read(fb, base_b + 2048 * j);
            const uint8_t *sb_at = stage + scales_b + 4 * (16 * S::TNG * (j / S::TNG) + (SQUARE ? 0 : 4 * S::TNG * q + 4 * (j % S::TNG)));
            f32x4 sum[S::TM];
            if constexpr (WIDE) {
#pragma unroll
                for (int k = 0; k < 4; k++)
#pragma unroll
                    for (int i = 0; i < S::TM; i++) sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.eights[k], fa[i].eights[k], k ? sum[i] : f32x4{0, 0, 0, 0}, 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < S::TM; i++) sum[i] = mfma_f8<FA, FB>(fb.codes, fa[i].codes);
            }
#pragma unroll
            for (int i = 0; i < S::TM; i++) {
                if constexpr (SQUARE) {
                    const float scale = sa[i] * *reinterpret_cast<const float *>(sb_at);
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[i][j][e] = __builtin_fmaf(sum[i][e], scale, acc[i][j][e]);
                } else {
                    const f32x4 sb = *reinterpret_cast<const f32x4 *>(sb_at);
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[i][j][e] = __builtin_fmaf(sum[i][e], sa[i] * sb[e], acc[i][j][e]);
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // no wave reads this stage any more
        load.issue(stage, first + min(s + S::STAGES, steps - 1));
    }
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");      // no load to LDS is under way
}

// ------------------------------------------------------------------ up to sixteen rows of A

// As single tokens give them: B is what has to be read, once, at the rate of memory. A block takes 16 rows of B (of each of MATRICES); its waves take the windows of four steps in turn, each with LDS of its own, so that none waits
// for another before the sums are added, in wave order. Four steps of B and A are under way a wave; a step's place is filled again as soon as it has been read.
template <int WAVES, int MATRICES>
struct F8Few {
    typedef F8FewLoader<MATRICES> Loader;
    static constexpr int SIDES = Loader::SIDES, STEP = Loader::STEP, BYTES = WAVES * Loader::WAVE;

    // sum[x] of wave 0: of row ar = lane mod 16 of A with the rows n0 + 4 (lane / 16) to that + 3 of matrix x
    template <int FA, int FB>
    static __device__ __forceinline__ void sums(f32x4 (&sum)[MATRICES], const F8Side &a, const F8Side &b, const F8Side &b2, uint32_t steps, int64_t n0, uint8_t *lds, int lane, int wave) {
        const int q = lane >> 4, ar = lane & 15;
        uint8_t *mine = lds + wave * Loader::WAVE;
        const Loader load(a, b, b2, steps, n0, lane);
        const int swizzle = f8_rotated((ar >> 1) & 7), x0 = ar * 128 + 16 * ((2 * q) ^ swizzle), x1 = ar * 128 + 16 * ((2 * q + 1) ^ swizzle);
        const uint32_t windows = (steps + 3) / 4;
#pragma unroll
        for (int x = 0; x < MATRICES; x++) sum[x] = f32x4{0, 0, 0, 0};
        auto do_window = [&](auto more, uint32_t window, uint32_t odd) {
#pragma unroll
            for (int s = 0; s < 4; s++) {
                // this step's loads have landed; those of the later ones, and what has been asked for of the next window, may be under way
                if constexpr (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * Loader::STEP_LOADS + (s ? Loader::SCALE_LOADS : 0)) : "memory");
                else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Loader::STEP_LOADS * (3 - s)) : "memory");
                u32x4 lo[SIDES], hi[SIDES];
#pragma unroll
                for (int i = 0; i < SIDES; i++) {
                    lo[i] = *reinterpret_cast<const u32x4 *>(mine + s * STEP + 2048 * i + x0);
                    hi[i] = *reinterpret_cast<const u32x4 *>(mine + s * STEP + 2048 * i + x1);
                }
                const float *scales = reinterpret_cast<const float *>(mine + 4 * STEP + (odd & 1) * Loader::SCALES) + 16 * SIDES * s;
                float sa = scales[ar];
                f32x4 sb[MATRICES];
#pragma unroll
                for (int x = 0; x < MATRICES; x++) sb[x] = *reinterpret_cast<const f32x4 *>(scales + 16 * (1 + x) + 4 * q);
                if constexpr (MATRICES == 1) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(lo[0]), "+v"(lo[1]), "+v"(hi[0]), "+v"(hi[1]), "+v"(sa), "+v"(sb[0])::"memory");
                else asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(lo[0]), "+v"(lo[1]), "+v"(lo[SIDES - 1]), "+v"(hi[0]), "+v"(hi[1]), "+v"(hi[SIDES - 1]), "+v"(sa), "+v"(sb[0]), "+v"(sb[MATRICES - 1])::"memory");
                if constexpr (more) {
                    if (s == 0) load.issue_scales(mine, window + WAVES, odd + 1);
                    load.issue_step(mine, window + WAVES, s);
                }
                if (4 * window + s >= steps) continue;
                F8Fragment<true, FA> fa;
                fa.set(lo[0], hi[0]);
#pragma unroll
                for (int x = 0; x < MATRICES; x++) {
                    F8Fragment<true, FB> fb;
                    fb.set(lo[1 + x], hi[1 + x]);
                    f32x4 block{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 4; k++) block = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.eights[k], fa.eights[k], block, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; e++) sum[x][e] = __builtin_fmaf(block[e], sa * sb[x][e], sum[x][e]);
                }
            }
        };
        if (uint32_t(wave) < windows) {
            load.issue_scales(mine, wave, 0);
#pragma unroll
            for (int s = 0; s < 4; s++) load.issue_step(mine, wave, s);
            uint32_t window = wave, odd = 0;
            for (; window + WAVES < windows; window += WAVES, odd++) do_window(std::true_type{}, window, odd);
            do_window(std::false_type{}, window, odd);
        }
        __syncthreads();
        f32x4 *part = reinterpret_cast<f32x4 *>(lds);
        if (wave > 0)
#pragma unroll
            for (int x = 0; x < MATRICES; x++) part[((wave - 1) * MATRICES + x) * 64 + lane] = sum[x];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < WAVES - 1; w++)
#pragma unroll
            for (int x = 0; x < MATRICES; x++) sum[x] += part[(w * MATRICES + x) * 64 + lane];
    }
};

}  // namespace dsllm
