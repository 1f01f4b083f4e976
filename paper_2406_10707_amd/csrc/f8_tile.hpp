// Tiles of products of 8-bit matrices with a scale for each block of 128: the sums that a block forms of what f8_loader.hpp loads. Used by the product (f8_gemm.hip) and by the gated
// block (f8_gated.hip).
//
// A block's products are summed by the matrix instructions, from zero; the vector units add the sum, times the two scales, to the f32 sums: four multiply-adds for 16 x 16 elements of C a lane. Sums therefore lie in ordinary
// registers, not in accumulation registers, which the vector units cannot read. There are two ways to a block's sum:
//   * v_mfma_f32_16x16x128_f8f6f4 takes the codes: 128 is a block. It adds eight products, of consecutive elements, at a time, each cut to a multiple of 2^-13 of 2^e, e the largest sum of two exponents among the eight
//     (a subnormal code has the smallest normal one's). Measured: beside 2^16, 2^3 stays, 15 becomes 8 and 7 becomes 0; between eights nothing is lost. So an eight is off by less than 7 * 2^-13 of its largest product, a sum by less than
//     2^-10 of the sum of magnitudes (of normal codes; an eight of subnormal ones by up to 2^3 more of its own products). In the mean over normally distributed data it is 1.5e-5 of the sum's size. The worst is a quarter of what the
//     rounding of a result to bf16 may be off by, 2^-8 of it, unless large products cancel: what stood beside them is lost then. Only for C in bf16: half a step of f16 is 2^-11.
//   * WIDE: v_mfma_f32_16x16x32_bf16, four times, of the codes as bf16, which holds them: half the rate, and sums as f32 gives them (1e-8). For results in f32 and f16, and for those that are rounded to 8 bits, whose scales are f32.
//
// B goes first: a lane then holds four consecutive columns of one row of C. Fragments of rows of A and B hold rows in an order of their own (below), so that a lane ends up with 4 TNG consecutive columns of TM consecutive rows.
//
// Measured, 8192 x 8192 x 8192: 463 us in 8 bits (2.37 PFLOP/s; at 2.0 GHz, 57 % of the matrix instructions' cycles at 4096 x 4096 x 11008), 865 us in bf16 (1.27 PFLOP/s; a plain bf16 product of that size by the image's library 776). What bounds both is the
// vector instructions beside the matrix instructions, and power. In bf16 a step of a 64 x 64 wave has 64 matrix instructions, 128 conversions, 64 multiply-adds and, with scales of single rows of B, 64 products of scales: 11008 x 4096 x 8192 added to f32 705 to
// 740 us, at 1.9 GHz, where the matrix instructions take 47 % of a SIMD's cycles and the vector instructions (4.9 cycles a conversion, 2.7 a multiply-add) about as many. Waves of 64 x 128 (256 x 256 tiles) have a quarter fewer conversions
// to a matrix instruction, spill two to nine registers, and cost 2 % less a step, so that conversions alone are not it; the same loop without conversions and multiply-adds runs at 1.6 PFLOP/s.
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
// The sums over steps [first, first + steps) of K. SQUARE: B's scales are those of 128 x 128, one for a group of columns. acc[i][j][e]: row 16 TM wm + TM ar + i, column 16 TN wn + 16 TNG (j / TNG) + 4 TNG q + 4 (j mod TNG) + e.
//
// The wave's own order is fixed by hand, and two waves share a SIMD. A's fragments of a step stay in registers, B's come one after the other; beside the matrix instructions stand the reads and conversions of what later ones need, and the
// multiply-adds of the sums that were in the place of theirs. One barrier a step, before its last fragments: then every wave has read the whole stage, and all loads of the next have landed, which were issued a step (STAGES - 1 steps)
// before. Behind it come the loads into the stage that is free now, and the reads of the next: A's fragments take the places of those whose last matrix instruction has been issued.
template <class S, bool SQUARE>
struct F8Stages {
    static constexpr int TM = S::TM, TN = S::TN, TNG = S::TNG;
    const F8Loader<S> &load;
    uint8_t *lds;
    const uint8_t *from;      // the stage that is read
    uint32_t first, steps, next, into;      // the stage behind it; the one that loads go to
    int x[2], base_a, base_b, scales_a, scales_b;      // a lane's two pieces of a place; places of the wave
    float sa[TM], sb[TN / TNG];

    // AHEAD: loads of a step that are out when the step before the STAGES - 1 before begins
    __device__ __forceinline__ F8Stages(uint8_t *lds_, const F8Loader<S> &load_, uint32_t first_, uint32_t steps_, int lane, int wm, int wn, int ahead)
        : load(load_), lds(lds_), from(lds_), first(first_), steps(steps_), next(S::STAGE), into((S::STAGES - 1) * S::STAGE) {
        const int q = lane >> 4, ar = lane & 15, swizzle = f8_rotated((ar >> 1) & 7);
        x[0] = ar * 128 + 16 * ((2 * q) ^ swizzle);
        x[1] = ar * 128 + 16 * ((2 * q + 1) ^ swizzle);
        base_a = wm * TM * 2048;
        base_b = S::BM * 128 + wn * TN * 2048;
        scales_a = S::CODES + 4 * (16 * TM * wm + TM * ar);
        scales_b = S::CODES + 4 * (S::BM + 16 * TN * wn) + (SQUARE ? 0 : 16 * TNG * q);
#pragma unroll
        for (int s = 0; s < S::STAGES - 1; s++) load.issue(lds + s * S::STAGE, first + min(uint32_t(s), steps - 1));
#pragma unroll
        for (int c = 0; c < ahead; c++) load.issue(lds + into, first + min(uint32_t(S::STAGES - 1), steps - 1), c);
    }
    // load c of the step `behind` the current one; past the end the last step's again, into a stage that nothing reads
    __device__ __forceinline__ void issue(uint32_t s, int behind, int c) const { load.issue(lds + into, first + min(s + behind, steps - 1), c); }
    __device__ __forceinline__ void turn() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S::STAGES - 2) * S::LOADS) : "memory");
        from = lds + next;
        next = next + S::STAGE == S::BYTES ? 0 : next + S::STAGE;
        into = into + S::STAGE == S::BYTES ? 0 : into + S::STAGE;
    }
    __device__ __forceinline__ u32x2 quarter(int base, int k) const { return *reinterpret_cast<const u32x2 *>(from + base + x[k >> 1] + 8 * (k & 1)); }
    __device__ __forceinline__ u32x4 half(int base, int h) const { return *reinterpret_cast<const u32x4 *>(from + base + x[h]); }
    __device__ __forceinline__ i32x8 fragment(int base) const {
        const u32x4 lo = half(base, 0), hi = half(base, 1);
        return i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
    }
    __device__ __forceinline__ int a_at(int i) const { return base_a + 2048 * i; }
    __device__ __forceinline__ int b_at(int j) const { return base_b + 2048 * j; }
    __device__ __forceinline__ void read_scales() {
#pragma unroll
        for (int i = 0; i < TM; i++) sa[i] = *reinterpret_cast<const float *>(from + scales_a + 4 * i);
        if constexpr (SQUARE)
#pragma unroll
            for (int g = 0; g < TN / TNG; g++) sb[g] = *reinterpret_cast<const float *>(from + scales_b + 64 * TNG * g);
    }
    __device__ __forceinline__ f32x4 row_scales(int j) const { return *reinterpret_cast<const f32x4 *>(from + scales_b + 4 * (16 * TNG * (j / TNG) + 4 * (j % TNG))); }
};

template <class S>
__device__ __forceinline__ void f8_clear(f32x4 (&acc)[S::TM][S::TN]) {
#pragma unroll
    for (int i = 0; i < S::TM; i++)
#pragma unroll
        for (int j = 0; j < S::TN; j++) acc[i][j] = f32x4{0, 0, 0, 0};
}

// In bf16: a step is TN times 4 blocks of TM matrix instructions, a quarter of fragment j (8 of a lane's 32 codes; any order of K will do that both sides share) with those of all of A's fragments. A block's next quarter of B is converted in
// front of it; those of A's next fragments in the blocks behind the barrier.
template <class S, bool SQUARE, int FA, int FB>
__device__ __forceinline__ void f8_sums_wide(f32x4 (&acc)[S::TM][S::TN], uint8_t *lds, const F8Loader<S> &load, uint32_t first, uint32_t steps, int lane, int wm, int wn) {
    constexpr int TM = S::TM, TN = S::TN, BLOCKS = 4 * TN, LAST = BLOCKS - 4, A_BLOCK = (S::LOADS + BLOCKS - 1) / BLOCKS, AHEAD = 4 * A_BLOCK < S::LOADS ? 4 * A_BLOCK : S::LOADS;
    static_assert(TN % 2 == 0 && BLOCKS * A_BLOCK >= S::LOADS, "a step's loads are out within a step");
    f8_clear<S>(acc);
    if (!steps) return;
    F8Stages<S, SQUARE> in(lds, load, first, steps, lane, wm, wn, AHEAD);
    bf16x8 a[TM][4], b[2];      // b: the quarter that counts and the next
    u32x2 raw_a[TM];            // a quarter that is still to be converted
    u32x4 raw_b[2];
    f32x4 sum[TM], sb_rows[2];
    float scale[TM], sa_before[TM];
    auto add = [&](int i, int j) {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if constexpr (SQUARE) acc[i][j][e] = __builtin_fmaf(sum[i][e], scale[i], acc[i][j][e]);
            else acc[i][j][e] = __builtin_fmaf(sum[i][e], (j == TN - 1 ? sa_before[i] : in.sa[i]) * sb_rows[j & 1][e], acc[i][j][e]);
    };
    wait_loads_and_meet<(S::STAGES - 2) * S::LOADS + AHEAD>();
    in.read_scales();
#pragma unroll
    for (int i = 0; i < TM; i++) {
        sum[i] = f32x4{0, 0, 0, 0};      // in the place of the fragment before the first: adds nothing
        scale[i] = sa_before[i] = 0;
#pragma unroll
        for (int k = 0; k < 3; k++) {
            const u32x2 r = in.quarter(in.a_at(i), k);
            a[i][k] = widened<FA>(r.x, r.y);
        }
        raw_a[i] = in.quarter(in.a_at(i), 3);
    }
#pragma unroll
    for (int h = 0; h < 2; h++) raw_b[h] = in.half(in.b_at(0), h);
    b[0] = widened<FB>(raw_b[0].x, raw_b[0].y);
    sb_rows[1] = f32x4{0, 0, 0, 0};
    if constexpr (!SQUARE) sb_rows[0] = in.row_scales(0);
    __builtin_amdgcn_sched_barrier(0);
    for (uint32_t s = 0; s < steps; s++)
        for_each_of([&](auto index) {
            constexpr int at = index, j = at / 4, k = at % 4, before = (j + TN - 1) % TN, to_j = (j + 1) % TN, to_k = (k + 1) % 4;
            if constexpr (at == LAST) in.turn();
#pragma unroll
            for (int i = 0; i < TM; i++) {
                if constexpr (k == 0) add(i, before);
                sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[at & 1], a[i][k], k ? sum[i] : f32x4{0, 0, 0, 0}, 0, 0, 0);
            }
            if constexpr (k == 0 && SQUARE && j % S::TNG == 0)
#pragma unroll
                for (int i = 0; i < TM; i++) scale[i] = in.sa[i] * in.sb[j / S::TNG];
            b[(at & 1) ^ 1] = widened<FB>(raw_b[to_k / 2][to_k % 2 * 2], raw_b[to_k / 2][to_k % 2 * 2 + 1]);
            if constexpr (k % 2 == 0) raw_b[k / 2] = in.half(in.b_at(to_j), k / 2);      // both its quarters are converted
            if constexpr (at > LAST || at == 0)
#pragma unroll
                for (int i = 0; i < TM; i++) a[i][(k + 3) % 4] = widened<FA>(raw_a[i].x, raw_a[i].y);
            if constexpr (at >= LAST)
#pragma unroll
                for (int i = 0; i < TM; i++) raw_a[i] = in.quarter(in.a_at(i), k);
            if constexpr (!SQUARE && k == 3 && at < LAST) sb_rows[(j + 1) & 1] = in.row_scales(j + 1);      // in the place of those that have been used
            if constexpr (at == BLOCKS - 1) {
                if constexpr (!SQUARE) {
#pragma unroll
                    for (int i = 0; i < TM; i++) sa_before[i] = in.sa[i];
                    sb_rows[0] = in.row_scales(0);
                }
                in.read_scales();
            }
            // a step's loads begin in the block of the barrier and go on in the next step
            constexpr int turn = (at + BLOCKS - LAST) % BLOCKS;
#pragma unroll
            for (int c = turn * A_BLOCK; c < (turn + 1) * A_BLOCK && c < S::LOADS; c++) in.issue(s, at >= LAST ? S::STAGES : S::STAGES - 1, c);
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, BLOCKS>{});
#pragma unroll
    for (int i = 0; i < TM; i++) add(i, TN - 1);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // no load to LDS is under way
}

// In 8 bits: one matrix instruction for a fragment of A with one of B. A step takes B's fragments one after the other up to the last two, then A's with both of these: so each of A's is free soon, and the reads of the next, of all waves behind
// the barrier, are spread over two fragments' time (with one, 8192^3 took 512 us).
template <class S, bool SQUARE, int FA, int FB>
__device__ __forceinline__ void f8_sums_narrow(f32x4 (&acc)[S::TM][S::TN], uint8_t *lds, const F8Loader<S> &load, uint32_t first, uint32_t steps, int lane, int wm, int wn) {
    constexpr int TM = S::TM, TN = S::TN, COUNT = TM * TN, LAST = COUNT - 2 * TM, EVERY = COUNT / S::LOADS > 0 ? COUNT / S::LOADS : 1, AT_ONCE = (S::LOADS * EVERY + COUNT - 1) / COUNT;
    static_assert(TN % 2 == 0 && TN <= 8, "");
    // load c goes out behind matrix instruction LAST + c / AT_ONCE * EVERY, of the step or of the next
    constexpr int AHEAD = ((COUNT - LAST + EVERY - 1) / EVERY) * AT_ONCE < S::LOADS ? ((COUNT - LAST + EVERY - 1) / EVERY) * AT_ONCE : S::LOADS;
    static_assert((S::LOADS + AT_ONCE - 1) / AT_ONCE * EVERY <= COUNT, "a step's loads are out within a step");
    constexpr int PLACES = TN > 2 ? 4 : 2;      // of B's fragments
    f8_clear<S>(acc);
    if (!steps) return;
    F8Stages<S, SQUARE> in(lds, load, first, steps, lane, wm, wn, AHEAD);
    i32x8 a[TM], b[PLACES];
    f32x4 sum[TM], sb_rows[SQUARE ? 1 : TN];
    float scale[TN / S::TNG][TM];      // of the step before until they have been used
    wait_loads_and_meet<(S::STAGES - 2) * S::LOADS + AHEAD>();
    // which fragments instruction n of a step takes
    auto row_of = [](int n) constexpr { return n < LAST ? n % TM : (n - LAST) / 2; };
    auto col_of = [](int n) constexpr { return n < LAST ? n / TM : TN - 2 + (n - LAST) % 2; };
    float sa_before[TM];
    f32x4 sb_before[2];
    auto add = [&](int n, bool of_step_before) {
        const int i = row_of(n), j = col_of(n);
#pragma unroll
        for (int e = 0; e < 4; e++)
            if constexpr (SQUARE) acc[i][j][e] = __builtin_fmaf(sum[n % TM][e], scale[j / S::TNG][i], acc[i][j][e]);
            else acc[i][j][e] = __builtin_fmaf(sum[n % TM][e], of_step_before ? sa_before[i] * sb_before[j % 2][e] : in.sa[i] * sb_rows[j][e], acc[i][j][e]);
    };
    in.read_scales();
    if constexpr (!SQUARE)
#pragma unroll
        for (int j = 0; j < TN; j++) sb_rows[j] = in.row_scales(j);
    sb_before[0] = sb_before[1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < TM; i++) {
        sum[i] = f32x4{0, 0, 0, 0};
        sa_before[i] = 0;
#pragma unroll
        for (int g = 0; g < TN / S::TNG; g++) scale[g][i] = 0;
        a[i] = in.fragment(in.a_at(i));
    }
    b[0] = in.fragment(in.b_at(0));
    b[1] = in.fragment(in.b_at(1));
    __builtin_amdgcn_sched_barrier(0);
    for (uint32_t s = 0; s < steps; s++)
        for_each_of([&](auto index) {
            constexpr int n = index, i = row_of(n), j = col_of(n);
            if constexpr (n == LAST) in.turn();
            add((n + COUNT - TM) % COUNT, n < TM);
            sum[n % TM] = mfma_f8<FA, FB>(b[j % PLACES], a[i]);
            // the scales of a group of columns, once the step before needs them no more: the last group's behind its last sums
            if constexpr (SQUARE && n == TM - 1)
#pragma unroll
                for (int g = 0; g < TN / S::TNG; g++)
#pragma unroll
                    for (int r = 0; r < TM; r++) scale[g][r] = in.sa[r] * in.sb[g];
            if constexpr (n < LAST && n % TM == 0 && j + 2 < TN) b[(j + 2) % PLACES] = in.fragment(in.b_at(j + 2));
            if constexpr (n >= LAST && n % 2 == 1) a[i] = in.fragment(in.a_at(i));
            if constexpr (PLACES == 4 && n == LAST) b[0] = in.fragment(in.b_at(0));
            if constexpr (PLACES == 4 && n == LAST + TM) b[1] = in.fragment(in.b_at(1));
            if constexpr (n == COUNT - 1) {
                if constexpr (PLACES == 2) {
                    b[0] = in.fragment(in.b_at(0));
                    b[1] = in.fragment(in.b_at(1));
                }
                if constexpr (!SQUARE) {
#pragma unroll
                    for (int r = 0; r < TM; r++) sa_before[r] = in.sa[r];
                    sb_before[0] = sb_rows[TN - 2];
                    sb_before[1] = sb_rows[TN - 1];
#pragma unroll
                    for (int c = 0; c < TN; c++) sb_rows[c] = in.row_scales(c);
                }
                in.read_scales();
            }
            constexpr int turn = (n + COUNT - LAST) % COUNT;
            if constexpr (turn % EVERY == 0)
#pragma unroll
                for (int c = turn / EVERY * AT_ONCE; c < (turn / EVERY + 1) * AT_ONCE && c < S::LOADS; c++) in.issue(s, n >= LAST ? S::STAGES : S::STAGES - 1, c);
            if constexpr (n % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, COUNT>{});
#pragma unroll
    for (int n = COUNT - TM; n < COUNT; n++) add(n, true);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <class S, bool SQUARE, bool WIDE, int FA, int FB>
__device__ __forceinline__ void f8_sums(f32x4 (&acc)[S::TM][S::TN], uint8_t *lds, const F8Loader<S> &load, uint32_t first, uint32_t steps, int lane, int wm, int wn) {
    if constexpr (WIDE) f8_sums_wide<S, SQUARE, FA, FB>(acc, lds, load, first, steps, lane, wm, wn);
    else f8_sums_narrow<S, SQUARE, FA, FB>(acc, lds, load, first, steps, lane, wm, wn);
}

// ------------------------------------------------------------------ up to sixteen rows of A

// As single tokens give them: B is what has to be read, once, at the rate of memory. A block takes 16 rows of B (of each of MATRICES); its waves take the windows of four steps in turn, each with LDS of its own, so that none waits
// for another before the sums are added, in wave order. Four steps of B and A are under way a wave; a step's place is filled again as soon as it has been read. One row through 4096 x 11008 10 us from memory that the last level of cache
// holds in part, 12.8 from HBM (3.5 TB/s), through 28672 x 8192 42 (5.6 TB/s). What the former waits for is not known: eight waves, with twice as much under way, take 13.0.
template <int WAVES, int MATRICES, bool EIGHT>
struct F8Few {
    typedef F8FewLoader<MATRICES, EIGHT> Loader;
    static constexpr int SIDES = Loader::SIDES, STEP = Loader::STEP, BYTES = WAVES * Loader::WAVE;

    // sum[x] of wave 0: of row ar = lane mod 16 of A with the rows n0 + 4 (lane / 16) to that + 3 of matrix x
    template <int FA, int FB>
    static __device__ __forceinline__ void sums(f32x4 (&sum)[MATRICES], const F8Side &a, const F8Side &b, const F8Side &b2, uint32_t steps, int64_t n0, uint8_t *lds, int lane, int wave) {
        const int q = lane >> 4, ar = lane & 15;
        uint8_t *mine = lds + wave * Loader::WAVE;
        const Loader load(a, b, b2, steps, n0, lane);
        int xa[2], xb[2];      // with eight rows of A lanes 8 to 15 take them again
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int place = EIGHT ? ar & 7 : ar;
            xa[h] = place * 128 + 16 * ((2 * q + h) ^ f8_rotated((place >> 1) & 7));
            xb[h] = ar * 128 + 16 * ((2 * q + h) ^ f8_rotated((ar >> 1) & 7));
        }
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
                    const uint8_t *at = mine + s * STEP + (i ? Loader::A_PLACES + 2048 * (i - 1) : 0);
                    lo[i] = *reinterpret_cast<const u32x4 *>(at + (i ? xb[0] : xa[0]));
                    hi[i] = *reinterpret_cast<const u32x4 *>(at + (i ? xb[1] : xa[1]));
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
                const bf16x8 fa[4] = {widened<FA>(lo[0].x, lo[0].y), widened<FA>(lo[0].z, lo[0].w), widened<FA>(hi[0].x, hi[0].y), widened<FA>(hi[0].z, hi[0].w)};
#pragma unroll
                for (int x = 0; x < MATRICES; x++) {
                    const u32x4 l = lo[1 + x], h = hi[1 + x];
                    const bf16x8 fb[4] = {widened<FB>(l.x, l.y), widened<FB>(l.z, l.w), widened<FB>(h.x, h.y), widened<FB>(h.z, h.w)};
                    f32x4 block{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 4; k++) block = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[k], fa[k], block, 0, 0, 0);
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
