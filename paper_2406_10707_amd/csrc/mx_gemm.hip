// The product of two MXFP4 matrices on the matrix cores (include/ckpt_train.h).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 E2M1 values: lane l holds the 32 consecutive values (16 bytes) of row
// l mod 16 that make up block l / 16 of the step, and that block's scale byte. A and B are both kept by rows along K, so both sides
// are read the same way; the instruction applies the two scales of a block to its partial sum.
#include <algorithm>
#include <type_traits>

#include "gemm_tile.hpp"
#include "mx_gemm_loader.hpp"
#include "train_util.hpp"

using namespace dsllm;

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// BYTE: which byte of the scale operands counts
template <int BYTE>
__device__ __forceinline__ f32x4 mfma_fp4(u32x4 a, u32x4 b, f32x4 c, uint32_t a_scale, uint32_t b_scale) {
    const i32x8 a8{int(a.x), int(a.y), int(a.z), int(a.w), 0, 0, 0, 0}, b8{int(b.x), int(b.y), int(b.z), int(b.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, BYTE, int(a_scale), BYTE, int(b_scale));
}

// ------------------------------------------------------------------ tiles through LDS

template <int OUT>
__device__ __forceinline__ void store_eight(const GemmArgs &p, typename Element<OUT>::one *c, int64_t columns, f32x4 lo, f32x4 hi) {
    typedef typename Element<OUT>::one Out;
    if (columns <= 0) return;
    if (p.vector && columns >= 8) {
        if constexpr (OUT == CKPT_F32) {
            f32x4 DSLLM_GLOBAL *at = (f32x4 DSLLM_GLOBAL *)c;
            if (p.accumulate) { lo += at[0]; hi += at[1]; }
            at[0] = lo;
            at[1] = hi;
        } else {
            typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
            bf16x8 DSLLM_GLOBAL *at = (bf16x8 DSLLM_GLOBAL *)c;
            if (p.accumulate) {
                const bf16x8 old = *at;
                lo += __builtin_convertvector(__builtin_shufflevector(old, old, 0, 1, 2, 3), f32x4);
                hi += __builtin_convertvector(__builtin_shufflevector(old, old, 4, 5, 6, 7), f32x4);
            }
            *at = __builtin_shufflevector(__builtin_convertvector(lo, bf16x4), __builtin_convertvector(hi, bf16x4), 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if (e >= columns) return;
        Out DSLLM_GLOBAL *at = (Out DSLLM_GLOBAL *)c + e;
        *at = Out((e < 4 ? lo[e & 3] : hi[e & 3]) + (p.accumulate ? float(*at) : 0.0f));
    }
}

// Sixteen bytes of C, with what is there added.
template <int OUT>
__device__ __forceinline__ u32x4 sum_of_sixteen_bytes(u32x4 sum, u32x4 old) {
    if constexpr (OUT == CKPT_F32) return __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, sum) + __builtin_bit_cast(f32x4, old));
    else return sum;
}

// Four waves, WM x WN, each computing (16 TM) x (16 TN) of the block's tile; ONE wave per SIMD or two. Nothing hides a wait but the wave's own order, so the
// order is fixed by hand: a step of 256 values is 2 TM TN matrix instructions, and between them go the reads of the fragments (those of one half under
// the instructions of the half before, READS instructions apart, or -READS of them behind each) and the loads of a later step, one every LOAD_EVERY. Two steps are in LDS:
// once every wave has read its second half's fragments the stage is free and the loads of step + 2 into it start; three quarters into the step those of
// step + 1 have landed for all. (Four steps in LDS: the loads are those of step + 4.) Tiles of more than 32 accumulators a wave name them as AGPRs in the instruction's own operands.
//
// 8192^3 takes 226 to 254 us = 4.3 to 4.9 PFLOP/s with 256 x 256 tiles, from card to card (gemm_long_kernel 3590 us); at 237: a step 2670 cycles, of which the matrix instructions are 2048, at 1.73 GHz, which the power allows (2.1 GHz
// without the panels' loads and reads); some 7000 cycles in front of a tile's 32 steps (the first loads of all waves) and 9000 behind them (the stores of C). Scales fetched 16 bytes a row and step cost 14 us
// more, scales read from LDS at addresses of 2 bytes 150, pieces 2 q + h without the rotation (two lanes a bank) 15.
template <int WM, int WN, int TM, int TN, int STAGES, int READS, int LOAD_EVERY, int OUT>
__device__ __forceinline__ void gemm_tile_body(const GemmArgs &p, const TileOrder &order) {
    constexpr int NW = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN, FRAGS = TM + TN, HALF = TM * TN;
    constexpr bool NAMED = TM * TN > 32;
    typedef StepLoader<BM, BN, NW, STAGES> Loader;
    static_assert(TN % 2 == 0, "B fragments come in pairs");
    constexpr int PACE = READS > 0 ? READS : 1, AT_ONCE = READS > 0 ? 1 : -READS;
    constexpr int READ_SPAN = (FRAGS + AT_ONCE - 1) / AT_ONCE * PACE;
    constexpr int FREE_AT = READ_SPAN + 8 < HALF ? READ_SPAN + 8 : READ_SPAN + 4 < HALF ? READ_SPAN + 4 : HALF;
    constexpr int LANDED_AT = HALF + HALF / 2;
    constexpr int FITTING = (2 * HALF - FREE_AT + LOAD_EVERY - 1) / LOAD_EVERY;
    constexpr int GONE = (LANDED_AT - FREE_AT + LOAD_EVERY - 1) / LOAD_EVERY;
    static_assert(READ_SPAN <= HALF && FREE_AT <= HALF + 2, "the reads of a half lie inside the half before");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[Loader::BYTES];
    const GemmTile t = gemm_tile(order);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN, q = lane >> 4;
    const int64_t row = int64_t(t.tm) * BM, col = int64_t(t.tn) * BN;
    const Loader load(p, row, col, lane, wave);
    const int ar = lane & 15, br = 8 * (ar >> 2) + (ar & 3);
    int at_a[2], at_b[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        at_a[h] = (16 * TM * wm + ar) * 128 + 16 * ((2 * q + h) ^ rotated((ar >> 1) & 7));
        at_b[h] = (BM + 16 * TN * wn + br) * 128 + 16 * ((2 * q + h) ^ rotated(((ar >> 1) & 1) | ((ar >> 2) << 1)));
    }
    const int at_sa = Loader::scale_at(16 * TM * wm + ar) + 4 * (q >> 1), at_sb = Loader::scale_at(BM + 16 * TN * wn + ar) + 4 * (q >> 1);
    const uint32_t down = 16 * (q & 1);
    u32x4 frag[2][FRAGS];      // [half of the step]: B fragments first, then A
    uint32_t scale[2][FRAGS];  // [step's parity]: the two halves' bytes lowest, once shifted down
    auto read = [&](int half, int stage, int i) {
        const uint8_t *at = lds + stage * Loader::PANEL + (i < TN ? at_b[half] + (i >> 1) * 4096 + (i & 1) * 512 : at_a[half] + (i - TN) * 2048);
        frag[half][i] = *reinterpret_cast<const u32x4 *>(at);
    };
    // of a step, the `turn`th of its window
    auto read_scale = [&](int to, uint32_t window, int turn, int i) {
        const int of_step = (turn >> 1) * 128 + (turn & 1) * 8;
        const uint8_t *at = lds + (window & 1) * Loader::SCALES + (i < TN ? (at_sb ^ of_step) + i * 512 : (at_sa ^ of_step) + (i - TN) * 512);
        scale[to][i] = *reinterpret_cast<const uint32_t *>(at);
    };
    // with named accumulators pinned where it stands: no matrix instruction in asm may follow at once that reads it
    auto shift_scale = [&](int which, int i) {
        if constexpr (NAMED) asm volatile("v_lshrrev_b32 %0, %1, %0" : "+v"(scale[which][i]) : "v"(down));
        else scale[which][i] >>= down;
    };
    // fragment i of the next step's first half is read behind matrix instruction READ_AT(i) of this step, its scales are shifted SHIFT_LATER instructions after that
    constexpr int SHIFT_LATER = NAMED ? 8 : 4;
    auto read_at = [](int i) constexpr { return LANDED_AT + i / AT_ONCE * PACE; };
    auto shift_at = [=](int i) constexpr { return read_at(i) + SHIFT_LATER; };
    static_assert(!NAMED || [](auto at) constexpr {      // fragment i (A's from TN on) first counts in instruction i (TN (i - TN)) of the next step
        for (int i = 0; i < FRAGS; i++)
            if (at(i) >= 2 * HALF + (i < TN ? 0 : TN * (i - TN)) - 1) return false;
        return true;
    }(shift_at), "scales are shifted before they count");
    const uint32_t first = blockIdx.y * p.steps_a_split, steps = min(p.steps - first, p.steps_a_split);
    load.issue_first(lds, first, steps);
    __builtin_amdgcn_sched_barrier(0);      // the loads go out first
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    wait_loads_and_meet<(STAGES - 1) * Loader::PANELS + 1>();
#pragma unroll
    for (int i = 0; i < FRAGS; i++) { read(0, 0, i); read_scale(0, 0, 0, i); }
#pragma unroll
    for (int i = 0; i < FRAGS; i++)
        if (!NAMED || shift_at(i) < 2 * HALF) shift_scale(0, i);
    if constexpr (NAMED) {
        // set by ordinary instructions, read by the asm below, for which the compiler inserts no wait states
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) asm volatile("" : "+a"(acc[i][j]));
        asm volatile("s_nop 7");
    }
    __builtin_amdgcn_sched_barrier(0);
    auto do_step = [&](auto turn_, uint32_t window) {
        constexpr int turn = turn_, stage = turn % STAGES, next = (turn + 1) % STAGES, now = turn & 1, COUNT = Loader::loads_of(turn);
        constexpr int UNDER_WAY = (GONE < COUNT ? GONE : COUNT) + (STAGES == 4 ? Loader::loads_of(turn + 3) + Loader::loads_of(turn + 2) : 0);
        const uint32_t window_next = window + (turn + 1) / 4;
        for_each_of([&](auto index) {
            constexpr int at = index, half = at / HALF, i = at % HALF / TN, j = i & 1 ? TN - 1 - at % TN : at % TN;
            if constexpr (at == FREE_AT) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if constexpr (at == LANDED_AT) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(UNDER_WAY) : "memory");
            if constexpr (NAMED && half == 0)
                asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                             : "+a"(acc[i][j]) : "v"(frag[half][j]), "v"(frag[half][TN + i]), "v"(scale[now][j]), "v"(scale[now][TN + i]));
            else if constexpr (NAMED)
                asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                             : "+a"(acc[i][j]) : "v"(frag[half][j]), "v"(frag[half][TN + i]), "v"(scale[now][j]), "v"(scale[now][TN + i]));
            else acc[i][j] = mfma_fp4<half>(frag[half][j], frag[half][TN + i], acc[i][j], scale[now][j], scale[now][TN + i]);
#pragma unroll
            for (int u = 0; u < AT_ONCE; u++) {
                if (at < HALF && at % PACE == 0 && at / PACE * AT_ONCE + u < FRAGS) read(1, stage, at / PACE * AT_ONCE + u);
                if (at >= LANDED_AT && (at - LANDED_AT) % PACE == 0 && (at - LANDED_AT) / PACE * AT_ONCE + u < FRAGS) {
                    read(0, next, (at - LANDED_AT) / PACE * AT_ONCE + u);
                    read_scale(now ^ 1, window_next, (turn + 1) % 4, (at - LANDED_AT) / PACE * AT_ONCE + u);
                }
            }
#pragma unroll
            for (int f = 0; f < FRAGS; f++) {
                if (shift_at(f) == at) shift_scale(now ^ 1, f);
                if (NAMED && shift_at(f) == at + 2 * HALF) shift_scale(now, f);      // of the reads of the step before
            }
            if constexpr (at >= FREE_AT && (at - FREE_AT) % LOAD_EVERY == 0 && (at - FREE_AT) / LOAD_EVERY < COUNT)
                load.template issue<turn>(lds, first, steps, window, (at - FREE_AT) / LOAD_EVERY);
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, 2 * HALF>{});
        // what there was no matrix instruction left for
#pragma unroll
        for (int i = FITTING; i < COUNT; i++) load.template issue<turn>(lds, first, steps, window, i);
#pragma unroll
        for (int i = (2 * HALF - LANDED_AT + PACE - 1) / PACE * AT_ONCE; i < FRAGS; i++) { read(0, next, i); read_scale(now ^ 1, window_next, (turn + 1) % 4, i); }
        if constexpr (!NAMED)
#pragma unroll
            for (int i = 0; i < FRAGS; i++)
                if (shift_at(i) >= 2 * HALF) shift_scale(now ^ 1, i);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (uint32_t window = 0;; window++) {
        do_step(std::integral_constant<int, 0>{}, window);
        if (4 * window + 1 == steps) break;
        do_step(std::integral_constant<int, 1>{}, window);
        if (4 * window + 2 == steps) break;
        do_step(std::integral_constant<int, 2>{}, window);
        if (4 * window + 3 == steps) break;
        do_step(std::integral_constant<int, 3>{}, window);
        if (4 * window + 4 == steps) break;
    }
    // the last matrix instructions' results are readable, and no load to LDS outlives the block
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_waitcnt vmcnt(0)" ::: "memory");
    typedef typename Element<OUT>::one Out;
    const int64_t part = blockIdx.y * p.c_split;
    if (p.vector && row + BM <= p.m && col + BN <= p.n) {
        // A whole tile goes through LDS, which is free now, so that a store is whole lines of C by neighbouring lanes (straight from the registers neighbouring lanes have different rows): 16384 x 16384 x 4096
        // 614 -> 573 us, 8192^3 to f32 275 -> 268 (other cards 254 and 273), 2304 x 768 x 8190 added to f32 17.7 -> 17.1, 1000 x 2304 x 768 to f32 6.6 -> 6.1, 8192^3 to bf16 even, 4096^3 36.2 -> 36.7. A wave has a part of
        // its own, rows of CP pieces of 16 bytes, of which CH are used; piece p of row r lies at place p ^ f(r). Few instructions a store: with the bounds of each beside it this was 40 KB of
        // code that every block fetched anew.
        constexpr int CH = OUT == CKPT_F32 ? 4 * TN : 2 * TN, CP = CH <= 4 ? 4 : CH <= 8 ? 8 : CH <= 16 ? 16 : 32, SHIFT = CP >= 16 ? 0 : CP == 8 ? 1 : 2, MASK = CP >= 16 ? 15 : CP - 1;
        constexpr int PART = Loader::BYTES / NW, FIT = PART / (16 * 16 * CP), AT_A_TIME = FIT < TM ? FIT : TM, ROWS = 64 / CP;
        static_assert(FIT >= 1 && PART % 16 == 0, "sixteen rows fit a wave's part");
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // no wave reads its panels any more, and all loads to LDS are over
        uint8_t *mine = lds + wave * PART;
        Out *tile = static_cast<Out *>(p.c) + part + row * p.ldc + col;
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(tile, 0, 0xFFFFFFFFu, 0x00020000);
        const uint32_t pitch = uint32_t(p.ldc) * sizeof(Out), piece = lane & (CP - 1), lane_row = lane / CP;
        const uint32_t lane_at = (wm * 16 * TM + lane_row) * pitch + wn * 16 * TN * sizeof(Out) + 16 * piece;
        auto store_tile = [&](auto add) {
#pragma unroll
            for (int i0 = 0; i0 < TM; i0 += AT_A_TIME) {
#pragma unroll
                for (int i = i0; i < i0 + AT_A_TIME && i < TM; i++)
#pragma unroll
                    for (int j = 0; j < TN; j += 2) {
                        // in their registers up to here: copied out all at once they would spill
                        if constexpr (NAMED) asm volatile("" : "+a"(acc[i][j]), "+a"(acc[i][j + 1]));
                        uint8_t *at = mine + (16 * (i - i0) + ar) * (16 * CP);
                        const int f = (ar >> SHIFT) & MASK;
                        if constexpr (OUT == CKPT_F32) {
                            *reinterpret_cast<f32x4 *>(at + 16 * ((4 * j + 2 * q) ^ f)) = acc[i][j];
                            *reinterpret_cast<f32x4 *>(at + 16 * ((4 * j + 2 * q + 1) ^ f)) = acc[i][j + 1];
                        } else {
                            f32x4 lo = acc[i][j], hi = acc[i][j + 1];
                            if constexpr (add) {      // before the rounding
                                const uint32_t there = (wm * 16 * TM + ar) * pitch + (wn * 16 * TN + 16 * j + 8 * q) * sizeof(Out);
                                typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
                                const bf16x8 old = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rc, there, 16 * i * pitch, 0));
                                lo += __builtin_convertvector(__builtin_shufflevector(old, old, 0, 1, 2, 3), f32x4);
                                hi += __builtin_convertvector(__builtin_shufflevector(old, old, 4, 5, 6, 7), f32x4);
                            }
                            typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
                            *reinterpret_cast<bf16x8 *>(at + 16 * ((2 * j + q) ^ f)) =
                                __builtin_shufflevector(__builtin_convertvector(lo, bf16x4), __builtin_convertvector(hi, bf16x4), 0, 1, 2, 3, 4, 5, 6, 7);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                asm volatile("" ::: "memory");      // other lanes' writes are read: a wave's go to LDS in the order of the program, which the compiler must not change
                constexpr int COUNT = 16 * AT_A_TIME / ROWS, BATCH = 8;
                const int left = (TM - i0 < AT_A_TIME ? 16 * (TM - i0) : 16 * AT_A_TIME) / ROWS;
#pragma unroll
                for (int t0 = 0; t0 < COUNT; t0 += BATCH) {
                    if (t0 >= left) break;
                    u32x4 old[BATCH], sum[BATCH];
                    if (CH < CP && piece >= CH) continue;
                    if constexpr (add && OUT == CKPT_F32)
#pragma unroll
                        for (int t = 0; t < BATCH; t++)
                            if (t0 + t < left) old[t] = __builtin_amdgcn_raw_buffer_load_b128(rc, lane_at, (16 * i0 + ROWS * (t0 + t)) * pitch, 0);
#pragma unroll
                    for (int t = 0; t < BATCH; t++) {
                        const int r = ROWS * (t0 + t) + lane_row;
                        if (t0 + t < left) sum[t] = *reinterpret_cast<const u32x4 *>(mine + r * (16 * CP) + 16 * (piece ^ ((r >> SHIFT) & MASK)));
                    }
#pragma unroll
                    for (int t = 0; t < BATCH; t++)
                        if (t0 + t < left) {
                            if constexpr (add && OUT == CKPT_F32) sum[t] = sum_of_sixteen_bytes<OUT>(sum[t], old[t]);
                            __builtin_amdgcn_raw_buffer_store_b128(sum[t], rc, lane_at, (16 * i0 + ROWS * (t0 + t)) * pitch, 0);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
                asm volatile("" ::: "memory");
            }
        };
        if (p.accumulate) store_tile(std::true_type{});
        else store_tile(std::false_type{});
        return;
    }
    const int64_t c_row = row + wm * 16 * TM + ar, c_col = col + wn * 16 * TN + 8 * q;
    Out *c = static_cast<Out *>(p.c) + part + c_row * p.ldc + c_col;
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const bool inside = c_row + 16 * i < p.m;
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
            if constexpr (NAMED) asm volatile("" : "+a"(acc[i][j]), "+a"(acc[i][j + 1]));
            if (inside) store_eight<OUT>(p, c + 16 * i * p.ldc + 16 * j, p.n - c_col - 16 * j, acc[i][j], acc[i][j + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// TOGETHER blocks share a compute unit. The bodies are the device's only: the host's pass needs no more than the names.
template <int TOGETHER, int WM, int WN, int TM, int TN, int STAGES, int READS, int LOAD_EVERY, int OUT>
__global__ __launch_bounds__(256, TOGETHER) void gemm_tile_kernel(GemmArgs p, TileOrder order) {
#if defined(__HIP_DEVICE_COMPILE__)
    gemm_tile_body<WM, WN, TM, TN, STAGES, READS, LOAD_EVERY, OUT>(p, order);
#endif
}

// ------------------------------------------------------------------ up to sixteen rows of A

// As single tokens give them: B is what has to be read, once, at the rate of memory. A block takes 16 rows of B; its WAVES waves take the windows of four steps in turn, each with LDS of its own, so that
// none waits for another before the sums are added, in wave order. Four steps of B and A are under way a wave; a step's place is filled again as soon as it has been read. LDS layouts as above (16 rows
// of B, 16 of A, whose last is repeated where there are fewer; in the scales' window rows 16 to 31 are A's). Addresses are 64-bit ones.
//
// One token, launched in a row: 16384 x 16384 26 us = 5.4 TB/s (64 x 64 tiles 31), 4096 x 16384 8.2 (tiles 15.2, in four parts 10.9), 11008 x 4096 5.9 with two waves (four 6.4, tiles 6.1); below that the
// launches are what counts (4.5 us). Sixteen rows: 27.5, 8.8, 5.9. Fragments read straight from memory took 33, 11.7 and 7.4: sixteen lines a request.
template <int WAVES, int OUT>
__global__ __launch_bounds__(64 * WAVES) void gemm_few_kernel(GemmArgs p) {
    constexpr int STEP = 2 * 16 * 128, SCALES = 32 * 32, WAVE = 4 * STEP + 2 * SCALES;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[WAVES * WAVE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, ar = lane & 15;
    uint8_t *mine = lds + wave * WAVE;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const uint8_t *from[4];      // this lane's piece of the rows lane / 8 of B, those 8 further, and of A's
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int r = 8 * (i & 1) + (lane >> 3);
        const uint32_t piece = 16 * ((lane & 7) ^ rotated((r >> 1) & 7));
        from[i] = (i < 2 ? p.b + min(n0 + r, p.n - 1) * p.b_pitch : p.a + min(int64_t(r), p.m - 1) * p.a_pitch) + piece;
    }
    const int sr = 8 * (lane >> 4) + (lane & 7);
    const uint8_t *scales_from = sr < 16 ? p.b_scale + min(n0 + sr, p.n - 1) * p.b_scale_pitch : p.a_scale + min(int64_t(sr - 16), p.m - 1) * p.a_scale_pitch;
    const uint32_t scale_half = 16 * (((lane >> 3) ^ (lane >> 4)) & 1), last_scales = uint32_t(sr < 16 ? p.b_scale_pitch : p.a_scale_pitch) - 16;
    auto issue_scales = [&](uint32_t window, uint32_t odd) {      // what a row has behind its end is not used, and not read
        const uint8_t *at = scales_from + min(32 * window + scale_half, last_scales);
        __builtin_amdgcn_global_load_lds((const DSLLM_GLB void *)at, (DSLLM_LDS void *)(mine + 4 * STEP + (odd & 1) * SCALES), 16, 0, 0);
    };
    auto issue_step = [&](uint32_t window, int s) {
        const uint64_t at = 128 * uint64_t(min(4 * window + s, p.steps - 1));
#pragma unroll
        for (int i = 0; i < 4; i++) __builtin_amdgcn_global_load_lds((const DSLLM_GLB void *)(from[i] + at), (DSLLM_LDS void *)(mine + s * STEP + 1024 * i), 16, 0, 0);
    };
    const int frag_at = ar * 128, swizzle = rotated((ar >> 1) & 7);
    const int scale_at_b = (ar >> 3) * 256 + ((ar >> 3) & 1) * 128 + (ar & 7) * 16 + 4 * (q >> 1), scale_at_a = scale_at_b + 512;
    const uint32_t down = 16 * (q & 1), windows = (p.steps + 3) / 4;
    f32x4 acc = {};
    auto do_window = [&](auto more, uint32_t window, uint32_t odd) {
#pragma unroll
        for (int s = 0; s < 4; s++) {
            // this step's loads have landed; those of the later ones, and what has been asked for of the next window, may be under way
            if constexpr (more) { if (s == 0) asm volatile("s_waitcnt vmcnt(12)" ::: "memory"); else asm volatile("s_waitcnt vmcnt(13)" ::: "memory"); }
            else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * (3 - s)) : "memory");
            u32x4 fb[2], fa[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                fb[h] = *reinterpret_cast<const u32x4 *>(mine + s * STEP + frag_at + 16 * ((2 * q + h) ^ swizzle));
                fa[h] = *reinterpret_cast<const u32x4 *>(mine + s * STEP + 2048 + frag_at + 16 * ((2 * q + h) ^ swizzle));
            }
            const uint8_t *sc = mine + 4 * STEP + (odd & 1) * SCALES;
            const int of_step = (s >> 1) * 128 + (s & 1) * 8;
            uint32_t sb = *reinterpret_cast<const uint32_t *>(sc + (scale_at_b ^ of_step)), sa = *reinterpret_cast<const uint32_t *>(sc + (scale_at_a ^ of_step));
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(fb[0]), "+v"(fb[1]), "+v"(fa[0]), "+v"(fa[1]), "+v"(sb), "+v"(sa)::"memory");
            if constexpr (more) {
                if (s == 0) issue_scales(window + WAVES, odd + 1);
                issue_step(window + WAVES, s);
            }
            if (4 * window + s >= p.steps) continue;
            acc = mfma_fp4<0>(fb[0], fa[0], acc, sb >> down, sa >> down);
            acc = mfma_fp4<1>(fb[1], fa[1], acc, sb >> down, sa >> down);
        }
    };
    if (uint32_t(wave) < windows) {
        issue_scales(wave, 0);
#pragma unroll
        for (int s = 0; s < 4; s++) issue_step(wave, s);
        uint32_t window = wave, odd = 0;
        for (; window + WAVES < windows; window += WAVES, odd++) do_window(std::true_type{}, window, odd);
        do_window(std::false_type{}, window, odd);
    }
    __syncthreads();
    f32x4 *part = reinterpret_cast<f32x4 *>(lds);
    if (wave > 0) part[(wave - 1) * 64 + lane] = acc;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < WAVES - 1; w++) acc += part[w * 64 + lane];
    typedef typename Element<OUT>::one Out;
    const int64_t first_col = n0 + 4 * q;
    if (ar >= p.m || first_col >= p.n) return;
    Out *c = static_cast<Out *>(p.c) + ar * p.ldc + first_col;
    const uint32_t count = uint32_t(min(p.n - first_col, int64_t(4)));
    if (p.accumulate) acc += load_upto4<OUT>(c, count);
    store_upto4<OUT>(c, acc, count);
}

// For rows of more than 2^23 bytes, which the loads above cannot address: four waves compute 64 x 64, a wave 32 x 32, straight from memory with 64-bit addresses. Rows
// past the end are the last row again, and not stored.
template <int OUT>
__global__ __launch_bounds__(256) void gemm_long_kernel(GemmArgs p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
    const int64_t row0 = int64_t(blockIdx.y) * 64 + 32 * (wave & 1), col0 = int64_t(blockIdx.x) * 64 + 32 * (wave >> 1);
    const uint8_t *a[2], *b[2], *as[2], *bs[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int64_t r = min(row0 + 16 * i + (lane & 15), p.m - 1), c = min(col0 + 16 * i + (lane & 15), p.n - 1);
        a[i] = p.a + r * p.a_pitch + 16 * q;
        b[i] = p.b + c * p.b_pitch + 16 * q;
        as[i] = p.a_scale + r * p.a_scale_pitch + q;
        bs[i] = p.b_scale + c * p.b_scale_pitch + q;
    }
    f32x4 acc[2][2] = {};
    for (uint32_t s = 0; s < 2 * p.steps; s++) {
        u32x4 fa[2], fb[2];
        uint32_t sa[2], sb[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            fa[i] = *(const u32x4 DSLLM_GLOBAL *)(a[i] + 64ull * s);
            fb[i] = *(const u32x4 DSLLM_GLOBAL *)(b[i] + 64ull * s);
            sa[i] = *(const uint8_t DSLLM_GLOBAL *)(as[i] + 4ull * s);
            sb[i] = *(const uint8_t DSLLM_GLOBAL *)(bs[i] + 4ull * s);
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++) acc[i][j] = mfma_fp4<0>(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
    }
    typedef typename Element<OUT>::one Out;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int64_t r = row0 + 16 * i + (lane & 15), c = col0 + 16 * j + 4 * q + e;
                if (r >= p.m || c >= p.n) continue;
                Out DSLLM_GLOBAL *at = (Out DSLLM_GLOBAL *)p.c + r * p.ldc + c;
                *at = Out(acc[i][j][e] + (p.accumulate ? float(*at) : 0.0f));
            }
}

// The product in parts of at most `rows` x `columns` of C, a launch each: one grid has fewer than 2^32 work-items along each axis, and 65535 blocks down.
template <int OUT, class F>
void launch_in_parts(const GemmArgs &p, int64_t rows, int64_t columns, F launch) {
    for (int64_t row = 0; row < p.m; row += rows)
        for (int64_t col = 0; col < p.n; col += columns) {
            GemmArgs part = p;
            part.a += row * p.a_pitch;
            part.b += col * p.b_pitch;
            part.a_scale += row * p.a_scale_pitch;
            part.b_scale += col * p.b_scale_pitch;
            part.c = static_cast<typename Element<OUT>::one *>(p.c) + row * p.ldc + col;
            part.m = std::min(rows, p.m - row);
            part.n = std::min(columns, p.n - col);
            launch(part);
        }
}

template <int OUT>
void launch_few(uint32_t waves, const GemmArgs &p, hipStream_t stream) {
    launch_in_parts<OUT>(p, 16, 16ll << 23, [&](const GemmArgs &part) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned((part.n + 15) / 16)), dim3(64 * waves), 0, stream, part); };
        if (waves == 2) go(gemm_few_kernel<2, OUT>);
        else go(gemm_few_kernel<4, OUT>);
    });
}

template <int OUT>
void launch_long(const GemmArgs &p, hipStream_t stream) {
    launch_in_parts<OUT>(p, 64ll << 15, 64ll << 23, [&](const GemmArgs &part) {
        hipLaunchKernelGGL(gemm_long_kernel<OUT>, dim3(unsigned((part.n + 63) / 64), unsigned((part.m + 63) / 64)), dim3(256), 0, stream, part);
    });
}

// The parts' sums of a product whose K was split, added in order. Rows of the parts are `pitch` elements apart, a multiple of 4.
template <int OUT>
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ parts, uint32_t splits, int64_t split, uint32_t pitch, GemmArgs p) {
    const uint64_t t = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    const uint32_t quads = pitch / 4, row = uint32_t(t / quads), col = 4 * uint32_t(t - uint64_t(row) * quads);
    if (row >= p.m) return;
    const float *at = parts + int64_t(row) * pitch + col;
    f32x4 sum = *(const f32x4 DSLLM_GLOBAL *)at;
    for (uint32_t s = 1; s < splits; s++) sum += *(const f32x4 DSLLM_GLOBAL *)(at + s * split);
    typedef typename Element<OUT>::one Out;
    Out *c = static_cast<Out *>(p.c) + row * p.ldc + col;
    const uint32_t count = uint32_t(min(p.n - col, int64_t(4)));
    if (p.accumulate) sum += load_upto4<OUT>(c, count);
    store_upto4<OUT>(c, sum, count);
}

// In the order of kMxGemmForms
template <int OUT>
void launch_form(int form, uint32_t splits, const GemmArgs &p, hipStream_t stream) {
    const MxGemmForm &f = kMxGemmForms[form];
    const uint32_t tiles_m = uint32_t((p.m + f.bm - 1) / f.bm), tiles_n = uint32_t((p.n + f.bn - 1) / f.bn);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(tiles_m * tiles_n, splits), dim3(256), 0, stream, p, TileOrder(tiles_m, tiles_n, true)); };
    switch (form) {
        case 0: go(gemm_tile_kernel<1, 2, 2, 8, 8, 2, 2, 4, OUT>); break;
        case 1: go(gemm_tile_kernel<1, 2, 2, 6, 6, 2, 1, 3, OUT>); break;
        case 2: go(gemm_tile_kernel<2, 2, 2, 4, 4, 2, 1, 1, OUT>); break;
        case 3: go(gemm_tile_kernel<2, 2, 2, 2, 4, 2, -2, 1, OUT>); break;
        case 4: go(gemm_tile_kernel<2, 2, 2, 2, 2, 4, -2, 1, OUT>); break;
        default: go(gemm_tile_kernel<3, 2, 2, 2, 2, 2, -2, 1, OUT>); break;
    }
}

int gemm(const ckpt_mx_matrix *a, const ckpt_mx_matrix *b, void *c, int32_t dtype, int64_t ldc, int32_t accumulate, void *workspace, uint64_t workspace_bytes,
         hipStream_t stream) {
    if (!a || !b) return refuse(CKPT_EINVAL, "null argument");
    if (dtype != CKPT_F32 && dtype != CKPT_BF16) return refuse(CKPT_EINVAL, "c_dtype must be CKPT_F32 or CKPT_BF16");
    DeviceRanges ranges;
    if (a->format != CKPT_MXFP4 || b->format != CKPT_MXFP4) return refuse(CKPT_EINVAL, "A and B must be CKPT_MXFP4");
    if (const char *why = wrong_mx_matrix(a, ranges)) return refuse(CKPT_EINVAL, std::string("A: ") + why);
    if (const char *why = wrong_mx_matrix(b, ranges)) return refuse(CKPT_EINVAL, std::string("B: ") + why);
    if (a->cols != b->cols) return refuse(CKPT_EINVAL, "A and B differ in their columns");
    const int64_t m = a->rows, n = b->rows, k = a->cols;
    if (m > 0x7FFFFFFF || n > 0x7FFFFFFF || k > 0x7FFFFFFF) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1");
    if (m == 0 || n == 0) return CKPT_OK;
    const uint32_t bytes = element_bytes(dtype);
    if (ldc < n || ldc > (1ll << 48) / m) return refuse(CKPT_EINVAL, "ldc is smaller than a row, or C too large");
    if (uint64_t(c) % bytes) return refuse(CKPT_EINVAL, "C is not aligned to its element");
    if (const char *why = ranges.wrong(c, (uint64_t(m - 1) * ldc + n) * bytes)) return refuse(CKPT_EINVAL, std::string("C: ") + why);
    const bool vector = uint64_t(c) % 16 == 0 && ldc * bytes % 16 == 0 && ldc <= 1 << 21;      // 256 rows in 32-bit offsets
    const uint32_t steps = uint32_t((k + 255) / 256);
    GemmArgs p{static_cast<const uint8_t *>(a->codes), static_cast<const uint8_t *>(b->codes), static_cast<const uint8_t *>(a->scales), static_cast<const uint8_t *>(b->scales),
               a->code_pitch, b->code_pitch, a->scale_pitch, b->scale_pitch, c, ldc, m, n, steps, steps, 0, accumulate, vector};
    if (const uint32_t waves = steps ? mx_gemm_few_waves(uint64_t(m), steps) : 0) {
        if (dtype == CKPT_F32) launch_few<CKPT_F32>(waves, p, stream);
        else launch_few<CKPT_BF16>(waves, p, stream);
        return launched();
    }
    const bool loadable = a->code_pitch <= 1u << 23 && b->code_pitch <= 1u << 23 && a->scale_pitch <= 1u << 23 && b->scale_pitch <= 1u << 23;
    MxGemmChoice choice = steps && loadable ? mx_gemm_choice(uint64_t(m), uint64_t(n), uint64_t(k), dtype == CKPT_F32, workspace ? workspace_bytes : 0) : MxGemmChoice{-1, 1};
    if (choice.splits > 1) {
        const uint64_t bytes_needed = mx_gemm_part_bytes(uint64_t(m), uint64_t(n)) * choice.splits;
        if (uint64_t(workspace) % 16) return refuse(CKPT_EINVAL, "workspace must be 16-byte aligned");
        if (const char *why = ranges.wrong(workspace, bytes_needed)) return refuse(CKPT_EINVAL, std::string("workspace: ") + why);
        const uint32_t pitch = uint32_t(mx_gemm_part_pitch(uint64_t(n)));
        GemmArgs parts = p;
        parts.c = workspace;
        parts.ldc = pitch;
        parts.accumulate = 0;
        parts.vector = pitch <= 1 << 21;
        parts.c_split = m * pitch;
        parts.steps_a_split = mx_gemm_steps_a_split(steps, choice.splits);
        launch_form<CKPT_F32>(choice.form, choice.splits, parts, stream);
        const uint64_t threads = uint64_t(m) * (pitch / 4);
        auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned((threads + 255) / 256)), dim3(256), 0, stream, static_cast<const float *>(workspace), choice.splits, parts.c_split, pitch, p); };
        if (dtype == CKPT_F32) join(join_kernel<CKPT_F32>);
        else join(join_kernel<CKPT_BF16>);
        return launched();
    }
    if (choice.form >= 0) {
        if (dtype == CKPT_F32) launch_form<CKPT_F32>(choice.form, 1, p, stream);
        else launch_form<CKPT_BF16>(choice.form, 1, p, stream);
        return launched();
    }
    if (dtype == CKPT_F32) launch_long<CKPT_F32>(p, stream);
    else launch_long<CKPT_BF16>(p, stream);
    return launched();
}

}  // namespace

extern "C" {

int ckpt_mx_gemm_workspace(int64_t m, int64_t n, int64_t k, uint64_t *bytes) {
    return at_c_entry([&] {
        if (!bytes || m < 0 || n < 0 || k < 0) return refuse(CKPT_EINVAL, "null argument or negative size");
        *bytes = 0;
        if (m > 0x7FFFFFFF || n > 0x7FFFFFFF || k > 0x7FFFFFFF) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1");
        if (!m || !n || !k || mx_gemm_few_waves(uint64_t(m), uint32_t((k + 255) / 256))) return int(CKPT_OK);
        for (bool f32 : {false, true}) {
            const MxGemmChoice c = mx_gemm_choice(uint64_t(m), uint64_t(n), uint64_t(k), f32, UINT64_MAX);
            if (c.splits > 1) *bytes = std::max(*bytes, mx_gemm_part_bytes(uint64_t(m), uint64_t(n)) * c.splits);
        }
        return int(CKPT_OK);
    });
}

int ckpt_mx_gemm(const ckpt_mx_matrix *a, const ckpt_mx_matrix *b, void *c, int32_t c_dtype, int64_t ldc, int32_t accumulate, void *workspace,
                 uint64_t workspace_bytes, void *stream) {
    return at_c_entry([&] { return gemm(a, b, c, c_dtype, ldc, accumulate, workspace, workspace_bytes, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
