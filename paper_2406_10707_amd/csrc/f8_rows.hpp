// Rounding of rows to 8 bits with a scale for 128 consecutive elements (include/ckpt_train.h).
#pragma once
#include <type_traits>

#include "f8_util.hpp"

namespace dsllm {

struct F8Source {
    const uint8_t *at;
    uint64_t ld;               // elements
    int64_t rows, cols;
    const float *scales;       // of a source in 8 bits
    uint64_t scale_pitch;
    uint32_t e5m2;
};

// A block of four waves takes 16 rows of 512 columns, a wave four of the rows, each with one load of all lanes: eight elements a lane, sixteen lanes a block of 128. The scales, which lie by blocks of columns, go out
// through LDS, sixteen neighbouring ones at a time. Bound by memory: 8192 x 4096 of bf16 17 us (5.9 TB/s).
template <int SRC>
__device__ __forceinline__ void f8_round_rows(const F8Source &src, const F8Held &to, int64_t row0, int64_t col0) {
    constexpr uint32_t kBytes = sizeof(typename Element<SRC>::one);
    __shared__ float scales[4][16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = col0 + 8 * lane;
    const float most = f8_most(to.e5m2);
    auto work = [&](auto whole) {
        Eight<SRC> x[4];
        const uint32_t count = whole ? 8 : col < src.cols ? uint32_t(min(src.cols - col, int64_t(8))) : 0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t row = row0 + 4 * wave + i;
            const uint8_t *at = src.at + (row * src.ld + col) * kBytes;
            if constexpr (whole) x[i].load(at);
            else x[i].load_upto(at, row < src.rows ? count : 0);
        }
        uint32_t amax = 0;      // of row lane mod 16 of the four: a scale's two divisions are some 25 instructions
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t found = most_of_16(bits_of(larger(larger(0, __builtin_convertvector(x[i].lo, f32x4)), __builtin_convertvector(x[i].hi, f32x4))));
            amax = (lane & 15) == uint32_t(i) ? found : amax;
        }
        const float mine = f8_inverse(amax, most), inverses[4] = {of_lane_of_16<0>(mine), of_lane_of_16<1>(mine), of_lane_of_16<2>(mine), of_lane_of_16<3>(mine)};
        if ((lane & 15) < 4) scales[lane >> 4][4 * wave + (lane & 15)] = f8_scale(amax, most);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t row = row0 + 4 * wave + i;
            const f32x4 lo = __builtin_convertvector(x[i].lo, f32x4), hi = __builtin_convertvector(x[i].hi, f32x4);
            if ((whole || row < src.rows) && col < to.cols + (-to.cols & 127)) {      // behind the last element zeros: they were loaded as such, but NaN times zero is no zero
                u32x2 codes{f8_codes(lo * inverses[i], to.e5m2), f8_codes(hi * inverses[i], to.e5m2)};
                if (count < 8) {
                    const uint64_t kept = (uint64_t(codes.y) << 32 | codes.x) & ((1ull << (8 * (count & 7))) - 1);
                    codes = u32x2{uint32_t(kept), uint32_t(kept >> 32)};
                }
                __builtin_nontemporal_store(codes, (u32x2 DSLLM_GLOBAL *)(to.codes + row * to.code_pitch + col));
            }
        }
    };
    if (row0 + 16 <= src.rows && col0 + 512 <= src.cols) work(std::true_type{});
    else work(std::false_type{});
    __syncthreads();
    if (threadIdx.x < 64) {
        const int64_t row = row0 + (lane & 15), block = col0 / 128 + (lane >> 4);
        if (row < to.rows && 128 * block < to.cols) ((float DSLLM_GLOBAL *)to.scales)[block * to.scale_pitch + row] = scales[lane >> 4][lane & 15];
    }
}

}  // namespace dsllm
