// What the matrix products share: which tile of C a block computes, and how its waves meet.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <utility>

namespace dsllm {

#define DSLLM_LDS __attribute__((address_space(3)))
#define DSLLM_GLB __attribute__((address_space(1)))

struct GemmTile { int tm, tn; };

// Which tile a block computes. Consecutive block ids go to different XCDs (8 of them, each with its own L2): each XCD is given
// a contiguous range of tiles, walked in strips 8 tiles tall so that neighbours share A and B panels. With a short K the
// stores of C are what counts, and those go better in block order where 8 does not divide the number of tiles (7808 x 3968 x
// 128 18.2 us, by XCD 18.9).
// The host prepares the divisions: three of them, on scalars, were 90 of the 150 instructions in front of a block's first load
// (and a branch costs some 40 cycles, so there is none). Products of 4 to 6 us take 4 % less than with divisions in the kernel, of
// 6 to 10 us 2 %, of 10 to 20 us 1 % (300 products; 1024 x 3072 x 768 7.7 -> 7.5 us, 896 x 3072 x 64 4.1 -> 3.5); those of
// 3 us are bound by the launches.
struct TileOrder {
    uint32_t xcd_bits, xcd_shift;            // of a block id: its XCD, what is left of it (0, 0: tiles go in the blocks' own order)
    uint32_t each, more;                     // tiles of every XCD; how many XCDs have one tile more
    uint32_t per_strip, strip_inverse;       // tiles of a full strip
    uint32_t full_strips, last_rows, last_inverse;       // the last strip may be less than 8 tall

    static uint32_t inverse(uint32_t d) { return 0xFFFFFFFFu / d; }
    // x / d: the upper half of x times the inverse is that or one less
    static __host__ __device__ __forceinline__ uint32_t divided(uint32_t x, uint32_t d, uint32_t inverse) {
        const uint32_t q = uint32_t((uint64_t(x) * inverse) >> 32);
        return x - q * d >= d ? q + 1 : q;
    }
    TileOrder(uint32_t tiles_m, uint32_t tiles_n, bool by_xcd) {
        const uint32_t n = tiles_m * tiles_n;
        const bool in_order = !by_xcd && n % 8;
        xcd_bits = in_order ? 0 : 7;
        xcd_shift = in_order ? 0 : 3;
        each = n / 8;
        more = n % 8;
        per_strip = 8 * tiles_n;
        strip_inverse = inverse(per_strip);
        full_strips = tiles_m / 8;
        last_rows = tiles_m % 8 ? tiles_m % 8 : 8;
        last_inverse = inverse(last_rows);
    }
};

__device__ __forceinline__ GemmTile gemm_tile(const TileOrder &o, uint32_t block = blockIdx.x) {
    const uint32_t xcd = block & o.xcd_bits, tile = xcd * o.each + min(xcd, o.more) + (block >> o.xcd_shift);
    const uint32_t s = TileOrder::divided(tile, o.per_strip, o.strip_inverse), in_s = tile - s * o.per_strip;
    const uint32_t rows_here = s < o.full_strips ? 8 : o.last_rows;
    const uint32_t col = TileOrder::divided(in_s, rows_here, s < o.full_strips ? 1u << 29 : o.last_inverse);
    return GemmTile{int(8 * s + in_s - col * rows_here), int(col)};
}

// This wave's loads are in LDS but for the latest N, its LDS reads are over, and every wave of the block is here.
template <int N>
__device__ __forceinline__ void wait_loads_and_meet() {
    static_assert(N >= 0 && N < 64, "vmcnt has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <class F, int... I>
__device__ __forceinline__ void for_each_of(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }

}  // namespace dsllm
