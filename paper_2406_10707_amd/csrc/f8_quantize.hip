// Conversion to matrices in 8 bits with a scale for each block of 128, their transposes, and back (include/ckpt_train.h).
#include <algorithm>
#include <type_traits>

#include "f8_rows.hpp"

using namespace dsllm;

namespace {

constexpr int kHeld = 0;      // a source that is itself held in 8 bits

// ------------------------------------------------------------------ rows alone

template <int SRC>
__global__ __launch_bounds__(256) void f8_rows_kernel(F8Source src, F8Held to, uint32_t across) {
    const uint32_t down = blockIdx.x / across;
    f8_round_rows<SRC>(src, to, 16 * int64_t(down), 512 * int64_t(blockIdx.x - down * across));
}

// ------------------------------------------------------------------ tiles: columns, both forms, blocks of 128 x 128

template <class F>
__device__ __forceinline__ void for_each_of_eight(F f) {
    f(std::integral_constant<int, 0>()); f(std::integral_constant<int, 1>()); f(std::integral_constant<int, 2>()); f(std::integral_constant<int, 3>());
    f(std::integral_constant<int, 4>()); f(std::integral_constant<int, 5>()); f(std::integral_constant<int, 6>()); f(std::integral_constant<int, 7>());
}

// Word i of four, each with four bytes, becomes the four words' bytes i.
__device__ __forceinline__ u32x4 transposed(u32x4 v) {
    const uint32_t ab_lo = __builtin_amdgcn_perm(v.y, v.x, 0x05010400), ab_hi = __builtin_amdgcn_perm(v.y, v.x, 0x07030602);      // x0 y0 x1 y1, x2 y2 x3 y3
    const uint32_t cd_lo = __builtin_amdgcn_perm(v.w, v.z, 0x05010400), cd_hi = __builtin_amdgcn_perm(v.w, v.z, 0x07030602);
    return u32x4{__builtin_amdgcn_perm(cd_lo, ab_lo, 0x05040100), __builtin_amdgcn_perm(cd_lo, ab_lo, 0x07060302), __builtin_amdgcn_perm(cd_hi, ab_hi, 0x05040100),
                 __builtin_amdgcn_perm(cd_hi, ab_hi, 0x07060302)};
}

// A tile of 128 x 128 elements, which stays in registers: a thread has eight rows of eight columns (of an f32 source twice four, half a tile apart: its loads are sixteen bytes of neighbouring lanes), sixteen lanes across, four groups of
// eight rows a wave. The rows' largest values are found among sixteen lanes, the columns' among a wave's four groups and, through LDS, the four waves; a scale is found by one lane (its two divisions are some 25 instructions) and
// handed to the others. The columns' codes go through LDS as bytes (128 columns of 128, and 16 more so that neighbouring columns begin in different banks), so that a store is whole lines. SQUARE: one scale for the tile, so that both forms
// have the same codes. Bound by memory: 8192 x 4096 of bf16 to both forms 28.5 us (a plain copy of as many bytes 26), 11008 x 4096 of f32 in blocks of 128 x 128 to both 51 (5.3 TB/s), the columns' form of 8192 x 4096 in 8 bits 12.9 (5.4 TB/s;
// 15.1 with the pieces of columns in LDS as they come). The 16-bit sources kept as they were stored and converted twice, for seven blocks a unit instead of five, and other orders of the tiles were no faster.
template <int SRC, bool BY_ROW, bool BY_COL, bool SQUARE>
__global__ __launch_bounds__(256) void f8_tile_kernel(F8Source src, F8Held by_row, F8Held by_col, uint32_t across_tiles) {
    constexpr bool HELD = SRC == kHeld, KEPT = HELD && SQUARE, APART = SRC == CKPT_F32;      // KEPT: codes and scales move as they are
    constexpr int PITCH = 128 + 16;
    __shared__ __attribute__((aligned(16))) uint8_t turned[BY_COL ? 128 * PITCH : 16];
    __shared__ __attribute__((aligned(16))) uint32_t most_of_wave[4][128];      // then what columns are multiplied with
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, across = threadIdx.x & 15, down = threadIdx.x >> 4;
    const uint32_t tile_down = blockIdx.x / across_tiles, tile_across = blockIdx.x - tile_down * across_tiles;
    const int64_t row0 = 128 * int64_t(tile_down) + 8 * down, col0 = 128 * int64_t(tile_across);
    const uint32_t in_lo = APART ? 4 * across : 8 * across, in_hi = APART ? 64 + 4 * across : 8 * across + 4;      // the thread's columns: four and four
    const int64_t col_lo = col0 + in_lo, col_hi = col0 + in_hi;
    const bool whole = 128 * int64_t(tile_down) + 128 <= src.rows && col0 + 128 <= src.cols;      // loads without conditions: all are under way before the first is waited for
    auto left_of = [&](int64_t col) { return col < src.cols ? uint32_t(min(src.cols - col, int64_t(4))) : 0; };
    const uint32_t count_lo = left_of(col_lo), count_hi = left_of(col_hi), rows_left = uint32_t(max(int64_t(0), min(src.rows - row0, int64_t(8))));
    f32x4 lo[8], hi[8];
    u32x2 codes[8];
    if constexpr (HELD) {
        const uint8_t *at = src.at + row0 * src.ld + col_lo;      // a row's codes reach to a multiple of 128
        const float DSLLM_GLOBAL *scales = (const float DSLLM_GLOBAL *)src.scales + tile_across * src.scale_pitch + row0;
        float scale[8];
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; i++) codes[i] = *(const u32x2 DSLLM_GLOBAL *)(at + i * src.ld);
            if constexpr (!KEPT) {
                typedef f32x4 four_aligned4 __attribute__((aligned(4)));
                const f32x4 upper = *(const four_aligned4 DSLLM_GLOBAL *)scales, lower = *(const four_aligned4 DSLLM_GLOBAL *)(scales + 4);
#pragma unroll
                for (int i = 0; i < 4; i++) { scale[i] = upper[i]; scale[4 + i] = lower[i]; }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                codes[i] = row0 + i < src.rows ? *(const u32x2 DSLLM_GLOBAL *)(at + i * src.ld) : u32x2{0, 0};
                if constexpr (!KEPT) scale[i] = row0 + i < src.rows ? scales[i] : 0;
            }
        }
        if constexpr (!KEPT)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                lo[i] = f8_values(codes[i].x, src.e5m2) * scale[i];
                hi[i] = f8_values(codes[i].y, src.e5m2) * scale[i];
            }
    } else if constexpr (APART) {
        const float *at = reinterpret_cast<const float *>(src.at) + row0 * src.ld + col_lo;
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                lo[i] = load4<SRC>(at + i * src.ld);
                hi[i] = load4<SRC>(at + i * src.ld + 64);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                lo[i] = load_upto4<SRC>(at + i * src.ld, row0 + i < src.rows ? count_lo : 0);
                hi[i] = load_upto4<SRC>(at + i * src.ld + 64, row0 + i < src.rows ? count_hi : 0);
            }
        }
    } else {
        constexpr uint32_t kBytes = sizeof(typename Element<SRC>::one);
        const uint8_t *at = src.at + (row0 * src.ld + col_lo) * kBytes;
        Eight<SRC> x[8];
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i].load(at + i * src.ld * kBytes);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i].load_upto(at + i * src.ld * kBytes, row0 + i < src.rows ? count_lo + count_hi : 0);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            lo[i] = __builtin_convertvector(x[i].lo, f32x4);
            hi[i] = __builtin_convertvector(x[i].hi, f32x4);
        }
    }
    auto bytes_kept = [](uint32_t n) { return n >= 4 ? ~0u : (1u << (8 * n)) - 1; };
    const uint32_t kept_lo = bytes_kept(count_lo), kept_hi = bytes_kept(count_hi);      // codes behind the last element are zero, whatever the block's scale
    auto put_row = [&](int i, u32x2 c) {
        if (!whole && row0 + i >= src.rows) return;
        uint8_t *at = by_row.codes + (row0 + i) * by_row.code_pitch + col_lo;
        if constexpr (APART) {
            __builtin_nontemporal_store(c.x, (uint32_t DSLLM_GLOBAL *)at);
            __builtin_nontemporal_store(c.y, (uint32_t DSLLM_GLOBAL *)(at + 64));
        } else __builtin_nontemporal_store(c, (u32x2 DSLLM_GLOBAL *)at);
    };
    if constexpr (SQUARE && !KEPT) {
        float largest = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) largest = larger(larger(largest, lo[i]), hi[i]);
        uint32_t amax = most_of_quarters(most_of_16(bits_of(largest)));
        if (lane == 0) most_of_wave[wave][0] = amax;
        __syncthreads();
        amax = max(max(most_of_wave[0][0], most_of_wave[1][0]), max(most_of_wave[2][0], most_of_wave[3][0]));
        const bool e5m2 = BY_ROW ? by_row.e5m2 : by_col.e5m2;
        const float inverse = f8_inverse(amax, f8_most(e5m2));
#pragma unroll
        for (int i = 0; i < 8; i++) {
            codes[i] = u32x2{f8_codes(lo[i] * inverse, e5m2) & kept_lo, f8_codes(hi[i] * inverse, e5m2) & kept_hi};
            if (!whole && row0 + i >= src.rows) codes[i] = u32x2{0, 0};
        }
        if (threadIdx.x == 0) {
            const float scale = f8_scale(amax, f8_most(e5m2));
            if constexpr (BY_ROW) ((float DSLLM_GLOBAL *)by_row.scales)[tile_across * by_row.scale_pitch + tile_down] = scale;
            if constexpr (BY_COL) ((float DSLLM_GLOBAL *)by_col.scales)[tile_down * by_col.scale_pitch + tile_across] = scale;
        }
        if constexpr (BY_ROW)
#pragma unroll
            for (int i = 0; i < 8; i++) put_row(i, codes[i]);
    }
    if constexpr (KEPT)
        if (threadIdx.x == 0) ((float DSLLM_GLOBAL *)by_col.scales)[tile_down * by_col.scale_pitch + tile_across] = ((const float DSLLM_GLOBAL *)src.scales)[tile_across * src.scale_pitch + tile_down];
    if constexpr (BY_ROW && !SQUARE) {
        uint32_t amax = 0;      // of row `across` of the eight
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t found = most_of_16(bits_of(larger(larger(0, lo[i]), hi[i])));
            amax = across == uint32_t(i) ? found : amax;
        }
        const float mine = f8_inverse(amax, f8_most(by_row.e5m2));
        if (across < 8 && row0 + across < src.rows) ((float DSLLM_GLOBAL *)by_row.scales)[tile_across * by_row.scale_pitch + row0 + across] = f8_scale(amax, f8_most(by_row.e5m2));
        for_each_of_eight([&](auto i) {
            const float inverse = of_lane_of_16<i>(mine);
            put_row(i, u32x2{f8_codes(lo[i] * inverse, by_row.e5m2) & kept_lo, f8_codes(hi[i] * inverse, by_row.e5m2) & kept_hi});
        });
    }
    if constexpr (BY_COL) {
        // a column's pieces of 16 bytes are rotated by one for each 16 columns: a wave's lanes, whose columns are 8 (4) apart, write to all banks
        auto place = [&](uint32_t c) { return reinterpret_cast<u32x2 *>(turned + c * PITCH + (16 * (c >> 4) + 8 * down) % 128); };
        if constexpr (!SQUARE) {
            uint32_t most[8];      // bits of magnitudes, which order like them
#pragma unroll
            for (int j = 0; j < 8; j++) {
                auto at = [&](int i) { return j < 4 ? lo[i][j & 3] : hi[i][j & 3]; };
                most[j] = most_of_quarters(bits_of(larger(larger(0, f32x4{at(0), at(1), at(2), at(3)}), f32x4{at(4), at(5), at(6), at(7)})));
            }
            if (lane < 16) {
                *reinterpret_cast<u32x4 *>(&most_of_wave[wave][in_lo]) = u32x4{most[0], most[1], most[2], most[3]};
                *reinterpret_cast<u32x4 *>(&most_of_wave[wave][in_hi]) = u32x4{most[4], most[5], most[6], most[7]};
            }
            __syncthreads();
            if (threadIdx.x < 128) {
                const uint32_t c = threadIdx.x, amax = max(max(most_of_wave[0][c], most_of_wave[1][c]), max(most_of_wave[2][c], most_of_wave[3][c]));
                most_of_wave[0][c] = __float_as_uint(f8_inverse(amax, f8_most(by_col.e5m2)));
                if (col0 + c < src.cols) ((float DSLLM_GLOBAL *)by_col.scales)[tile_down * by_col.scale_pitch + col0 + c] = f8_scale(amax, f8_most(by_col.e5m2));
            }
            __syncthreads();
            const f32x4 by_lo = *reinterpret_cast<const f32x4 *>(&most_of_wave[0][in_lo]), by_hi = *reinterpret_cast<const f32x4 *>(&most_of_wave[0][in_hi]);
            const uint32_t upper = bytes_kept(rows_left), lower = bytes_kept(rows_left > 4 ? rows_left - 4 : 0);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                auto at = [&](int i) { return j < 4 ? lo[i][j & 3] : hi[i][j & 3]; };
                const float by = j < 4 ? by_lo[j & 3] : by_hi[j & 3];
                *place((j < 4 ? in_lo : in_hi) + (j & 3)) =
                    u32x2{f8_codes(f32x4{at(0), at(1), at(2), at(3)} * by, by_col.e5m2) & upper, f8_codes(f32x4{at(4), at(5), at(6), at(7)} * by, by_col.e5m2) & lower};
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; h++) {      // the four columns of one half of the thread's
                const u32x4 upper = transposed(u32x4{codes[0][h], codes[1][h], codes[2][h], codes[3][h]}), lower = transposed(u32x4{codes[4][h], codes[5][h], codes[6][h], codes[7][h]});
#pragma unroll
                for (int j = 0; j < 4; j++) *place((h ? in_hi : in_lo) + j) = u32x2{upper[j], lower[j]};
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t c = 32 * i + (threadIdx.x >> 3), piece = 16 * (threadIdx.x & 7);
            if (whole || col0 + c < src.cols)
                __builtin_nontemporal_store(*reinterpret_cast<const u32x4 *>(turned + c * PITCH + (16 * (c >> 4) + piece) % 128), (u32x4 DSLLM_GLOBAL *)(by_col.codes + (col0 + c) * by_col.code_pitch + 128 * uint64_t(tile_down) + piece));
        }
    }
}

// ------------------------------------------------------------------ values

// Eight elements a lane, 512 of a row a wave. Bound by memory. Results in 32 bits are stored four at a time, a wave's store in whole lines: 11008 x 4096 with eight side by side took 60 to 65 us, now 33 (6.9 TB/s; bf16 22, 6.1 TB/s).
template <int DST>
__global__ __launch_bounds__(256) void f8_values_kernel(F8Held from, uint8_t *dst, uint64_t ld, uint32_t pieces) {
    constexpr uint32_t N = DST == CKPT_F32 ? 4 : 8, BYTES = sizeof(typename Element<DST>::one);
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t item = uint64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = item / pieces, first = (item - row * pieces) * 512 + N * lane;
    if (row >= from.rows) return;
    uint32_t codes[8 / N][N / 4];
    float scale[8 / N];
#pragma unroll
    for (uint32_t i = 0; i < 8 / N; i++) {
        const int64_t col = first + 64 * N * i;
        if (col >= from.cols) break;
        scale[i] = ((const float DSLLM_GLOBAL *)from.scales)[(col / 128) * from.scale_pitch + (row >> from.shift)];
        const uint32_t DSLLM_GLOBAL *at = (const uint32_t DSLLM_GLOBAL *)(from.codes + row * from.code_pitch + col);
        codes[i][0] = at[0];
        if constexpr (N == 8) codes[i][1] = at[1];
    }
#pragma unroll
    for (uint32_t i = 0; i < 8 / N; i++) {
        const int64_t col = first + 64 * N * i;
        if (col >= from.cols) return;
        uint8_t *at = dst + (row * ld + col) * BYTES;
        const f32x4 lo = f8_values(codes[i][0], from.e5m2) * scale[i];
        if constexpr (N == 4) store_upto4<DST>(at, lo, uint32_t(min(from.cols - col, int64_t(4))));
        else {
            const f32x4 hi = f8_values(codes[i][1], from.e5m2) * scale[i];
            if (col + 8 <= from.cols) store8<DST>(at, lo, hi);
            else {
                store_upto4<DST>(at, lo, uint32_t(from.cols - col));
                if (col + 4 < from.cols) store_upto4<DST>(at + 4 * BYTES, hi, uint32_t(from.cols - col - 4));
            }
        }
    }
}

// ------------------------------------------------------------------ host

constexpr const char *kTooLarge = "the matrix takes 2^24 blocks of threads or more";
bool fits_grid(uint64_t down, uint64_t across) { return down < 1u << 24 && across < 1u << 24 && down * across < 1u << 24; }

template <int SRC>
int launch_quantize(const F8Source &src, const F8Held &by_row, const F8Held &by_col, bool square, hipStream_t stream) {
    if (!by_col.codes && !square) {
        const uint64_t down = (uint64_t(src.rows) + 15) / 16, across = (uint64_t(src.cols) + 511) / 512;
        if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooLarge);
        hipLaunchKernelGGL(f8_rows_kernel<SRC>, dim3(unsigned(down * across)), dim3(256), 0, stream, src, by_row, uint32_t(across));
        return launched();
    }
    const uint64_t down = (uint64_t(src.rows) + 127) / 128, across = (uint64_t(src.cols) + 127) / 128;
    if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooLarge);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(down * across)), dim3(256), 0, stream, src, by_row, by_col, uint32_t(across)); };
    if (square) !by_col.codes ? go(f8_tile_kernel<SRC, true, false, true>) : by_row.codes ? go(f8_tile_kernel<SRC, true, true, true>) : go(f8_tile_kernel<SRC, false, true, true>);
    else by_row.codes ? go(f8_tile_kernel<SRC, true, true, false>) : go(f8_tile_kernel<SRC, false, true, false>);
    return launched();
}

int quantize(const void *src, int32_t dtype, int64_t ld, const ckpt_f8_matrix *by_row, const ckpt_f8_matrix *by_col, hipStream_t stream) {
    if (!by_row && !by_col) return refuse(CKPT_EINVAL, "neither by_row nor by_col");
    const uint32_t bytes = element_bytes(dtype);
    if (!bytes) return refuse(CKPT_EINVAL, "src_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    DeviceRanges ranges;
    for (const ckpt_f8_matrix *m : {by_row, by_col})
        if (m)
            if (const char *why = wrong_f8_matrix(m, ranges)) return refuse(CKPT_EINVAL, std::string(m == by_row ? "by_row: " : "by_col: ") + why);
    if (by_row && by_col) {
        if (by_row->rows != by_col->cols || by_row->cols != by_col->rows) return refuse(CKPT_EINVAL, "by_col is not of the transpose's size");
        if (by_row->block_rows != by_col->block_rows) return refuse(CKPT_EINVAL, "by_row and by_col differ in block_rows");
        if (by_row->block_rows == 128 && by_row->format != by_col->format) return refuse(CKPT_EINVAL, "by_row and by_col differ in their format: with block_rows 128 they hold the same values");
    }
    const int64_t rows = by_row ? by_row->rows : by_col->cols, cols = by_row ? by_row->cols : by_col->rows;
    if (rows == 0 || cols == 0) return CKPT_OK;
    if (ld < cols || ld > (1ll << 48) / rows) return refuse(CKPT_EINVAL, "ld is smaller than a row, or the matrix too large");
    if (uint64_t(src) % bytes) return refuse(CKPT_EINVAL, "src is not aligned to its element");
    if (const char *why = ranges.wrong(src, (uint64_t(rows - 1) * ld + cols) * bytes)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    for (const ckpt_f8_matrix *m : {by_row, by_col})
        if (m && (overlaps_itself(*m) || overlap(*m, plain_rows(src, rows, cols, ld, bytes)))) return refuse(CKPT_EINVAL, std::string(m == by_row ? "by_row: " : "by_col: ") + "overlaps src or itself");
    if (by_row && by_col && overlap(*by_row, *by_col)) return refuse(CKPT_EINVAL, "by_row and by_col overlap");
    const F8Source from{static_cast<const uint8_t *>(src), uint64_t(ld), rows, cols, nullptr, 0, 0};
    const bool square = (by_row ? by_row : by_col)->block_rows == 128;
    switch (dtype) {
        case CKPT_F32: return launch_quantize<CKPT_F32>(from, F8Held(by_row), F8Held(by_col), square, stream);
        case CKPT_BF16: return launch_quantize<CKPT_BF16>(from, F8Held(by_row), F8Held(by_col), square, stream);
        default: return launch_quantize<CKPT_F16>(from, F8Held(by_row), F8Held(by_col), square, stream);
    }
}

int columns(const ckpt_f8_matrix *src, const ckpt_f8_matrix *by_col, hipStream_t stream) {
    if (!src || !by_col) return refuse(CKPT_EINVAL, "null argument");
    DeviceRanges ranges;
    if (const char *why = wrong_f8_matrix(src, ranges)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    if (const char *why = wrong_f8_matrix(by_col, ranges)) return refuse(CKPT_EINVAL, std::string("by_col: ") + why);
    if (src->rows != by_col->cols || src->cols != by_col->rows) return refuse(CKPT_EINVAL, "by_col is not of the transpose's size");
    if (src->block_rows != by_col->block_rows) return refuse(CKPT_EINVAL, "src and by_col differ in block_rows");
    if (src->block_rows == 128 && src->format != by_col->format) return refuse(CKPT_EINVAL, "src and by_col differ in their format: with block_rows 128 the values stay as they are");
    if (src->rows == 0 || src->cols == 0) return CKPT_OK;
    if (overlaps_itself(*by_col) || overlap(*by_col, *src)) return refuse(CKPT_EINVAL, "by_col: overlaps src or itself");
    const F8Source from{static_cast<const uint8_t *>(src->codes), src->code_pitch, src->rows, src->cols, src->scales, src->scale_pitch, src->format == CKPT_F8_E5M2};
    const uint64_t down = (uint64_t(src->rows) + 127) / 128, across = (uint64_t(src->cols) + 127) / 128;
    if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooLarge);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(down * across)), dim3(256), 0, stream, from, F8Held(), F8Held(by_col), uint32_t(across)); };
    src->block_rows == 128 ? go(f8_tile_kernel<kHeld, false, true, true>) : go(f8_tile_kernel<kHeld, false, true, false>);
    return launched();
}

int dequantize(const ckpt_f8_matrix *m, void *dst, int32_t dtype, int64_t ld, hipStream_t stream) {
    if (!m) return refuse(CKPT_EINVAL, "null argument");
    const uint32_t bytes = element_bytes(dtype);
    if (!bytes) return refuse(CKPT_EINVAL, "dst_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    DeviceRanges ranges;
    if (const char *why = wrong_f8_matrix(m, ranges)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    if (m->rows == 0 || m->cols == 0) return CKPT_OK;
    if (ld < m->cols || ld > (1ll << 48) / m->rows) return refuse(CKPT_EINVAL, "ld is smaller than a row, or the matrix too large");
    if (uint64_t(dst) % bytes) return refuse(CKPT_EINVAL, "dst is not aligned to its element");
    if (const char *why = ranges.wrong(dst, (uint64_t(m->rows - 1) * ld + m->cols) * bytes)) return refuse(CKPT_EINVAL, std::string("dst: ") + why);
    if (overlap(*m, plain_rows(dst, m->rows, m->cols, ld, bytes))) return refuse(CKPT_EINVAL, "dst: overlaps src");
    const uint64_t pieces = (uint64_t(m->cols) + 511) / 512;
    if (uint64_t(m->rows) > 1ull << 26 || !fits_grid((m->rows + 3) / 4, pieces)) return refuse(CKPT_EINVAL, kTooLarge);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned((m->rows * pieces + 3) / 4)), dim3(256), 0, stream, F8Held(m), static_cast<uint8_t *>(dst), uint64_t(ld), uint32_t(pieces)); };
    switch (dtype) {
        case CKPT_F32: go(f8_values_kernel<CKPT_F32>); break;
        case CKPT_BF16: go(f8_values_kernel<CKPT_BF16>); break;
        default: go(f8_values_kernel<CKPT_F16>);
    }
    return launched();
}

}  // namespace

const char *dsllm::wrong_f8_matrix(const ckpt_f8_matrix *m, DeviceRanges &ranges) {
    if (m->format != CKPT_F8_E4M3 && m->format != CKPT_F8_E5M2) return "format must be CKPT_F8_E4M3 or CKPT_F8_E5M2";
    if (m->block_rows != 1 && m->block_rows != 128) return "block_rows must be 1 or 128";
    if (m->rows < 0 || m->cols < 0 || m->rows > 1ll << 40 || m->cols > 1ll << 40) return "rows or cols out of range";
    if (m->rows == 0 || m->cols == 0) return nullptr;
    const uint64_t rows = uint64_t(m->rows), padded = f8_padded(m->cols), scale_rows = (rows + m->block_rows - 1) / m->block_rows;
    if (m->code_pitch % 16 || uint64_t(m->codes) % 16 || uint64_t(m->scales) % 4) return "a pitch and an address of 16 bytes are wanted for the codes, one of 4 for the scales";
    if (m->code_pitch < padded || m->scale_pitch < scale_rows) return "a pitch is smaller than a row, or than a block of columns";
    if (m->code_pitch > (1ull << 48) / rows || m->scale_pitch > (1ull << 48) / padded) return "the matrix is too large";
    if (const char *why = ranges.wrong(m->codes, (rows - 1) * m->code_pitch + padded)) return why;
    return ranges.wrong(m->scales, 4 * ((padded / 128 - 1) * m->scale_pitch + scale_rows));
}

bool dsllm::share_bytes(const Rows &a, const Rows &b) {
    if (a.at >= b.end() || b.at >= a.end()) return false;
    if (a.pitch == b.pitch) {
        const Rows &first = a.at <= b.at ? a : b, &second = a.at <= b.at ? b : a;
        const uint64_t apart = (second.at - first.at) % a.pitch;
        return apart < first.width || apart + second.width > a.pitch;
    }
    const Rows &few = a.rows <= b.rows ? a : b, &many = a.rows <= b.rows ? b : a;
    if (few.rows > 1 << 16) return true;
    for (uint64_t r = 0; r < few.rows; r++) {
        const uint64_t lo = few.at + r * few.pitch, hi = lo + few.width, k = lo < many.at + many.width ? 0 : (lo - many.at - many.width) / many.pitch + 1;      // the first row of the other that ends behind lo
        if (k < many.rows && many.at + k * many.pitch < hi) return true;
    }
    return false;
}
static Rows codes_of(const ckpt_f8_matrix &m) { return Rows{uint64_t(m.codes), f8_padded(m.cols), m.code_pitch, uint64_t(m.rows)}; }
static Rows scales_of(const ckpt_f8_matrix &m) { return Rows{uint64_t(m.scales), 4 * ((uint64_t(m.rows) + m.block_rows - 1) / m.block_rows), 4 * m.scale_pitch, f8_padded(m.cols) / 128}; }
bool dsllm::overlap(const ckpt_f8_matrix &m, const Rows &rows) { return m.rows && m.cols && (share_bytes(codes_of(m), rows) || share_bytes(scales_of(m), rows)); }
bool dsllm::overlap(const ckpt_f8_matrix &a, const ckpt_f8_matrix &b) { return a.rows && a.cols && (overlap(b, codes_of(a)) || overlap(b, scales_of(a))); }
bool dsllm::overlaps_itself(const ckpt_f8_matrix &m) { return m.rows && m.cols && share_bytes(codes_of(m), scales_of(m)); }

extern "C" {

int ckpt_f8_layout(int32_t format, int32_t block_rows, int64_t rows, int64_t cols, ckpt_f8_matrix *out) {
    return at_c_entry([&] {
        if (!out) return refuse(CKPT_EINVAL, "null argument");
        *out = ckpt_f8_matrix{};
        if (format != CKPT_F8_E4M3 && format != CKPT_F8_E5M2) return refuse(CKPT_EINVAL, "format must be CKPT_F8_E4M3 or CKPT_F8_E5M2");
        if (block_rows != 1 && block_rows != 128) return refuse(CKPT_EINVAL, "block_rows must be 1 or 128");
        if (rows < 0 || cols < 0 || rows > 1ll << 40 || cols > 1ll << 40) return refuse(CKPT_EINVAL, "rows or cols out of range");
        out->format = format;
        out->block_rows = block_rows;
        out->rows = rows;
        out->cols = cols;
        out->code_pitch = f8_padded(cols);
        out->scale_pitch = (uint64_t(rows) + block_rows - 1) / block_rows;
        return int(CKPT_OK);
    });
}

int ckpt_f8_quantize(const void *src, int32_t src_dtype, int64_t ld, const ckpt_f8_matrix *by_row, const ckpt_f8_matrix *by_col, void *stream) {
    return at_c_entry([&] { return quantize(src, src_dtype, ld, by_row, by_col, static_cast<hipStream_t>(stream)); });
}

int ckpt_f8_columns(const ckpt_f8_matrix *src, const ckpt_f8_matrix *by_col, void *stream) {
    return at_c_entry([&] { return columns(src, by_col, static_cast<hipStream_t>(stream)); });
}

int ckpt_f8_dequantize(const ckpt_f8_matrix *src, void *dst, int32_t dst_dtype, int64_t ld, void *stream) {
    return at_c_entry([&] { return dequantize(src, dst, dst_dtype, ld, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
