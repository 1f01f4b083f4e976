// Conversion to block-scaled formats and back (include/ckpt_train.h).
#include <algorithm>
#include <type_traits>

#include "train_util.hpp"

using namespace dsllm;

namespace {

struct RowArgs {
    const uint8_t *src;
    uint64_t ld;                // elements
    uint64_t rows, cols;
    uint8_t *codes, *scales;
    uint64_t code_pitch, scale_pitch;
    uint64_t blocks;            // of a row, with those behind its end that are to be zero
    uint64_t key;
    uint64_t pieces;            // of a row, a wave's work each
};

// E2M1 codes of eight values of a row (eight times four bits), a block of which lies in four neighbouring lanes; `byte` is its scale.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t fp4_codes_of_eight(f32x4 lo, f32x4 hi, uint64_t first_group_of_random, uint32_t *byte) {
    *byte = scale_byte<CKPT_MXFP4>(most_of_4(max(magnitude_bits(lo), magnitude_bits(hi))));
    const float inverse = inverse_scale(*byte);
    lo *= inverse;
    hi *= inverse;
    if constexpr (STOCHASTIC) return fp4_stochastic(lo, mix64(first_group_of_random)) | fp4_stochastic(hi, mix64(first_group_of_random + 1)) << 16;
    else return fp4_nearest(lo) | fp4_nearest(hi) << 16;
}

// A wave takes 1024 elements of a row in groups of 512, eight elements a lane; four lanes a block of 32. Bound by memory: 60 M f32 to 8 bits 52 us = 5.8 TB/s, 55 stochastically (three 64-bit products for
// every four elements; with four elements a lane 48 and 59: its accesses are whole lines, but there is more to do for each), 45 M bf16 to 4 bits 22 us = 5.2 TB/s (four a lane 24, one group of them 27),
// stochastically 35, from f32 37 and 43. Rows of fewer than 1024 elements leave lanes without work.
constexpr uint32_t kGroups = 2, kRowPiece = 512 * kGroups;
template <int SRC, int FORMAT, bool STOCHASTIC, bool NONZERO>
__global__ __launch_bounds__(256) void rows_kernel(RowArgs a) {
    constexpr uint32_t kBytes = sizeof(typename Element<SRC>::one);
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t item = uint64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t row = item / a.pieces, first = (item - row * a.pieces) * kRowPiece;
    if (row >= a.rows) return;
    auto work = [&](auto whole) {
        Eight<SRC> x[kGroups];
        uint32_t count[kGroups];
#pragma unroll
        for (int k = 0; k < int(kGroups); k++) {
            const uint64_t col = first + 512 * k + 8 * lane;
            count[k] = whole ? 8 : col < a.cols ? uint32_t(min(a.cols - col, uint64_t(8))) : 0;
            if constexpr (whole) x[k].load(a.src + (row * a.ld + col) * kBytes);
            else x[k].load_upto(a.src + (row * a.ld + col) * kBytes, count[k]);
        }
#pragma unroll
        for (int k = 0; k < int(kGroups); k++) {
            const uint64_t col = first + 512 * k + 8 * lane, random = a.key + row * ((a.cols + 3) / 4) + col / 4;
            const f32x4 lo = __builtin_convertvector(x[k].lo, f32x4), hi = __builtin_convertvector(x[k].hi, f32x4);
            uint32_t byte;
            if constexpr (FORMAT == CKPT_MXFP4) {
                uint32_t codes = fp4_codes_of_eight<STOCHASTIC>(lo, hi, random, &byte);
                if (count[k] < 8) codes &= (1u << (4 * count[k])) - 1;
                if (col / 2 < a.code_pitch) *(uint32_t DSLLM_GLOBAL *)(a.codes + row * a.code_pitch + col / 2) = codes;
            } else {
                byte = scale_byte<CKPT_MXFP8>(most_of_4(max(magnitude_bits(lo), magnitude_bits(hi))));
                const f32x4 y0 = lo * inverse_scale(byte), y1 = hi * inverse_scale(byte);
                const uint32_t c0 = STOCHASTIC ? fp8_stochastic<NONZERO>(y0, lo, mix64(random)) : fp8_nearest<NONZERO>(y0, lo);
                const uint32_t c1 = STOCHASTIC ? fp8_stochastic<NONZERO>(y1, hi, mix64(random + 1)) : fp8_nearest<NONZERO>(y1, hi);
                uint8_t *at = a.codes + row * a.code_pitch + col;
                if (whole || count[k] == 8) {
                    typedef u32x2 two_bytealigned __attribute__((aligned(1)));
                    __builtin_nontemporal_store(u32x2{c0, c1}, (two_bytealigned DSLLM_GLOBAL *)at);
                } else if (col < a.code_pitch) {      // what the row has behind its last element is zero
                    const uint32_t room = uint32_t(min(a.code_pitch - col, uint64_t(8)));
                    const uint64_t both = (uint64_t(c1) << 32 | c0) & ((1ull << (8 * count[k])) - 1);
                    store_bytes(at, uint32_t(both), min(room, 4u));
                    if (room > 4) store_bytes(at + 4, uint32_t(both >> 32), room - 4);
                }
            }
            if ((lane & 3) == 0 && col / 32 < a.scale_pitch) ((uint8_t DSLLM_GLOBAL *)a.scales)[row * a.scale_pitch + col / 32] = uint8_t(byte);
        }
    };
    // a piece that ends inside the row has loads without conditions: all are under way before the first is waited for
    if (first + kRowPiece <= a.cols) work(std::true_type{});
    else work(std::false_type{});
}

// A tile of 128 x 128 elements, to the columns' form and, with BY_ROW, to the rows' as well, 64 rows at a time: read once, 16 lanes a row, rounded by rows as it comes, put into LDS, and read
// from there by columns while the other 64 rows are under way. In LDS the rows of the second 32 begin 32 words further round the banks: the 32 columns x 2 blocks of 32 rows that a wave reads at
// once lie in 64 different ones; the counter all the same has conflicts in half of the cycles that LDS works, a tenth of the kernel's. 45 M f32 to both forms 47 to 52 us = 4.8 to 4.4 TB/s (all 128 rows at a
// time, two blocks a unit instead of four: 52 beside 47; by two kernels that each read src 100), bf16 34 us (four elements a lane: 37), stochastically 68 to 70 and 65; by columns alone 42 and 25,
// stochastically 47 and 39. Loads that stand under a condition, with the conversion to f32 beside them, are waited for one by one: bf16 took 83 us with them. What it writes beyond the two forms, a third more, is scales: four
// bytes of 32 at a time, of two XCDs' L2 (runs of tiles for each XCD write less and take 1 to 8 % longer).
struct TileArgs {
    RowArgs by_row, by_col;      // by_col: rows, cols are src's; codes, scales its transpose's
    uint32_t tiles_across;
};
template <int SRC, bool STOCHASTIC, bool BY_ROW>
__global__ __launch_bounds__(256, 4) void tile_kernel(TileArgs p) {
    constexpr uint32_t kBytes = sizeof(typename Element<SRC>::one);
    __shared__ float tile[128 * 64 + 32];
    const RowArgs &a = p.by_row, &c = p.by_col;
    const uint64_t tile_row = blockIdx.x / p.tiles_across, row0 = 128 * tile_row, col0 = 128 * (blockIdx.x - tile_row * uint64_t(p.tiles_across));
    const uint32_t across = threadIdx.x & 15, down = threadIdx.x >> 4;
    const uint64_t col = col0 + 8 * across;
    const uint32_t count = col < c.cols ? uint32_t(min(c.cols - col, uint64_t(8))) : 0;
    const bool whole = row0 + 128 <= c.rows && col0 + 128 <= c.cols;      // loads without conditions: all are under way before the first is waited for
    const uint8_t *src = c.src + ((row0 + down) * c.ld + col) * kBytes;
    Eight<SRC> x[4];
    auto load = [&](int half) {
        if (whole) {
#pragma unroll
            for (int i = 0; i < 4; i++) x[i].load(src + (64 * half + 16 * i) * c.ld * kBytes);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) x[i].load_upto(src + (64 * half + 16 * i) * c.ld * kBytes, row0 + 64 * half + 16 * i + down < c.rows ? count : 0);
        }
    };
    load(0);
#pragma unroll
    for (int half = 0; half < 2; half++) {
        if (half) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t r = 16 * i + down;
            const uint64_t row = row0 + 64 * half + r;
            const f32x4 lo = __builtin_convertvector(x[i].lo, f32x4), hi = __builtin_convertvector(x[i].hi, f32x4);
            float *at = tile + 128 * r + 32 * (r >> 5) + 8 * across;
            *reinterpret_cast<f32x4 *>(at) = lo;
            *reinterpret_cast<f32x4 *>(at + 4) = hi;
            if constexpr (BY_ROW) {
                uint32_t byte, codes = fp4_codes_of_eight<STOCHASTIC>(lo, hi, a.key + row * ((a.cols + 3) / 4) + col / 4, &byte);
                if (count < 8) codes &= (1u << (4 * count)) - 1;
                if (row < a.rows) {
                    if (col / 2 < a.code_pitch) *(uint32_t DSLLM_GLOBAL *)(a.codes + row * a.code_pitch + col / 2) = codes;
                    if ((across & 3) == 0 && col / 32 < a.scale_pitch) ((uint8_t DSLLM_GLOBAL *)a.scales)[row * a.scale_pitch + col / 32] = uint8_t(byte);
                }
            }
        }
        if (half == 0) load(1);
        __syncthreads();
        const uint32_t of_rows = threadIdx.x & 1, of_cols = threadIdx.x >> 1;
        const uint64_t first = row0 + 64 * half + 32 * of_rows, block = first / 32, out = col0 + of_cols;
        f32x4 y[8];
        uint32_t most = 0;
#pragma unroll
        for (int g = 0; g < 8; g++) {
#pragma unroll
            for (int j = 0; j < 4; j++) y[g][j] = tile[128 * (32 * of_rows + 4 * g + j) + 32 * of_rows + of_cols];
            most = max(most, magnitude_bits(y[g]));
        }
        if (out >= c.cols) continue;
        const uint32_t byte = scale_byte<CKPT_MXFP4>(most);
        u32x4 codes{0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < 8; g++) {
            const f32x4 v = y[g] * inverse_scale(byte);
            uint32_t four = STOCHASTIC ? fp4_stochastic(v, mix64(c.key + out * ((c.rows + 3) / 4) + first / 4 + g)) : fp4_nearest(v);
            if (!whole && first + 4 * g + 4 > c.rows) four = first + 4 * g < c.rows ? four & ((1u << (4 * (c.rows - first - 4 * g))) - 1) : 0;
            codes[g / 2] |= four << (16 * (g & 1));
        }
        if (16 * block < c.code_pitch) *(u32x4 DSLLM_GLOBAL *)(c.codes + out * c.code_pitch + 16 * block) = codes;
        if (block < c.scale_pitch) ((uint8_t DSLLM_GLOBAL *)c.scales)[out * c.scale_pitch + block] = uint8_t(byte);
    }
}

struct ValueArgs {
    const uint8_t *codes, *scales;
    uint64_t code_pitch, scale_pitch, rows, cols, ld;
    uint8_t *dst;
    uint64_t pieces;
};

// Eight elements a lane, 512 of a row a wave. Bound by memory: 45 M 4-bit values to bf16 17.3 us = 6.6 TB/s (more a lane is no faster), 8-bit ones
// 27 us; to f32, whose eight are two stores of half of every 32 bytes, 69 and 44.
constexpr uint32_t kValuePiece = 512;
template <int FORMAT, int DST>
__global__ __launch_bounds__(256) void values_kernel(ValueArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t item = uint64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t row = item / a.pieces, col = (item - row * a.pieces) * kValuePiece + 8 * lane;
    if (row >= a.rows || col >= a.cols) return;
    const float scale = scale_value(((const uint8_t DSLLM_GLOBAL *)a.scales)[row * a.scale_pitch + col / 32]);
    uint32_t codes[2];
    if constexpr (FORMAT == CKPT_MXFP4) {
        codes[0] = *(const uint32_t DSLLM_GLOBAL *)(a.codes + row * a.code_pitch + col / 2);
        codes[1] = codes[0] >> 16;
    } else {
        codes[0] = load_bytes(a.codes + row * a.code_pitch + col, uint32_t(min(a.cols - col, uint64_t(4))));
        codes[1] = col + 4 < a.cols ? load_bytes(a.codes + row * a.code_pitch + col + 4, uint32_t(min(a.cols - col - 4, uint64_t(4)))) : 0;
    }
    f32x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; h++) v[h] = FORMAT == CKPT_MXFP4 ? fp4_values(codes[h], scale) : fp8_values(codes[h]) * scale;
    uint8_t *at = a.dst + (row * a.ld + col) * sizeof(typename Element<DST>::one);
    if (col + 8 <= a.cols) store8<DST>(at, v[0], v[1]);
    else {
        store_upto4<DST>(at, v[0], uint32_t(a.cols - col));
        if (col + 4 < a.cols) store_upto4<DST>(at + 4 * sizeof(typename Element<DST>::one), v[1], uint32_t(a.cols - col - 4));
    }
}

uint64_t zeroed_blocks(const ckpt_mx_matrix &m) {
    const uint64_t codes = m.format == CKPT_MXFP4 ? m.code_pitch / 16 : (m.code_pitch + 31) / 32;
    return codes > m.scale_pitch ? codes : m.scale_pitch;
}

// Returns false if the grid would have 2^32 work-items or more.
bool fits_grid(uint64_t blocks) { return blocks < 1u << 24; }

template <int SRC>
bool launch_quantize(RowArgs rows, RowArgs cols, int format, bool by_row, bool by_col, int rounding, hipStream_t stream) {
    const bool stochastic = rounding & CKPT_ROUND_STOCHASTIC, nonzero = rounding & CKPT_ROUND_NONZERO;
    if (by_col) {
        const uint64_t across = ((by_row ? std::max(rows.cols, 32 * rows.blocks) : cols.cols) + 127) / 128, down = (std::max(cols.rows, 32 * cols.blocks) + 127) / 128;
        if (!fits_grid(across) || !fits_grid(down) || !fits_grid(across * down)) return false;
        const TileArgs p{rows, cols, uint32_t(across)};
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(across * down)), dim3(256), 0, stream, p); };
        if (by_row) stochastic ? go(tile_kernel<SRC, true, true>) : go(tile_kernel<SRC, false, true>);
        else stochastic ? go(tile_kernel<SRC, true, false>) : go(tile_kernel<SRC, false, false>);
        return true;
    }
    auto go = [&](auto kernel) {
        rows.pieces = (32 * rows.blocks + kRowPiece - 1) / kRowPiece;
        if (rows.pieces > 1ull << 30 || rows.rows > 1ull << 32 || !fits_grid((rows.rows * rows.pieces + 3) / 4)) return false;
        hipLaunchKernelGGL(kernel, dim3(unsigned((rows.rows * rows.pieces + 3) / 4)), dim3(256), 0, stream, rows);
        return true;
    };
    if (format == CKPT_MXFP4) return stochastic ? go(rows_kernel<SRC, CKPT_MXFP4, true, false>) : go(rows_kernel<SRC, CKPT_MXFP4, false, false>);
    if (nonzero) return stochastic ? go(rows_kernel<SRC, CKPT_MXFP8, true, true>) : go(rows_kernel<SRC, CKPT_MXFP8, false, true>);
    return stochastic ? go(rows_kernel<SRC, CKPT_MXFP8, true, false>) : go(rows_kernel<SRC, CKPT_MXFP8, false, false>);
}

int quantize(const void *src, int32_t dtype, int64_t ld, const ckpt_mx_matrix *by_row, const ckpt_mx_matrix *by_col, int32_t rounding, uint64_t seed, hipStream_t stream) {
    if (!by_row && !by_col) return refuse(CKPT_EINVAL, "neither by_row nor by_col");
    const uint32_t bytes = element_bytes(dtype);
    if (!bytes) return refuse(CKPT_EINVAL, "src_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    if (rounding < 0 || rounding > 3) return refuse(CKPT_EINVAL, "rounding is CKPT_ROUND_NEAREST or CKPT_ROUND_STOCHASTIC, with or without CKPT_ROUND_NONZERO");
    DeviceRanges ranges;
    for (const ckpt_mx_matrix *m : {by_row, by_col})
        if (m)
            if (const char *why = wrong_mx_matrix(m, ranges)) return refuse(CKPT_EINVAL, std::string(m == by_row ? "by_row: " : "by_col: ") + why);
    if (by_col && by_col->format != CKPT_MXFP4) return refuse(CKPT_EINVAL, "by_col: only CKPT_MXFP4");
    if (by_col && by_row && by_row->format != CKPT_MXFP4) return refuse(CKPT_EINVAL, "by_row: only CKPT_MXFP4 beside by_col");
    if (by_row && by_row->format == CKPT_MXFP4 && (rounding & CKPT_ROUND_NONZERO)) return refuse(CKPT_EINVAL, "CKPT_ROUND_NONZERO is for CKPT_MXFP8");
    if (by_col && (rounding & CKPT_ROUND_NONZERO)) return refuse(CKPT_EINVAL, "CKPT_ROUND_NONZERO is for CKPT_MXFP8");
    if (by_row && by_col && (by_row->rows != by_col->cols || by_row->cols != by_col->rows)) return refuse(CKPT_EINVAL, "by_col is not of the transpose's size");
    const int64_t rows = by_row ? by_row->rows : by_col->cols, cols = by_row ? by_row->cols : by_col->rows;
    if (rows == 0 || cols == 0) return CKPT_OK;
    if (ld < cols || ld > (1ll << 48) / rows) return refuse(CKPT_EINVAL, "ld is smaller than a row, or the matrix too large");
    if (uint64_t(src) % bytes) return refuse(CKPT_EINVAL, "src is not aligned to its element");
    if (const char *why = ranges.wrong(src, (uint64_t(rows - 1) * ld + cols) * bytes)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    RowArgs r{static_cast<const uint8_t *>(src), uint64_t(ld), uint64_t(rows), uint64_t(cols), nullptr, nullptr, 0, 0, 0, 0, 0}, c = r;
    auto fill = [](RowArgs &a, const ckpt_mx_matrix *m, uint64_t key) {
        if (!m) return;
        a.codes = static_cast<uint8_t *>(m->codes);
        a.scales = static_cast<uint8_t *>(m->scales);
        a.code_pitch = m->code_pitch;
        a.scale_pitch = m->scale_pitch;
        a.blocks = zeroed_blocks(*m);
        a.key = key;
    };
    fill(r, by_row, mix64(seed));
    fill(c, by_col, mix64(~seed));
    const int format = by_row ? by_row->format : CKPT_MXFP4;
    bool fits;
    switch (dtype) {
        case CKPT_F32: fits = launch_quantize<CKPT_F32>(r, c, format, by_row, by_col, rounding, stream); break;
        case CKPT_BF16: fits = launch_quantize<CKPT_BF16>(r, c, format, by_row, by_col, rounding, stream); break;
        default: fits = launch_quantize<CKPT_F16>(r, c, format, by_row, by_col, rounding, stream);
    }
    if (!fits) return refuse(CKPT_EINVAL, "the matrix takes more than 2^24 blocks of threads");
    return launched();
}

int dequantize(const ckpt_mx_matrix *m, void *dst, int32_t dtype, int64_t ld, hipStream_t stream) {
    if (!m) return refuse(CKPT_EINVAL, "null argument");
    const uint32_t bytes = element_bytes(dtype);
    if (!bytes) return refuse(CKPT_EINVAL, "dst_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    DeviceRanges ranges;
    if (const char *why = wrong_mx_matrix(m, ranges)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    if (m->rows == 0 || m->cols == 0) return CKPT_OK;
    if (ld < m->cols || ld > (1ll << 48) / m->rows) return refuse(CKPT_EINVAL, "ld is smaller than a row, or the matrix too large");
    if (uint64_t(dst) % bytes) return refuse(CKPT_EINVAL, "dst is not aligned to its element");
    if (const char *why = ranges.wrong(dst, (uint64_t(m->rows - 1) * ld + m->cols) * bytes)) return refuse(CKPT_EINVAL, std::string("dst: ") + why);
    ValueArgs a{static_cast<const uint8_t *>(m->codes), static_cast<const uint8_t *>(m->scales), m->code_pitch, m->scale_pitch,
                uint64_t(m->rows), uint64_t(m->cols), uint64_t(ld), static_cast<uint8_t *>(dst), 0};
    a.pieces = (a.cols + kValuePiece - 1) / kValuePiece;
    if (a.rows > 1ull << 32 || a.pieces > 1ull << 30 || !fits_grid((a.rows * a.pieces + 3) / 4)) return refuse(CKPT_EINVAL, "the matrix takes more than 2^24 blocks of threads");
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned((a.rows * a.pieces + 3) / 4)), dim3(256), 0, stream, a); };
    const bool four = m->format == CKPT_MXFP4;
    switch (dtype) {
        case CKPT_F32: four ? go(values_kernel<CKPT_MXFP4, CKPT_F32>) : go(values_kernel<CKPT_MXFP8, CKPT_F32>); break;
        case CKPT_BF16: four ? go(values_kernel<CKPT_MXFP4, CKPT_BF16>) : go(values_kernel<CKPT_MXFP8, CKPT_BF16>); break;
        default: four ? go(values_kernel<CKPT_MXFP4, CKPT_F16>) : go(values_kernel<CKPT_MXFP8, CKPT_F16>);
    }
    return launched();
}

}  // namespace

const char *dsllm::wrong_mx_matrix(const ckpt_mx_matrix *m, DeviceRanges &ranges) {
    if (m->format != CKPT_MXFP4 && m->format != CKPT_MXFP8) return "format must be CKPT_MXFP4 or CKPT_MXFP8";
    if (m->reserved) return "reserved field not zero";
    if (m->rows < 0 || m->cols < 0 || m->rows > 1ll << 40 || m->cols > 1ll << 40) return "rows or cols out of range";
    if (m->rows == 0 || m->cols == 0) return nullptr;
    const uint64_t cols = uint64_t(m->cols), rows = uint64_t(m->rows);
    if (m->format == CKPT_MXFP4) {
        if (m->code_pitch % 128 || m->scale_pitch % 16 || uint64_t(m->codes) % 16 || uint64_t(m->scales) % 16) return "pitches of 128 and 16, addresses of 16 bytes are wanted";
        if (m->code_pitch < (cols + 1) / 2 || m->scale_pitch < m->code_pitch / 16) return "a pitch is smaller than a row";
    } else if (m->code_pitch < cols || m->scale_pitch < (cols + 31) / 32) return "a pitch is smaller than a row";
    if (m->code_pitch > (1ull << 48) / rows || m->scale_pitch > (1ull << 48) / rows) return "the matrix is too large";
    if (const char *why = ranges.wrong(m->codes, rows * m->code_pitch)) return why;
    return ranges.wrong(m->scales, rows * m->scale_pitch);
}

extern "C" {

int ckpt_mx_layout(int32_t format, int64_t rows, int64_t cols, ckpt_mx_matrix *out) {
    return at_c_entry([&] {
        if (!out) return refuse(CKPT_EINVAL, "null argument");
        *out = ckpt_mx_matrix{};
        if (format != CKPT_MXFP4 && format != CKPT_MXFP8) return refuse(CKPT_EINVAL, "format must be CKPT_MXFP4 or CKPT_MXFP8");
        if (rows < 0 || cols < 0 || rows > 1ll << 40 || cols > 1ll << 40) return refuse(CKPT_EINVAL, "rows or cols out of range");
        const uint64_t c = uint64_t(cols);
        out->format = format;
        out->rows = rows;
        out->cols = cols;
        out->code_pitch = format == CKPT_MXFP4 ? (c + 255) / 256 * 128 : c;
        out->scale_pitch = format == CKPT_MXFP4 ? (c + 511) / 512 * 16 : (c + 31) / 32;
        return int(CKPT_OK);
    });
}

int ckpt_mx_quantize(const void *src, int32_t src_dtype, int64_t ld, const ckpt_mx_matrix *by_row, const ckpt_mx_matrix *by_col, int32_t rounding,
                     uint64_t seed, void *stream) {
    return at_c_entry([&] { return quantize(src, src_dtype, ld, by_row, by_col, rounding, seed, static_cast<hipStream_t>(stream)); });
}

int ckpt_mx_dequantize(const ckpt_mx_matrix *src, void *dst, int32_t dst_dtype, int64_t ld, void *stream) {
    return at_c_entry([&] { return dequantize(src, dst, dst_dtype, ld, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
