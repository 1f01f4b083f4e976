// Conversion to block-scaled formats and back (include/ckpt_train.h).
#include "train_util.hpp"

using namespace dsllm;

namespace dsllm {
const char *wrong_mx_matrix(const ckpt_mx_matrix *m, DeviceRanges &ranges);
}

namespace {

struct RowArgs {
    const uint8_t *src;
    uint64_t ld;                // elements
    uint64_t rows, cols;
    uint8_t *codes, *scales;
    uint64_t code_pitch, scale_pitch;
    uint64_t blocks;            // of a row, with those behind its end that are to be zero
    uint64_t key;
};

// Eight lanes a block of 32 elements of a row, four each.
template <int SRC, int FORMAT, bool STOCHASTIC, bool NONZERO>
__global__ __launch_bounds__(256) void rows_kernel(RowArgs a) {
    const uint64_t total = a.rows * a.blocks, per_row = (a.cols + 3) / 4;
    for (uint64_t b = uint64_t(blockIdx.x) * 32 + threadIdx.x / 8; b < total; b += uint64_t(gridDim.x) * 32) {
        const uint64_t row = b / a.blocks, block = b - row * a.blocks, col = 32 * block + 4 * (threadIdx.x & 7);
        const uint32_t count = col < a.cols ? uint32_t(a.cols - col < 4 ? a.cols - col : 4) : 0;
        const f32x4 x = load_upto4<SRC>(a.src + (row * a.ld + col) * sizeof(typename Element<SRC>::one), count);
        const uint32_t byte = scale_byte<FORMAT>(most_of_8(magnitude_bits(x)));
        const f32x4 y = x * inverse_scale(byte);
        uint32_t codes;
        if constexpr (STOCHASTIC) {
            const uint64_t r = mix64(a.key + row * per_row + col / 4);
            codes = FORMAT == CKPT_MXFP4 ? fp4_stochastic(y, r) : fp8_stochastic<NONZERO>(y, r);
        } else {
            codes = FORMAT == CKPT_MXFP4 ? fp4_nearest(y) : fp8_nearest<NONZERO>(y);
        }
        if (FORMAT == CKPT_MXFP4) {
            if (count < 4) codes &= (1u << (4 * count)) - 1;
            if (col / 2 < a.code_pitch) *(uint16_t DSLLM_GLOBAL *)(a.codes + row * a.code_pitch + col / 2) = uint16_t(codes);
        } else {
            if (count < 4) codes &= (1u << (8 * count)) - 1;
            if (col < a.code_pitch) store_bytes(a.codes + row * a.code_pitch + col, codes, uint32_t(a.code_pitch - col < 4 ? a.code_pitch - col : 4));
        }
        if ((threadIdx.x & 7) == 0 && block < a.scale_pitch) a.scales[row * a.scale_pitch + block] = uint8_t(byte);
    }
}

// A thread a block of 32 elements of a column: row `col` of the transpose. Blocks behind the last row are zero.
template <int SRC, bool STOCHASTIC>
__global__ __launch_bounds__(256) void columns_kernel(RowArgs a) {      // rows, cols: of src; codes, scales: of its transpose
    const uint64_t total = a.cols * a.blocks, per_row = (a.rows + 3) / 4;
    for (uint64_t t = uint64_t(blockIdx.x) * 256 + threadIdx.x; t < total; t += uint64_t(gridDim.x) * 256) {
        const uint64_t block = t / a.cols, col = t - block * a.cols, row = 32 * block;
        f32x4 x[8];
        uint32_t most = 0;
#pragma unroll
        for (int g = 0; g < 8; g++) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint64_t r = row + 4 * g + j;
                x[g][j] = r < a.rows ? float(((const typename Element<SRC>::one DSLLM_GLOBAL *)a.src)[r * a.ld + col]) : 0.0f;
            }
            most = max(most, magnitude_bits(x[g]));
        }
        const uint32_t byte = scale_byte<CKPT_MXFP4>(most);
        u32x4 codes{0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < 8; g++) {
            const f32x4 y = x[g] * inverse_scale(byte);
            uint32_t c = STOCHASTIC ? fp4_stochastic(y, mix64(a.key + col * per_row + row / 4 + g)) : fp4_nearest(y);
            if (row + 4 * g + 4 > a.rows) c = row + 4 * g < a.rows ? c & ((1u << (4 * (a.rows - row - 4 * g))) - 1) : 0;
            codes[g / 2] |= c << (16 * (g & 1));
        }
        if (16 * block < a.code_pitch) *(u32x4 DSLLM_GLOBAL *)(a.codes + col * a.code_pitch + 16 * block) = codes;
        if (block < a.scale_pitch) a.scales[col * a.scale_pitch + block] = uint8_t(byte);
    }
}

struct ValueArgs {
    const uint8_t *codes, *scales;
    uint64_t code_pitch, scale_pitch, rows, cols, ld;
    uint8_t *dst;
};

template <int FORMAT, int DST>
__global__ __launch_bounds__(256) void values_kernel(ValueArgs a) {
    const uint64_t per_row = (a.cols + 3) / 4, total = a.rows * per_row;
    for (uint64_t t = uint64_t(blockIdx.x) * 256 + threadIdx.x; t < total; t += uint64_t(gridDim.x) * 256) {
        const uint64_t row = t / per_row, col = 4 * (t - row * per_row);
        const uint32_t count = uint32_t(a.cols - col < 4 ? a.cols - col : 4);
        const float scale = scale_value(a.scales[row * a.scale_pitch + col / 32]);
        f32x4 v;
        if constexpr (FORMAT == CKPT_MXFP4) v = fp4_values(*(const uint16_t DSLLM_GLOBAL *)(a.codes + row * a.code_pitch + col / 2), scale);
        else v = fp8_values(load_bytes(a.codes + row * a.code_pitch + col, count)) * scale;
        store_upto4<DST>(a.dst + (row * a.ld + col) * sizeof(typename Element<DST>::one), v, count);
    }
}

unsigned grid_for(uint64_t items, unsigned per_block) {
    const uint64_t blocks = (items + per_block - 1) / per_block, most = 1u << 20;
    return unsigned(blocks < most ? blocks : most);
}

uint64_t zeroed_blocks(const ckpt_mx_matrix &m) {
    const uint64_t codes = m.format == CKPT_MXFP4 ? m.code_pitch / 16 : (m.code_pitch + 31) / 32;
    return codes > m.scale_pitch ? codes : m.scale_pitch;
}

template <int SRC>
void launch_quantize(const RowArgs &rows, const RowArgs &cols, int format, bool by_row, bool by_col, int rounding, hipStream_t stream) {
    const bool stochastic = rounding & CKPT_ROUND_STOCHASTIC, nonzero = rounding & CKPT_ROUND_NONZERO;
    if (by_row) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid_for(rows.rows * rows.blocks, 32)), dim3(256), 0, stream, rows); };
        if (format == CKPT_MXFP4) stochastic ? go(rows_kernel<SRC, CKPT_MXFP4, true, false>) : go(rows_kernel<SRC, CKPT_MXFP4, false, false>);
        else if (nonzero) stochastic ? go(rows_kernel<SRC, CKPT_MXFP8, true, true>) : go(rows_kernel<SRC, CKPT_MXFP8, false, true>);
        else stochastic ? go(rows_kernel<SRC, CKPT_MXFP8, true, false>) : go(rows_kernel<SRC, CKPT_MXFP8, false, false>);
    }
    if (by_col) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid_for(cols.cols * cols.blocks, 256)), dim3(256), 0, stream, cols); };
        stochastic ? go(columns_kernel<SRC, true>) : go(columns_kernel<SRC, false>);
    }
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
    if (by_row && by_row->format == CKPT_MXFP4 && (rounding & CKPT_ROUND_NONZERO)) return refuse(CKPT_EINVAL, "CKPT_ROUND_NONZERO is for CKPT_MXFP8");
    if (by_col && (rounding & CKPT_ROUND_NONZERO)) return refuse(CKPT_EINVAL, "CKPT_ROUND_NONZERO is for CKPT_MXFP8");
    if (by_row && by_col && (by_row->rows != by_col->cols || by_row->cols != by_col->rows)) return refuse(CKPT_EINVAL, "by_col is not of the transpose's size");
    const int64_t rows = by_row ? by_row->rows : by_col->cols, cols = by_row ? by_row->cols : by_col->rows;
    if (rows == 0 || cols == 0) return CKPT_OK;
    if (ld < cols || ld > (1ll << 48) / rows) return refuse(CKPT_EINVAL, "ld is smaller than a row, or the matrix too large");
    if (uint64_t(src) % bytes) return refuse(CKPT_EINVAL, "src is not aligned to its element");
    if (const char *why = ranges.wrong(src, (uint64_t(rows - 1) * ld + cols) * bytes)) return refuse(CKPT_EINVAL, std::string("src: ") + why);
    RowArgs r{static_cast<const uint8_t *>(src), uint64_t(ld), uint64_t(rows), uint64_t(cols), nullptr, nullptr, 0, 0, 0, 0}, c = r;
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
    switch (dtype) {
        case CKPT_F32: launch_quantize<CKPT_F32>(r, c, format, by_row, by_col, rounding, stream); break;
        case CKPT_BF16: launch_quantize<CKPT_BF16>(r, c, format, by_row, by_col, rounding, stream); break;
        default: launch_quantize<CKPT_F16>(r, c, format, by_row, by_col, rounding, stream);
    }
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
    const ValueArgs a{static_cast<const uint8_t *>(m->codes), static_cast<const uint8_t *>(m->scales), m->code_pitch, m->scale_pitch,
                      uint64_t(m->rows), uint64_t(m->cols), uint64_t(ld), static_cast<uint8_t *>(dst)};
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid_for(a.rows * ((a.cols + 3) / 4), 256)), dim3(256), 0, stream, a); };
    const bool four = m->format == CKPT_MXFP4;
    switch (dtype) {
        case CKPT_F32: four ? go(values_kernel<CKPT_MXFP4, CKPT_F32>) : go(values_kernel<CKPT_MXFP8, CKPT_F32>); break;
        case CKPT_BF16: four ? go(values_kernel<CKPT_MXFP4, CKPT_BF16>) : go(values_kernel<CKPT_MXFP8, CKPT_BF16>); break;
        default: four ? go(values_kernel<CKPT_MXFP4, CKPT_F16>) : go(values_kernel<CKPT_MXFP8, CKPT_F16>);
    }
    return launched();
}

}  // namespace

// nullptr if the matrix is well formed and its rows are device memory
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
