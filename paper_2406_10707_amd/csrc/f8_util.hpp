// Matrices in 8 bits with a scale for each block of 128 (include/ckpt_train.h): what their kernels share.
#pragma once
#include "train_util.hpp"

namespace dsllm {

// nullptr if the matrix is well formed and its codes and scales are device memory, else what is wrong
const char *wrong_f8_matrix(const ckpt_f8_matrix *m, DeviceRanges &ranges);

inline uint64_t f8_padded(int64_t cols) { return (uint64_t(cols) + 127) / 128 * 128; }

// `rows` of `width` bytes, `pitch` apart, from address `at` on
struct Rows {
    uint64_t at, width, pitch, rows;
    uint64_t end() const { return at + (rows - 1) * pitch + width; }
};
inline Rows plain_rows(const void *p, int64_t rows, int64_t cols, int64_t ld, uint32_t bytes) { return Rows{uint64_t(p), uint64_t(cols) * bytes, uint64_t(ld) * bytes, uint64_t(rows)}; }
// Whether they have a byte in common. Rows may lie between one another's; of different pitches, and more than 2^16 rows on both sides that lie in one range, they are taken to have.
bool share_bytes(const Rows &a, const Rows &b);
// Whether codes or scales do. An empty matrix shares nothing.
bool overlap(const ckpt_f8_matrix &a, const ckpt_f8_matrix &b);
bool overlap(const ckpt_f8_matrix &m, const Rows &rows);
bool overlaps_itself(const ckpt_f8_matrix &m);      // its codes with its scales

inline uint32_t f8_row_shift(const ckpt_f8_matrix &m) { return m.block_rows == 128 ? 7 : 0; }

// A matrix as kernels read or write it; codes nullptr: not wanted
struct F8Held {
    uint8_t *codes;
    float *scales;
    uint64_t code_pitch, scale_pitch;
    int64_t rows, cols;
    uint32_t shift;      // rows to a scale: 2^shift
    uint32_t e5m2;

    F8Held() : codes(nullptr), scales(nullptr), code_pitch(0), scale_pitch(0), rows(0), cols(0), shift(0), e5m2(0) {}
    explicit F8Held(const ckpt_f8_matrix *m) : F8Held() {
        if (!m) return;
        codes = static_cast<uint8_t *>(m->codes);
        scales = m->scales;
        code_pitch = m->code_pitch;
        scale_pitch = m->scale_pitch;
        rows = m->rows;
        cols = m->cols;
        shift = f8_row_shift(*m);
        e5m2 = m->format == CKPT_F8_E5M2;
    }
};

#if defined(__HIPCC__)
// ------------------------------------------------------------------ a block's scale, codes

__device__ __forceinline__ float f8_most(bool e5m2) { return e5m2 ? 57344.0f : 448.0f; }
// What the block's elements are multiplied with, from the bits of its largest magnitude. NaN for a block with an infinity or a NaN.
__device__ __forceinline__ float f8_inverse(uint32_t amax_bits, float most) {
    if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return fminf(most / __uint_as_float(amax_bits), 0x1p126f);
}
__device__ __forceinline__ float f8_scale(uint32_t amax_bits, float most) {
    if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return fmaxf(__uint_as_float(amax_bits) / most, 0x1p-126f);
}
// Codes of four values of at most the format's largest, element 0 lowest. The conversions round to nearest, ties to even. Each writes half of a word and leaves the other half: what is there before the first does not matter, and a value
// that is not needed any more is no instruction.
__device__ __forceinline__ uint32_t f8_codes(f32x4 y, bool e5m2) {
    int r = int(__float_as_uint(y[0]));
    if (e5m2) {
        r = __builtin_amdgcn_cvt_pk_bf8_f32(y[0], y[1], r, false);
        r = __builtin_amdgcn_cvt_pk_bf8_f32(y[2], y[3], r, true);
    } else {
        r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], r, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
    }
    return uint32_t(r);
}
__device__ __forceinline__ f32x4 f8_values(uint32_t codes, bool e5m2) {
    if (!e5m2) return fp8_values(codes);
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_bf8(int(codes), false), hi = __builtin_amdgcn_cvt_pk_f32_bf8(int(codes), true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// The larger of `most` and the magnitudes of four values, NaN if one is: v_maximum3_f32, two values an instruction.
__device__ __forceinline__ float larger(float most, f32x4 v) {
    most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_fabsf(v[0]), __builtin_fabsf(v[1])), most);
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_fabsf(v[2]), __builtin_fabsf(v[3])), most);
}
// Magnitudes' bits order like them, NaN (whose sign is cleared as any other's) above all.
__device__ __forceinline__ uint32_t bits_of(float magnitude) { return __float_as_uint(magnitude); }

// The largest of sixteen neighbouring lanes' values (lanes 16 i to 16 i + 15), in all of them.
__device__ __forceinline__ uint32_t most_of_16(uint32_t v) {
    v = most_of_8(v);
    return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x140, 0xF, 0xF, true)));      // the sixteen mirrored
}
// The same of several values at a time: between an instruction and one that takes its result from another lane stand those of the other values instead of waits.
template <int N>
__device__ __forceinline__ void most_of_16(uint32_t (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; k++) v[k] = max(v[k], uint32_t(__builtin_amdgcn_mov_dpp(int(v[k]), 0xB1, 0xF, 0xF, true)));
#pragma unroll
    for (int k = 0; k < N; k++) v[k] = max(v[k], uint32_t(__builtin_amdgcn_mov_dpp(int(v[k]), 0x4E, 0xF, 0xF, true)));
#pragma unroll
    for (int k = 0; k < N; k++) v[k] = max(v[k], uint32_t(__builtin_amdgcn_mov_dpp(int(v[k]), 0x141, 0xF, 0xF, true)));
#pragma unroll
    for (int k = 0; k < N; k++) v[k] = max(v[k], uint32_t(__builtin_amdgcn_mov_dpp(int(v[k]), 0x140, 0xF, 0xF, true)));
}

// Lane I's value of each sixteen neighbouring lanes, in all of them.
template <int I>
__device__ __forceinline__ float of_lane_of_16(float v) { return __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(int(__float_as_uint(v)), 0x150 + I, 0xF, 0xF, true))); }
// The largest of lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them.
__device__ __forceinline__ uint32_t most_of_quarters(uint32_t v) {
    v = max(v, uint32_t(__shfl_xor(int(v), 16)));
    return max(v, uint32_t(__shfl_xor(int(v), 32)));
}
#endif

}  // namespace dsllm
