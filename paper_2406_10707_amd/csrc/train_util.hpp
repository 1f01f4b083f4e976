// What the operators of include/ckpt_train.h share: argument checks on the host, random bits and block-scaled formats on the device.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <new>
#include <string>

#include "../../include/ckpt.h"
#include "../../include/ckpt_train.h"
#include "kernel_util.hpp"

namespace dsllm {

extern thread_local std::string g_last_error;
inline int refuse(int code, const char *text) {
    try { g_last_error = text; } catch (...) {}
    return code;
}
inline int refuse(int code, const std::string &text) { return refuse(code, text.c_str()); }
// Nothing is thrown out of a C entry point.
template <class F>
int at_c_entry(F f) {
    try { return f(); }
    catch (const std::bad_alloc &) { return refuse(CKPT_ENOMEM, "out of host memory"); }
    catch (...) { return refuse(CKPT_EINVAL, "unexpected failure"); }
}
inline int launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CKPT_OK : refuse(CKPT_EHIP, hipGetErrorString(e));
}

// Whether address ranges are device memory of the current GPU, inside their allocations. Keeps the latest allocation: a list's
// tensors mostly share a few, and two queries are 0.12 us.
class DeviceRanges {
    int dev_ = -1;
    uint64_t lo_ = 1, hi_ = 0;

public:
    // nullptr if it is, else what is wrong
    const char *wrong(const void *p, uint64_t nbytes) {
        if (!p) return "null device pointer";
        const uint64_t a = uint64_t(p);
        if (a < lo_ || a >= hi_) {
            if (dev_ < 0 && hipGetDevice(&dev_) != hipSuccess) { (void)hipGetLastError(); return "no current device"; }
            hipPointerAttribute_t attr;
            if (hipPointerGetAttributes(&attr, p) != hipSuccess || attr.type != hipMemoryTypeDevice || attr.device != dev_) {
                (void)hipGetLastError();
                return "not device memory of the current GPU";
            }
            void *base = nullptr;
            size_t span = 0;
            if (hipMemGetAddressRange(reinterpret_cast<hipDeviceptr_t *>(&base), &span, reinterpret_cast<hipDeviceptr_t>(const_cast<void *>(p))) != hipSuccess) {
                (void)hipGetLastError();
                return "not inside a device allocation";
            }
            lo_ = uint64_t(base);
            hi_ = lo_ + span;
        }
        return a < lo_ || a >= hi_ || nbytes > hi_ - a ? "range runs past its allocation" : nullptr;
    }
};

// nullptr if the matrix is well formed and its rows are device memory, else what is wrong
const char *wrong_mx_matrix(const ckpt_mx_matrix *m, DeviceRanges &ranges);

inline uint32_t element_bytes(int32_t dtype) { return dtype == CKPT_F32 ? 4 : dtype == CKPT_BF16 || dtype == CKPT_F16 ? 2 : 0; }

// ------------------------------------------------------------------ random bits (ckpt_proxy.h: mix)

__host__ __device__ __forceinline__ uint64_t mix64(uint64_t x) {
    uint64_t z = x + 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

#if defined(__HIPCC__)
// ------------------------------------------------------------------ loads and stores of four elements at any element's address

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
template <int DTYPE> struct Element;
template <> struct Element<CKPT_F32> { typedef float one; typedef f32x4 four; };
template <> struct Element<CKPT_BF16> { typedef __bf16 one; typedef bf16x4 four; };
template <> struct Element<CKPT_F16> { typedef _Float16 one; typedef f16x4 four; };

// Four elements as f32; the target takes vector accesses at any address.
template <int DTYPE>
__device__ __forceinline__ f32x4 load4(const void *p) {
    typedef typename Element<DTYPE>::four four_bytealigned __attribute__((aligned(1)));
    return __builtin_convertvector(__builtin_nontemporal_load((const four_bytealigned DSLLM_GLOBAL *)p), f32x4);
}
template <int DTYPE>
__device__ __forceinline__ void store4(void *p, f32x4 v) {
    typedef typename Element<DTYPE>::four four_bytealigned __attribute__((aligned(1)));
    __builtin_nontemporal_store(__builtin_convertvector(v, typename Element<DTYPE>::four), (four_bytealigned DSLLM_GLOBAL *)p);
}
template <int DTYPE>
__device__ __forceinline__ void store8(void *p, f32x4 lo, f32x4 hi) {
    if constexpr (DTYPE == CKPT_F32) {
        store4<DTYPE>(p, lo);
        store4<DTYPE>(static_cast<float *>(p) + 4, hi);
    } else {
        typedef typename Element<DTYPE>::one eight __attribute__((ext_vector_type(8)));
        typedef eight eight_bytealigned __attribute__((aligned(1)));
        const typename Element<DTYPE>::four a = __builtin_convertvector(lo, typename Element<DTYPE>::four), b = __builtin_convertvector(hi, typename Element<DTYPE>::four);
        __builtin_nontemporal_store(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), (eight_bytealigned DSLLM_GLOBAL *)p);
    }
}
// Eight elements, as they are stored; 16 bytes an access.
template <int DTYPE>
struct Eight {
    typename Element<DTYPE>::four lo, hi;
    __device__ __forceinline__ void load(const void *p) {
        if constexpr (DTYPE == CKPT_F32) {
            typedef f32x4 four_bytealigned __attribute__((aligned(1)));
            lo = ((const four_bytealigned DSLLM_GLOBAL *)p)[0];      // not as read once: each access takes half of every 32 bytes
            hi = ((const four_bytealigned DSLLM_GLOBAL *)p)[1];
        } else {
            typedef typename Element<DTYPE>::one eight __attribute__((ext_vector_type(8)));
            typedef eight eight_bytealigned __attribute__((aligned(1)));
            const eight e = __builtin_nontemporal_load((const eight_bytealigned DSLLM_GLOBAL *)p);
            lo = __builtin_shufflevector(e, e, 0, 1, 2, 3);
            hi = __builtin_shufflevector(e, e, 4, 5, 6, 7);
        }
    }
    // the first `count` of them, 0 in the place of the others
    __device__ __forceinline__ void load_upto(const void *p, uint32_t count) {
        if (count >= 8) return load(p);
        typedef const typename Element<DTYPE>::one DSLLM_GLOBAL *Pointer;
#pragma unroll
        for (uint32_t j = 0; j < 8; j++) (j < 4 ? lo : hi)[j & 3] = j < count ? ((Pointer)p)[j] : typename Element<DTYPE>::one(0);
    }
};
// The first `count` of them, 0 in the place of the others.
template <int DTYPE>
__device__ __forceinline__ f32x4 load_upto4(const void *p, uint32_t count) {
    typedef const typename Element<DTYPE>::one DSLLM_GLOBAL *Pointer;
    if (count >= 4) return load4<DTYPE>(p);
    f32x4 v{0, 0, 0, 0};
    for (uint32_t j = 0; j < 3; j++)
        if (j < count) v[j] = float(((Pointer)p)[j]);
    return v;
}
template <int DTYPE>
__device__ __forceinline__ void store_upto4(void *p, f32x4 v, uint32_t count) {
    typedef typename Element<DTYPE>::one one;
    if (count >= 4) return store4<DTYPE>(p, v);
    for (uint32_t j = 0; j < 3; j++)
        if (j < count) ((one DSLLM_GLOBAL *)p)[j] = one(v[j]);
}
typedef uint32_t u32_bytealigned __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t load_bytes(const uint8_t *p, uint32_t count) {
    if (count >= 4) return __builtin_nontemporal_load((const u32_bytealigned DSLLM_GLOBAL *)p);
    uint32_t v = 0;
    for (uint32_t j = 0; j < 3; j++)
        if (j < count) v |= uint32_t(((const uint8_t DSLLM_GLOBAL *)p)[j]) << (8 * j);
    return v;
}
__device__ __forceinline__ void store_bytes(uint8_t *p, uint32_t v, uint32_t count) {
    if (count >= 4) { __builtin_nontemporal_store(v, (u32_bytealigned DSLLM_GLOBAL *)p); return; }
    for (uint32_t j = 0; j < 3; j++)
        if (j < count) ((uint8_t DSLLM_GLOBAL *)p)[j] = uint8_t(v >> (8 * j));
}

// ------------------------------------------------------------------ block-scaled formats

// The smallest power of two at which the largest value fits: the exponent of amax less the exponent of 6 (448), one more if
// amax's fraction is above that of 6 (448). Infinities and NaN give 255. The bits of |x| order like |x|, NaN above all.
template <int FORMAT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return 255;
    const int below = FORMAT == CKPT_MXFP4 ? 2 : 8;
    const uint32_t round_up = 0x800000u - 1 - (FORMAT == CKPT_MXFP4 ? 0x400000u : 0x600000u);
    const int e = int((amax_bits + round_up) >> 23) - below;
    return e < 0 ? 0 : uint32_t(e);
}
// 2^(127 - byte), and NaN for byte 255: what a block's values are multiplied with. Bytes other than that are at most 253.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7FC00000u : (254 - byte) << 23); }
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7FC00000u : byte == 0 ? 0x00400000u : byte << 23);
}

// Sixteen random bits of element j
__device__ __forceinline__ uint32_t field(uint64_t r, int j) { return uint32_t(r >> (16 * j)) & 0xFFFFu; }

// E2M1 codes of four values of at most 6, element 0 lowest: sixteen bits.
__device__ __forceinline__ uint32_t fp4_nearest(f32x4 y) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[0], y[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[2], y[3], 1.0f, 1);
    return r & 0xFFFFu;
}
// From 1 on a code is the upper bits of the f32 pattern, the 22 below are rounded away; smaller values are multiples of 0.5. Rounding is adding the random bits at the place of what
// is cut off and cutting. NaN gives some code (its block's scale says NaN).
__device__ __forceinline__ uint32_t fp4_stochastic(f32x4 y, uint64_t random) {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float a = fabsf(y[j]);
        const uint32_t bits = field(random, j);
        const uint32_t normal = ((__float_as_uint(a) + (bits << 6)) >> 22) - 252u;
        const uint32_t small = (uint32_t(fminf(a, 1.0f) * 131072.0f) + bits) >> 16;
        const uint32_t code = a >= 1.0f ? normal : small;
        r |= (code & 7u) << (4 * j) | (__float_as_uint(y[j]) >> 31) << (4 * j + 3);
    }
    return r;
}
// E4M3 codes of four values y = x / scale of at most 448, element 0 in the lowest byte. NaN gives some code (its block's scale says NaN). NONZERO: what is not zero is at least code 1. That
// is x's to say: y is zero where x lies 2^149 and more below the block's largest.
template <bool NONZERO>
__device__ __forceinline__ uint32_t fp8_nearest(f32x4 y, f32x4 x) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
    uint32_t codes = uint32_t(r);
    if (NONZERO) {
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (x[j] != 0 && !(codes & (0x7Fu << (8 * j)))) codes |= 1u << (8 * j);
    }
    return codes;
}
// From 2^-6 on a code is the upper bits of the f32 pattern, the twenty below are rounded away; smaller values are multiples of 2^-9. SIGNED: there may be negative ones.
template <bool NONZERO, bool SIGNED = true>
__device__ __forceinline__ uint32_t fp8_stochastic(f32x4 y, f32x4 x, uint64_t random) {
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float a = SIGNED ? fabsf(y[j]) : y[j];
        const uint32_t bits = field(random, j);
        const uint32_t normal = ((__float_as_uint(a) + (bits << 4)) >> 20) - 960u;
        const uint32_t small = (uint32_t(fminf(a, 0.015625f) * 33554432.0f) + bits) >> 16;
        uint32_t code = a >= 0.015625f ? normal : small;
        if (NONZERO) code = max(code, min(__float_as_uint(SIGNED ? fabsf(x[j]) : x[j]), 1u));
        if (SIGNED) code = (code & 0x7Fu) | (__float_as_uint(y[j]) >> 31 << 7);
        else code &= 0xFFu;
        r |= code << (8 * j);
    }
    return r;
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f32x4 fp8_values(uint32_t codes) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
// The values of four E2M1 codes times a power of two.
__device__ __forceinline__ f32x4 fp4_values(uint32_t codes, float scale) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    return f32x4{lo[0], lo[1], hi[0], hi[1]} * scale;
}

// The largest of eight neighbouring lanes' values (lanes 8 i to 8 i + 7), in all of them.
__device__ __forceinline__ uint32_t most_of_8(uint32_t v) {
    v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0xB1, 0xF, 0xF, true)));     // neighbours exchanged
    v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x4E, 0xF, 0xF, true)));     // pairs exchanged
    return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x141, 0xF, 0xF, true)));  // the eight mirrored
}
// Of four neighbouring lanes
__device__ __forceinline__ uint32_t most_of_4(uint32_t v) {
    v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0xB1, 0xF, 0xF, true)));
    return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x4E, 0xF, 0xF, true)));
}
__device__ __forceinline__ uint32_t magnitude_bits(f32x4 v) {
    const uint32_t m = 0x7FFFFFFFu;
    return max(max(__float_as_uint(v[0]) & m, __float_as_uint(v[1]) & m), max(__float_as_uint(v[2]) & m, __float_as_uint(v[3]) & m));
}
#endif

}  // namespace dsllm
