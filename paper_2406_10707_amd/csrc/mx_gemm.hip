// The product of two MXFP4 matrices on the matrix cores (include/ckpt_train.h).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 E2M1 values: lane l holds the 32 consecutive values (16 bytes) of row
// l mod 16 that make up block l / 16 of the step, and that block's scale byte. A and B are both kept by rows along K, so both sides
// are read the same way; the instruction applies the two scales of a block to its partial sum.
#include "train_util.hpp"

using namespace dsllm;

namespace dsllm {
const char *wrong_mx_matrix(const ckpt_mx_matrix *m, DeviceRanges &ranges);
}

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct GemmArgs {
    const uint8_t *a, *b, *a_scale, *b_scale;
    uint64_t a_pitch, b_pitch, a_scale_pitch, b_scale_pitch;
    void *c;
    int64_t ldc;
    int64_t m, n;
    uint32_t steps;        // of 128 values
    int accumulate;
};

__device__ __forceinline__ f32x4 mfma_fp4(u32x4 a, u32x4 b, f32x4 c, uint32_t a_scale, uint32_t b_scale) {
    const i32x8 a8{int(a.x), int(a.y), int(a.z), int(a.w), 0, 0, 0, 0}, b8{int(b.x), int(b.y), int(b.z), int(b.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, int(a_scale), 0, int(b_scale));
}

// Four waves compute 64 x 64, a wave 32 x 32, straight from memory. Rows past the end are the last row again, and not stored.
template <int OUT>
__global__ __launch_bounds__(256) void gemm_simple_kernel(GemmArgs p) {
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
    for (uint32_t s = 0; s < p.steps; s++) {
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
            for (int j = 0; j < 2; j++) acc[i][j] = mfma_fp4(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
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
    (void)workspace; (void)workspace_bytes;
    GemmArgs p{static_cast<const uint8_t *>(a->codes), static_cast<const uint8_t *>(b->codes), static_cast<const uint8_t *>(a->scales), static_cast<const uint8_t *>(b->scales),
               a->code_pitch, b->code_pitch, a->scale_pitch, b->scale_pitch, c, ldc, m, n, uint32_t((k + 127) / 128), accumulate};
    const dim3 grid(unsigned((n + 63) / 64), unsigned((m + 63) / 64));
    if (grid.y > 65535) return refuse(CKPT_EINVAL, "too many rows");
    if (dtype == CKPT_F32) hipLaunchKernelGGL(gemm_simple_kernel<CKPT_F32>, grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(gemm_simple_kernel<CKPT_BF16>, grid, dim3(256), 0, stream, p);
    return launched();
}

}  // namespace

extern "C" {

int ckpt_mx_gemm_workspace(int64_t m, int64_t n, int64_t k, uint64_t *bytes) {
    return at_c_entry([&] {
        if (!bytes || m < 0 || n < 0 || k < 0) return refuse(CKPT_EINVAL, "null argument or negative size");
        *bytes = 0;
        return int(CKPT_OK);
    });
}

int ckpt_mx_gemm(const ckpt_mx_matrix *a, const ckpt_mx_matrix *b, void *c, int32_t c_dtype, int64_t ldc, int32_t accumulate, void *workspace,
                 uint64_t workspace_bytes, void *stream) {
    return at_c_entry([&] { return gemm(a, b, c, c_dtype, ldc, accumulate, workspace, workspace_bytes, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
