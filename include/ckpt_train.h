/*
 * The operators of a training step around the shard that libdsllm_ckpt snapshots: the norm of all gradients with the
 * clipping factor, the AdamW step over the whole tensor list with moments in 32 or in 8 bits, block-scaled 4-bit and 8-bit
 * floating point (the OCP microscaling formats MXFP4 and MXFP8 E4M3), and the product of two MXFP4 matrices.
 *
 * Same conventions as ckpt.h: plain C ABI, "dev" pointers are device memory of the CURRENT HIP device, a stream argument
 * is a hipStream_t passed as void*, calls return a ckpt_status (0 = ok, negative = error) and never throw or abort,
 * ckpt_last_error() gives the text. Bad arguments are refused before anything is launched. Every call but
 * ckpt_optim_create and ckpt_optim_destroy only enqueues on the stream: it neither allocates nor waits, so it may be
 * captured into a HIP graph (the numbers passed by value, the step number among them, are then part of the graph).
 * Calls on different streams may overlap as long as they write different memory. All kernels are deterministic: the
 * same inputs give the same bits, whatever else runs.
 */
#ifndef DSLLM_CKPT_TRAIN_H
#define DSLLM_CKPT_TRAIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- block-scaled matrices ----
 *
 * A row's elements are divided into blocks of 32; a block shares the scale 2^(byte - 127) (E8M0), byte 255 makes all 32 NaN.
 *   CKPT_MXFP4  E2M1 codes, two to a byte, the even column in the low half: 0 .5 1 1.5 2 3 4 6, bit 3 the sign
 *   CKPT_MXFP8  E4M3 codes (no infinities, 0x7F is NaN), one to a byte
 * The scale of a block is the smallest power of two (at least 2^-127) at which no element lies beyond the format's largest
 * value (6; 448): nothing saturates. A block with an infinity or a NaN is NaN as a whole; one of zeros has byte 0.
 * Elements are rounded to the nearest value, ties to the even code, or stochastically: with |x| between n and n + 1 steps
 * of the grid, floor(|x| / step + r / 65536) steps, r sixteen bits drawn for the element. The four elements 4g .. 4g + 3 of
 * a row take the sixteen-bit fields, lowest first, of mix(key + row * ceil(cols / 4) + g), mix as in ckpt_proxy.h.
 * (A float above 3.5 * 2^126 may stand for infinity once rounded up.) */
typedef enum { CKPT_MXFP4 = 1, CKPT_MXFP8 = 2 } ckpt_mx_format;
typedef enum { CKPT_ROUND_NEAREST = 0, CKPT_ROUND_STOCHASTIC = 1,
               CKPT_ROUND_NONZERO = 2 /* or'ed in, MXFP8: what is not zero becomes at least the smallest value */ } ckpt_rounding;

/* rows x cols elements. Row r: codes at codes + r * code_pitch, scales at scales + r * scale_pitch.
 * MXFP4: code_pitch a multiple of 128 that holds cols / 2 bytes, scale_pitch a multiple of 16 that holds a byte for each
 * block of the pitch (code_pitch / 16), both addresses 16-byte aligned; what a row has behind its last element is zero
 * (ckpt_mx_quantize writes it so, ckpt_mx_gemm relies on it). MXFP8: pitches of at least cols and ceil(cols / 32) bytes; ckpt_mx_quantize
 * writes all of a row's pitch here too, zeros behind its last element. Rows of a matrix may not overlap. */
typedef struct {
    int32_t format;        /* ckpt_mx_format */
    int32_t reserved;      /* must be zero */
    int64_t rows, cols;
    void *codes;
    uint64_t code_pitch;
    void *scales;
    uint64_t scale_pitch;
} ckpt_mx_matrix;

/* Fills format, rows, cols and the smallest pitches; codes and scales are set to NULL. The caller allocates
 * rows * code_pitch and rows * scale_pitch bytes. */
int ckpt_mx_layout(int32_t format, int64_t rows, int64_t cols, ckpt_mx_matrix *out);

/* Rounds src, a row-major matrix of src_dtype (CKPT_F32, CKPT_BF16, CKPT_F16; aligned to its element) with `ld` elements from row
 * to row, to by_row (rows x cols, blocks along the columns) and / or by_col (the transpose: cols x rows, blocks along the
 * rows), in one pass over src. Either may be NULL. by_col takes MXFP4 only, as does by_row beside it. Random bits: key = mix(seed) for by_row, mix(~seed) for
 * by_col. A product that contracts over the columns of src takes by_row, one that contracts over its rows by_col. */
int ckpt_mx_quantize(const void *src, int32_t src_dtype, int64_t ld, const ckpt_mx_matrix *by_row, const ckpt_mx_matrix *by_col,
                     int32_t rounding, uint64_t seed, void *stream);

/* The values that a matrix stands for, as a row-major matrix of dst_dtype with `ld` elements from row to row. */
int ckpt_mx_dequantize(const ckpt_mx_matrix *src, void *dst, int32_t dst_dtype, int64_t ld, void *stream);

/* C = A * B^T, or C += A * B^T with accumulate != 0. A is M x K, B is N x K, both MXFP4; C is row-major, CKPT_BF16 or CKPT_F32, `ldc`
 * elements from row to row. Accumulated in f32 on the matrix cores; one rounding at the end. A linear layer y = x W^T takes (x, W)
 * forward, (dy, W by columns) for dx and (dy by columns, x by columns) for dW. Some sizes split K among blocks and need
 * workspace: ckpt_mx_gemm_workspace bytes (16-byte aligned, contents do not matter, not shared by calls that may overlap);
 * with less (or NULL) the call runs with fewer parts or unsplit. C must not overlap A, B or the workspace. */
int ckpt_mx_gemm_workspace(int64_t m, int64_t n, int64_t k, uint64_t *bytes);
int ckpt_mx_gemm(const ckpt_mx_matrix *a, const ckpt_mx_matrix *b, void *c, int32_t c_dtype, int64_t ldc, int32_t accumulate,
                 void *workspace, uint64_t workspace_bytes, void *stream);

/* ---- the update phase over a list of tensors ---- */

typedef struct ckpt_optim ckpt_optim;   /* opaque, library-owned: the list, laid out on the device */

/* One parameter tensor, all parts contiguous and aligned to their element size only. An optimizer that is only asked for
 * the norm needs numel and dev_grad alone (dev_master NULL in every tensor). */
typedef struct {
    uint64_t numel;          /* 0: nothing to do */
    const void *dev_grad;    /* grad_dtype */
    void *dev_param;         /* the working copy, written only; param_dtype, ignored if that is 0 */
    float *dev_master;       /* f32 master weights */
    void *dev_m, *dev_v;     /* first and second moment: f32, or E4M3 codes */
    void *dev_m_scale, *dev_v_scale;  /* 8-bit moments: ceil(numel / 32) scale bytes each */
    double weight_decay;
} ckpt_optim_tensor;

typedef struct {
    int32_t grad_dtype;      /* CKPT_F32, CKPT_BF16, CKPT_F16 */
    int32_t param_dtype;     /* CKPT_BF16, CKPT_F16, or 0: no working copy */
    int32_t state_bits;      /* 32 or 8 */
    int32_t reserved;        /* must be zero */
} ckpt_optim_config;

/* Copies the list to the device, once. The memory must stay allocated, at these addresses, while the handle lives.
 * Tensors must not overlap. A handle belongs to the device that was current, and to one stream at a time (its
 * ckpt_optim_grad_norm calls share scratch memory). */
int ckpt_optim_create(const ckpt_optim_tensor *tensors, size_t n, const ckpt_optim_config *cfg, ckpt_optim **out);
/* Waits for the handle's device, whichever is current, then frees the handle. */
int ckpt_optim_destroy(ckpt_optim *opt);
/* New gradient addresses, one for each tensor, for work enqueued behind this on the stream. */
int ckpt_optim_set_grads(ckpt_optim *opt, const void *const *dev_grads, size_t n, void *stream);

/* What ckpt_optim_grad_norm writes, in device memory (8-byte aligned). */
typedef struct {
    double sum_squares;      /* of all gradients as they are, for a sum over ranks */
    float norm;              /* grad_scale * sqrt(sum_squares) */
    float scale;             /* what the step multiplies gradients with: grad_scale * min(1, max_norm / norm) */
    int32_t nonfinite;       /* 1: a gradient is an infinity or a NaN, or f32 does not hold what the step would make of them: norm
                                above f32's largest, or what clipping leaves of it above 2^63. The step then changes nothing */
    int32_t reserved;
} ckpt_norm_result;

/* grad_scale: what gradients are to be multiplied with in any case (1 / (loss scale * accumulated batches)).
 * At least 0. max_norm <= 0: no clipping. Sums in 64 bits. With nonfinite set scale is 0. */
int ckpt_optim_grad_norm(ckpt_optim *opt, double max_norm, double grad_scale, ckpt_norm_result *dev_out, void *stream);

typedef struct {
    double lr, beta1, beta2, eps;      /* eps at least 1e-30; below 1e-12 v may reach 2e31 (1 - beta2^step), else 3e38 of it */
    uint64_t step;                     /* 1, 2, ... */
    uint64_t seed;                     /* stochastic rounding */
    int32_t rounding;                  /* of 8-bit moments: CKPT_ROUND_NEAREST or CKPT_ROUND_STOCHASTIC */
    int32_t reserved;                  /* must be zero */
    const ckpt_norm_result *dev_norm;  /* NULL: gradients as they are */
} ckpt_adamw_args;

/* One AdamW step on every tensor, in f32, with g = scale * gradient:
 *   m = beta1 m + (1 - beta1) g      v = beta2 v + (1 - beta2) g^2       every operation rounded to f32, none fused
 *   master = master (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 *   param = master rounded to nearest even
 * 8-bit moments are read, updated and rounded as MXFP8 in blocks of 32 from the tensor's start; the update takes m and v before the rounding, and a v
 * that is not zero is never rounded to zero (the next step divides by its root). With beta2 near 1 a step changes v by less than half a
 * code, which rounding to nearest undoes for ever: long runs round stochastically. Element i of a tensor takes field i mod 4 of
 * mix(mix(mix(seed) + step) + 8 * (blocks of all tensors before) + i / 4) for m, field 3 - i mod 4 for v. A block with an
 * infinite or NaN moment becomes NaN as a whole: give dev_norm, and a step that would make one is left out. */
int ckpt_optim_adamw_step(ckpt_optim *opt, const ckpt_adamw_args *args, void *stream);

#ifdef __cplusplus
}
#endif
#endif
