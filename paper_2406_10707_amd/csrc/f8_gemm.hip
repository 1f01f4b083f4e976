// The product of two 8-bit matrices with a scale for each block of 128 (include/ckpt_train.h).
#include <algorithm>
#include <type_traits>

#include "f8_forms.hpp"
#include "f8_tile.hpp"

using namespace dsllm;

namespace {

struct F8Gemm {
    F8Side a, b;
    void *c;
    int64_t ldc, m, n;
    uint32_t steps, steps_a_split;
    int64_t c_split;      // elements of C from one part of K to the next
    int32_t accumulate, dtype;
};

// ------------------------------------------------------------------ tiles through LDS

// What a lane loads or stores of a row of C at once, at any element's address: sixteen bytes.
template <int OUT>
struct Run {
    static constexpr int COUNT = OUT == CKPT_F32 ? 4 : 8;
    f32x4 v[COUNT / 4];
    __device__ __forceinline__ void load(const void *at, int64_t count) {
        typedef const typename Element<OUT>::one *Pointer;
        if (count >= COUNT) {
            if constexpr (OUT == CKPT_F32) v[0] = load4<OUT>(at);
            else {
                Eight<OUT> e;
                e.load(at);
                v[0] = __builtin_convertvector(e.lo, f32x4);
                v[1] = __builtin_convertvector(e.hi, f32x4);
            }
        } else
#pragma unroll
            for (int h = 0; h < COUNT / 4; h++) v[h] = count > 4 * h ? load_upto4<OUT>((Pointer)at + 4 * h, uint32_t(count - 4 * h)) : f32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void store(void *at, int64_t count) const {
        typedef typename Element<OUT>::one *Pointer;
        if (count >= COUNT) {
            if constexpr (OUT == CKPT_F32) store4<OUT>(at, v[0]);
            else store8<OUT>(at, v[0], v[1]);
        } else
#pragma unroll
            for (int h = 0; h < COUNT / 4; h++)
                if (count > 4 * h) store_upto4<OUT>((Pointer)at + 4 * h, v[h], uint32_t(count - 4 * h));
    }
};

// A wave's sums go to C through LDS, sixteen rows at a time (fragment i: rows ar TM + i), so that a store is whole lines: a lane has 4 TNG columns of a row, neighbouring lanes other rows. Rows in LDS are 16 bytes longer than their 16 TN
// sums: sixteen lanes' writes then go to different banks.
template <class S, int OUT, bool ADD>
__device__ __forceinline__ void store_sums(const F8Gemm &p, f32x4 (&acc)[S::TM][S::TN], uint8_t *lds, int64_t row, int64_t col, int lane, int wave, int wm, int wn) {
    typedef typename Element<OUT>::one One;
    typedef Run<OUT> Piece;
    constexpr int PITCH = 64 * S::TN + 16, LANES = 16 * S::TN / Piece::COUNT, ROWS = 64 / LANES, TURNS = 16 / ROWS, BATCH = TURNS < 4 ? TURNS : 4;      // lanes for a row's 16 TN columns
    static_assert(S::NW * 16 * PITCH <= S::BYTES && LANES <= 64 && TURNS % BATCH == 0, "a wave's rows fit its part");
    const int q = lane >> 4, ar = lane & 15, piece = lane % LANES, in = lane / LANES;
    uint8_t *mine = lds + wave * 16 * PITCH;
    const int64_t c_row = row + 16 * S::TM * wm, c_col = col + 16 * S::TN * wn + Piece::COUNT * piece, left = p.n - c_col;
    One *c = static_cast<One *>(p.c) + blockIdx.y * p.c_split + c_col;
    const bool whole = row + S::BM <= p.m && col + S::BN <= p.n;
    auto store = [&](auto whole_) {
#pragma unroll
        for (int i = 0; i < S::TM; i++) {
#pragma unroll
            for (int j = 0; j < S::TN; j++) *reinterpret_cast<f32x4 *>(mine + ar * PITCH + 4 * (16 * S::TNG * (j / S::TNG) + 4 * S::TNG * q + 4 * (j % S::TNG))) = acc[i][j];
            asm volatile("" ::: "memory");      // other lanes' writes are read: a wave's go to LDS in the order of the program, which the compiler must not change
#pragma unroll
            for (int t0 = 0; t0 < TURNS; t0 += BATCH) {
                Piece old[BATCH];
#pragma unroll
                for (int t = 0; t < BATCH; t++) {
                    const int64_t r = c_row + S::TM * (ROWS * (t0 + t) + in) + i;
                    if constexpr (ADD)
                        if (whole_ || r < p.m) old[t].load(c + r * p.ldc, whole_ ? Piece::COUNT : left);
                }
#pragma unroll
                for (int t = 0; t < BATCH; t++) {
                    const int64_t r = c_row + S::TM * (ROWS * (t0 + t) + in) + i;
                    const f32x4 *at = reinterpret_cast<const f32x4 *>(mine + (ROWS * (t0 + t) + in) * PITCH + 4 * Piece::COUNT * piece);
                    Piece out;
#pragma unroll
                    for (int h = 0; h < Piece::COUNT / 4; h++) out.v[h] = ADD ? at[h] + old[t].v[h] : at[h];
                    if (whole_ || (r < p.m && left > 0)) out.store(c + r * p.ldc, whole_ ? Piece::COUNT : left);
                }
            }
            asm volatile("" ::: "memory");
        }
    };
    if (whole) store(std::true_type{});
    else store(std::false_type{});
}

template <class S, bool SQUARE, bool WIDE, int FA, int FB>
__global__ __launch_bounds__(S::THREADS, 2) void f8_gemm_kernel(F8Gemm p, TileOrder order) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::BYTES];
    const GemmTile t = gemm_tile(order);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    const int64_t row = int64_t(t.tm) * S::BM, col = int64_t(t.tn) * S::BN;
    const uint32_t first = blockIdx.y * p.steps_a_split;
    const F8Loader<S> load(p.a, p.b, p.b, p.steps, row, col, lane, wave);
    f32x4 acc[S::TM][S::TN];
    f8_sums<S, SQUARE, WIDE, FA, FB>(acc, lds, load, first, min(p.steps - first, p.steps_a_split), lane, wm, wn);
    auto out = [&](auto dtype) {
        if (p.accumulate) store_sums<S, dtype, true>(p, acc, lds, row, col, lane, wave, wm, wn);
        else store_sums<S, dtype, false>(p, acc, lds, row, col, lane, wave, wm, wn);
    };
    if (p.dtype == CKPT_F32) out(std::integral_constant<int, CKPT_F32>());
    else out(std::integral_constant<int, WIDE ? CKPT_F16 : CKPT_BF16>());
}

// ------------------------------------------------------------------ up to sixteen rows of A

template <int OUT>
__device__ __forceinline__ void store_four(void *c, f32x4 sum, uint32_t count, bool accumulate) {
    if (accumulate) sum += load_upto4<OUT>(c, count);
    store_upto4<OUT>(c, sum, count);
}
__device__ __forceinline__ void store_four(const F8Gemm &p, int64_t row, int64_t col, f32x4 sum) {
    const uint32_t count = uint32_t(min(p.n - col, int64_t(4)));
    const int64_t at = row * p.ldc + col;
    if (p.dtype == CKPT_F32) store_four<CKPT_F32>(static_cast<float *>(p.c) + at, sum, count, p.accumulate);
    else if (p.dtype == CKPT_BF16) store_four<CKPT_BF16>(static_cast<__bf16 *>(p.c) + at, sum, count, p.accumulate);
    else store_four<CKPT_F16>(static_cast<_Float16 *>(p.c) + at, sum, count, p.accumulate);
}

template <int WAVES, bool EIGHT, int FA, int FB>
__global__ __launch_bounds__(64 * WAVES) void f8_few_kernel(F8Gemm p) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[F8Few<WAVES, 1, EIGHT>::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    f32x4 sum[1];
    F8Few<WAVES, 1, EIGHT>::template sums<FA, FB>(sum, p.a, p.b, p.b, p.steps, n0, lds, lane, wave);
    const int64_t col = n0 + 4 * (lane >> 4);
    if (wave == 0 && (lane & 15) < p.m && col < p.n) store_four(p, lane & 15, col, sum[0]);
}

// The parts' sums of a product whose K was split, added in order. Rows of the parts are `pitch` elements apart, a multiple of 4.
__global__ __launch_bounds__(256) void f8_join_kernel(const float *__restrict__ parts, uint32_t splits, int64_t split, uint32_t pitch, F8Gemm p) {
    const uint64_t t = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    const uint32_t quads = pitch / 4, row = uint32_t(t / quads), col = 4 * uint32_t(t - uint64_t(row) * quads);
    if (row >= p.m) return;
    const float *at = parts + int64_t(row) * pitch + col;
    f32x4 sum = *(const f32x4 DSLLM_GLOBAL *)at;
    for (uint32_t s = 1; s < splits; s++) sum += *(const f32x4 DSLLM_GLOBAL *)(at + s * split);
    store_four(p, row, col, sum);
}

// ------------------------------------------------------------------ host

template <class F>
void with_formats(bool a_e5m2, bool b_e5m2, F f) {
    const std::integral_constant<int, 0> e4m3;
    const std::integral_constant<int, 1> e5m2;
    if (a_e5m2) b_e5m2 ? f(e5m2, e5m2) : f(e5m2, e4m3);
    else b_e5m2 ? f(e4m3, e5m2) : f(e4m3, e4m3);
}

// The product in parts of at most `rows` x `columns` of C, a launch each: one grid has fewer than 2^32 work-items.
template <class F>
void launch_in_parts(const F8Gemm &p, int64_t rows, int64_t columns, F launch) {
    const uint32_t bytes = element_bytes(p.dtype);
    for (int64_t row = 0; row < p.m; row += rows)
        for (int64_t col = 0; col < p.n; col += columns) {
            F8Gemm part = p;
            auto from = [](F8Side &side, int64_t first, int64_t most) {      // both are multiples of 128
                side.codes += first * side.pitch;
                side.scales += first >> side.shift;
                side.rows = std::min(most, side.rows - first);
            };
            from(part.a, row, rows);
            from(part.b, col, columns);
            part.c = static_cast<uint8_t *>(p.c) + (row * p.ldc + col) * bytes;
            part.m = part.a.rows;
            part.n = part.b.rows;
            launch(part);
        }
}

// False: the form has no kernel for these sums and scales, and nothing was launched.
bool launch_form(const F8Choice &choice, const F8Gemm &p, bool wide, bool a_e5m2, bool b_e5m2, hipStream_t stream) {
    if (choice.form < 0 || !f8_form_has(choice.form, wide, !p.b.shift)) return false;
    const F8Form &f = kF8Forms[choice.form];
    const int64_t tiles_each = std::max<int64_t>(1, std::min<int64_t>((p.n + f.bn - 1) / f.bn, int64_t(kF8MostTiles)));
    const int64_t columns = tiles_each * f.bn, rows = std::max<int64_t>(1, int64_t(kF8MostTiles) / tiles_each) * f.bm;
    launch_in_parts(p, (rows + 127) / 128 * 128, (columns + 127) / 128 * 128, [&](const F8Gemm &part) {
        const uint32_t tiles_m = uint32_t((part.m + f.bm - 1) / f.bm), tiles_n = uint32_t((part.n + f.bn - 1) / f.bn);
        with_formats(a_e5m2, b_e5m2, [&](auto fa, auto fb) {
            auto go = [&](auto form) {
                typedef typename F8GemmShape<form>::type S;
                static_assert(S::BM == kF8Forms[form].bm && S::BN == kF8Forms[form].bn, "the table's tile");
                const dim3 grid(tiles_m * tiles_n, choice.splits), block(S::THREADS);
                const TileOrder order(tiles_m, tiles_n, true);
                auto launch = [&](auto square, auto wide_) {
                    if constexpr (f8_form_has(form, wide_, !square)) hipLaunchKernelGGL((f8_gemm_kernel<S, square, wide_, fa, fb>), grid, block, 0, stream, part, order);
                };
                if (part.b.shift) wide ? launch(std::true_type(), std::true_type()) : launch(std::true_type(), std::false_type());
                else wide ? launch(std::false_type(), std::true_type()) : launch(std::false_type(), std::false_type());
            };
            switch (choice.form) {
                case 0: go(std::integral_constant<int, 0>()); break;
                case 1: go(std::integral_constant<int, 1>()); break;
                case 2: go(std::integral_constant<int, 2>()); break;
                default: go(std::integral_constant<int, 3>()); break;
            }
            static_assert(kF8FormCount == 4, "every form is launched");
        });
    });
    return true;
}
constexpr const char *kNoForm = "no kernel for a product of this size";

int gemm(const ckpt_f8_matrix *a, const ckpt_f8_matrix *b, void *c, int32_t dtype, int64_t ldc, int32_t accumulate, void *workspace, uint64_t workspace_bytes, hipStream_t stream) {
    if (!a || !b) return refuse(CKPT_EINVAL, "null argument");
    const uint32_t bytes = element_bytes(dtype);
    if (!bytes) return refuse(CKPT_EINVAL, "c_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    DeviceRanges ranges;
    if (const char *why = wrong_f8_matrix(a, ranges)) return refuse(CKPT_EINVAL, std::string("A: ") + why);
    if (const char *why = wrong_f8_matrix(b, ranges)) return refuse(CKPT_EINVAL, std::string("B: ") + why);
    if (a->cols != b->cols) return refuse(CKPT_EINVAL, "A and B differ in their columns");
    const int64_t m = a->rows, n = b->rows, k = a->cols;
    if (m > 0x7FFFFFFF || n > 0x7FFFFFFF) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1");
    if (const char *why = wrong_f8_contraction(a)) return refuse(CKPT_EINVAL, std::string("A: ") + why);
    if (const char *why = wrong_f8_contraction(b)) return refuse(CKPT_EINVAL, std::string("B: ") + why);
    if (m == 0 || n == 0) return CKPT_OK;
    if (ldc < n || ldc > (1ll << 48) / m) return refuse(CKPT_EINVAL, "ldc is smaller than a row, or C too large");
    if (uint64_t(c) % bytes) return refuse(CKPT_EINVAL, "C is not aligned to its element");
    if (const char *why = ranges.wrong(c, (uint64_t(m - 1) * ldc + n) * bytes)) return refuse(CKPT_EINVAL, std::string("C: ") + why);
    const Rows c_rows = plain_rows(c, m, n, ldc, bytes);
    if (overlap(*a, c_rows) || overlap(*b, c_rows)) return refuse(CKPT_EINVAL, "C: overlaps A or B");
    if (k == 0 && accumulate) return CKPT_OK;
    const uint32_t steps = f8_steps(uint64_t(k));
    F8Gemm p{f8_side(a), f8_side(b), c, ldc, m, n, steps, steps, 0, accumulate, dtype};
    const bool a_e5m2 = a->format == CKPT_F8_E5M2, b_e5m2 = b->format == CKPT_F8_E5M2, wide = dtype != CKPT_BF16;
    if (uint64_t(m) <= kF8Few) {
        const uint32_t waves = f8_few_waves(uint64_t(n), steps);
        launch_in_parts(p, 128, 16ll << 22, [&](const F8Gemm &part) {
            with_formats(a_e5m2, b_e5m2, [&](auto fa, auto fb) {
                const dim3 grid(unsigned((part.n + 15) / 16));
                auto launch = [&](auto waves_, auto eight) { hipLaunchKernelGGL((f8_few_kernel<waves_, eight, fa, fb>), grid, dim3(64 * waves_), 0, stream, part); };
                if (waves == 2) m <= 8 ? launch(std::integral_constant<int, 2>(), std::true_type()) : launch(std::integral_constant<int, 2>(), std::false_type());
                else m <= 8 ? launch(std::integral_constant<int, 4>(), std::true_type()) : launch(std::integral_constant<int, 4>(), std::false_type());
            });
        });
        return launched();
    }
    const F8Choice choice = f8_choice(uint64_t(m), uint64_t(n), uint64_t(k), wide, !p.b.shift, workspace ? workspace_bytes : 0);
    if (choice.splits == 1) return launch_form(choice, p, wide, a_e5m2, b_e5m2, stream) ? launched() : refuse(CKPT_EINVAL, kNoForm);
    if (uint64_t(workspace) % 16) return refuse(CKPT_EINVAL, "workspace must be 16-byte aligned");
    const uint64_t part_bytes = f8_part_bytes(uint64_t(m), uint64_t(n)) * choice.splits;
    if (const char *why = ranges.wrong(workspace, part_bytes)) return refuse(CKPT_EINVAL, std::string("workspace: ") + why);
    const Rows part_rows{uint64_t(workspace), part_bytes, part_bytes, 1};
    if (overlap(*a, part_rows) || overlap(*b, part_rows) || share_bytes(c_rows, part_rows)) return refuse(CKPT_EINVAL, "workspace: overlaps A, B or C");
    const uint32_t pitch = uint32_t(f8_part_pitch(uint64_t(n)));
    F8Gemm parts = p;
    parts.c = workspace;
    parts.ldc = pitch;
    parts.accumulate = 0;
    parts.dtype = CKPT_F32;
    parts.c_split = m * pitch;
    parts.steps_a_split = (steps + choice.splits - 1) / choice.splits;
    if (!launch_form(choice, parts, wide, a_e5m2, b_e5m2, stream)) return refuse(CKPT_EINVAL, kNoForm);
    const uint64_t threads = uint64_t(m) * (pitch / 4);
    hipLaunchKernelGGL(f8_join_kernel, dim3(unsigned((threads + 255) / 256)), dim3(256), 0, stream, static_cast<const float *>(workspace), choice.splits, parts.c_split, pitch, p);
    return launched();
}

}  // namespace

extern "C" {

int ckpt_f8_gemm_workspace(int64_t m, int64_t n, int64_t k, uint64_t *bytes) {
    return at_c_entry([&] {
        if (!bytes || m < 0 || n < 0 || k < 0) return refuse(CKPT_EINVAL, "null argument or negative size");
        *bytes = 0;
        if (m > 0x7FFFFFFF || n > 0x7FFFFFFF || k > kF8LongestRow) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1, or what is contracted over 2^23");
        if (!n || !k || uint64_t(m) <= kF8Few) return int(CKPT_OK);
        for (int kind = 0; kind < 4; kind++) {
            const F8Choice c = f8_choice(uint64_t(m), uint64_t(n), uint64_t(k), kind & 1, kind >> 1, UINT64_MAX);
            if (c.splits > 1) *bytes = std::max(*bytes, f8_part_bytes(uint64_t(m), uint64_t(n)) * c.splits);
        }
        return int(CKPT_OK);
    });
}

int ckpt_f8_gemm(const ckpt_f8_matrix *a, const ckpt_f8_matrix *b, void *c, int32_t c_dtype, int64_t ldc, int32_t accumulate, void *workspace, uint64_t workspace_bytes,
                 void *stream) {
    return at_c_entry([&] { return gemm(a, b, c, c_dtype, ldc, accumulate, workspace, workspace_bytes, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
