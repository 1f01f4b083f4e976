// The update phase over a list of tensors (include/ckpt_train.h): the norm of all gradients and the AdamW step, a launch each.
#include <math.h>

#include <algorithm>
#include <memory>
#include <type_traits>
#include <vector>

#include "train_util.hpp"

using namespace dsllm;

namespace {

struct TensorEntry {
    const uint8_t *grad;
    uint8_t *param;
    float *master;
    uint8_t *m, *v, *m_scale, *v_scale;
    uint64_t first_block;      // blocks of 32 of all tensors before it
    double weight_decay;
};

// What one block, or a run of them, works on: `count` elements of a tensor from element `first` on.
struct Span {
    uint32_t tensor, count;
    uint64_t first;
};
constexpr uint32_t kSpan = 4096, kNormBlocks = 1024;
constexpr uint32_t kGroups32 = 1, kGroups8 = 2;      // groups of 256 elements that a wave of the step takes

constexpr uint32_t kNormGroups = 32, kUngrouped = 64;      // blocks are counted in groups, each on a line of its own, where there are more than kUngrouped
struct NormScratch {
    uint64_t partial[kNormBlocks];      // bits of doubles
    struct { uint32_t arrived, unused[31]; } group[kNormGroups], all;
};

}  // namespace

struct ckpt_optim {
    int device = 0;
    size_t n = 0;
    uint32_t n_spans = 0;                        // of the norm: tensors cut at every kSpan elements
    uint32_t n_full = 0, n_pieces = 0;           // of the step: spans of kSpan elements, and what they leave in pieces of a wave each
    ckpt_optim_config cfg{};
    bool has_state = false;
    TensorEntry *dev_tensors = nullptr;
    Span *dev_spans = nullptr, *dev_step_spans = nullptr;
    NormScratch *dev_scratch = nullptr;
    std::vector<uint64_t> numels;
};

namespace {

// ------------------------------------------------------------------ gradient norm

__device__ __forceinline__ double sum_over_wave(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// One pass over all gradients, squares in 64 bits (no f32 gradient overflows them, and only an infinity or a NaN makes the sum one); a block's sum goes to its place in the scratch memory, the
// block that finds itself the last adds them up in order. Bound by memory: 124 M f32 gradients 70 to 72 us = 6.9 TB/s, 405 M bf16 119 us = 6.8 TB/s. Some 8 MB have to be under way: f32 with 512 blocks of 256
// (1024: 73 us, 512 of 512: 82), two bytes with 1024 of 512 (512: 160). One counter takes some 10 ns a block, one behind the other; with a counter for each of 32 groups 56 M bf16 take 20 us (one counter: 26),
// 1 M 4.4 (6.1), and blocks pay from four spans each on (16 M bf16 8.4 us, with one for every sixteen 13.3).
inline uint32_t norm_blocks(uint32_t n_spans, uint32_t most) {
    const uint32_t wanted = n_spans / 4 < 256 ? 256 : n_spans / 4 > most ? most : n_spans / 4;
    return n_spans < 1 ? 1 : n_spans < wanted ? n_spans : wanted;
}

template <int N>
__device__ __forceinline__ double sum_of_parts(const double (&part)[N]) {
    double s = part[0];
#pragma unroll
    for (int i = 1; i < N; i++) s += part[i];
    return s;
}

// 4 PIECE elements in accesses of 16 bytes, at any element's address
template <int GRAD, uint32_t PIECE>
__device__ __forceinline__ void load_piece(f32x4 *v, const uint8_t *p) {
    if constexpr (PIECE == 1) v[0] = load4<GRAD>(p);
    else {
        Eight<GRAD> e;
        e.load(p);
        v[0] = __builtin_convertvector(e.lo, f32x4);
        v[1] = __builtin_convertvector(e.hi, f32x4);
    }
}

template <int GRAD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(const TensorEntry *__restrict__ tensors, const Span *__restrict__ spans, uint32_t n_spans,
                                                  NormScratch *scratch, ckpt_norm_result *out, double max_norm, double grad_scale) {
    __shared__ double part[THREADS / 64];
    __shared__ bool last;
    constexpr uint32_t kPiece = GRAD == CKPT_F32 ? 1 : 2, kPasses = kSpan / (4 * THREADS), kBytes = sizeof(typename Element<GRAD>::one);
    double sum = 0;
    auto add = [&](f32x4 v) {
#pragma unroll
        for (int j = 0; j < 4; j++) sum += double(v[j]) * double(v[j]);
    };
    for (uint32_t s = blockIdx.x; s < n_spans; s += gridDim.x) {
        const Span span = spans[s];
        const uint8_t *g = tensors[span.tensor].grad + span.first * kBytes;
        if (span.count == kSpan) {
            f32x4 v[kPasses];
#pragma unroll
            for (uint32_t k = 0; k < kPasses; k += kPiece) load_piece<GRAD, kPiece>(&v[k], g + (4 * kPiece * (threadIdx.x + THREADS * (k / kPiece))) * kBytes);
#pragma unroll
            for (uint32_t k = 0; k < kPasses; k++) add(v[k]);
        } else {
            for (uint32_t i = 4 * threadIdx.x; i < span.count; i += 4 * THREADS) add(load_upto4<GRAD>(g + i * kBytes, span.count - i));
        }
    }
    sum = sum_over_wave(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        // The partial sum is at the place where all compute units see it once the exchange has returned, and only then is the block counted: the order comes from waiting for the
        // value, not from a release (which writes the whole L2 back: 36 ns a block, one behind the other).
        const uint64_t before = __hip_atomic_exchange(&scratch->partial[blockIdx.x], uint64_t(__double_as_longlong(sum_of_parts(part))), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::"v"(before) : "memory");
        uint32_t wanted = gridDim.x;
        bool counts = true;      // the last of a group stands for all of it
        if (gridDim.x > kUngrouped) {
            const uint32_t g = blockIdx.x % kNormGroups, members = (gridDim.x - g + kNormGroups - 1) / kNormGroups;
            counts = __hip_atomic_fetch_add(&scratch->group[g].arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1;
            wanted = kNormGroups;
        }
        last = counts && __hip_atomic_fetch_add(&scratch->all.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == wanted - 1;
    }
    __syncthreads();
    if (!last) return;
    if (threadIdx.x < kNormGroups) __hip_atomic_store(&scratch->group[threadIdx.x].arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = 0;
    for (uint32_t b = threadIdx.x; b < gridDim.x; b += THREADS) sum += __longlong_as_double(int64_t(__hip_atomic_load(&scratch->partial[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
    sum = sum_over_wave(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = sum_of_parts(part);
    __hip_atomic_store(&scratch->all.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // An infinity or a NaN makes the sum one (and fails every comparison). A step squares scale * gradient in f32, which holds 2^64 squared no more; up to 2^63 a second moment has room for
    // being rounded up in 8 bits.
    const double norm = grad_scale * sqrt(sum);
    const bool clipped = max_norm > 0 && norm > max_norm, usable = norm <= double(__FLT_MAX__) && (clipped ? max_norm : norm) <= 0x1p63;
    out->sum_squares = sum;
    out->norm = float(norm);
    out->scale = !usable ? 0.0f : clipped ? float(grad_scale * (max_norm / norm)) : float(grad_scale);
    out->nonfinite = usable ? 0 : 1;
    out->reserved = 0;
}

// ------------------------------------------------------------------ AdamW step

struct StepArgs {
    float beta1, one_less_beta1, beta2, one_less_beta2, eps, lr, inv_bc1, inv_bc2, root_back;
    double lr64;
    uint64_t key;
    const ckpt_norm_result *norm;
};

// Four elements: the moments in f32, each operation rounded by itself, so that the 8-bit moments do not depend on what a compiler fuses.
__device__ __forceinline__ void update_moments(f32x4 g, f32x4 &m, f32x4 &v, const StepArgs &a) {
#pragma clang fp contract(off)
    m = m * a.beta1 + g * a.one_less_beta1;
    v = v * a.beta2 + (g * g) * a.one_less_beta2;
}
// The root and the quotient by the approximate instructions (1 ulp each): the error is 1e-7 of the update, which is some 1e-4 of the weight. The root's takes subnormal numbers as zero, which is up to 1.1e-19
// of the root: beside a smaller eps than kSmallEps inv_bc2 comes multiplied by 2^24, and root_back divides by 2^12 (else 1; in the addition's own instruction either way).
constexpr double kSmallEps = 1e-12;
__device__ __forceinline__ f32x4 updated(f32x4 w, f32x4 m, f32x4 v, float keep, const StepArgs &a) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float root = __builtin_fmaf(__builtin_amdgcn_sqrtf(v[j] * a.inv_bc2), a.root_back, a.eps);
        w[j] = w[j] * keep - a.lr * (m[j] * a.inv_bc1 * __builtin_amdgcn_rcpf(root));
    }
    return w;
}

// Bound by memory: 32-bit moments move 28 or 30 bytes an element, 8-bit ones 16.1 with gradients in 16 bits. Blocks of one wave in address order keep the chip in a narrow front of each of the seven to
// nine streams, and shared memory that nothing uses keeps the front narrower still where the grid is larger than the chip: 124 M elements with f32 gradients 609 us, with room for twelve waves to a
// compute unit 570 = 6.5 TB/s, for seven 596 (two groups a lane: 620, 604, 592; blocks of four waves that loop over a span 665). 8-bit moments need more waves, or more a lane: 405 M
// elements 1057 us with one group, with two 1084 and, with room for twenty waves, 1055 (twelve waves: 1760 and 1171). Stochastic rounding fills the vector units as well (98 % of their cycles with 80 instructions
// an element, 94 % now): without the sign of v and with the least code by two integer instructions 1040 us, with spans that every block finds work in 1009 on the same card; other cards 1045 to 1063 = 6.1
// to 6.2 TB/s, to nearest 1051. Tensors without gaps have lines that two blocks write: 78 M elements with 8-bit moments 291 us, each at a multiple of 32 elements 229.
constexpr unsigned kFreeBlocks = 256 * 36;
constexpr uint32_t kSpansALaunch = 1u << 21;      // a grid has fewer than 2^32 work-items
// A wave a block, GROUPS groups of four elements a lane, 256 elements apart: kSpan / (256 GROUPS) blocks for each of n_full spans, one for each of the pieces behind them (blocks that find nothing to do
// cost 1 ns each: 4000 tensors of some 250 elements took 64 us with sixteen for each, 10 so). Every block of 32 elements lies in eight neighbouring lanes.
// PARAM 0: no working copy. BITS: of the moments.
template <int GRAD, int PARAM, int BITS, bool STOCHASTIC, int GROUPS>
__global__ __launch_bounds__(64) void adamw_kernel(const TensorEntry *__restrict__ tensors, const Span *__restrict__ full, uint32_t n_full, const Span *__restrict__ pieces, StepArgs a) {
    constexpr uint32_t kWave = 256 * GROUPS, kBlocks = kSpan / kWave;
    const bool piece = blockIdx.x >= n_full * kBlocks;
    const Span span = *(piece ? pieces + (blockIdx.x - n_full * kBlocks) : full + blockIdx.x / kBlocks);
    const uint32_t start = piece ? 0 : blockIdx.x % kBlocks * kWave;
    const TensorEntry &t = tensors[span.tensor];
    float scale = 1.0f;
    if (a.norm) {
        if (a.norm->nonfinite) return;
        scale = a.norm->scale;
    }
    const float keep = float(1.0 - a.lr64 * t.weight_decay);
    const uint64_t e0 = span.first + start;
    const uint32_t left = span.count - start;
    auto work = [&](auto whole) {
        f32x4 g[GROUPS], w[GROUPS], m[GROUPS], v[GROUPS];
        uint32_t mc[GROUPS], vc[GROUPS], mb[GROUPS], vb[GROUPS], count[GROUPS];
#pragma unroll
        for (int k = 0; k < GROUPS; k++) {
            const uint32_t i = 256 * k + 4 * threadIdx.x;
            const uint64_t e = e0 + i;
            count[k] = whole ? 4 : i < left ? left - i : 0;
            g[k] = load_upto4<GRAD>(t.grad + e * sizeof(typename Element<GRAD>::one), count[k]);
            w[k] = load_upto4<CKPT_F32>(t.master + e, count[k]);
            if constexpr (BITS == 32) {
                m[k] = load_upto4<CKPT_F32>(t.m + 4 * e, count[k]);
                v[k] = load_upto4<CKPT_F32>(t.v + 4 * e, count[k]);
            } else {
                mc[k] = load_bytes(t.m + e, count[k]);
                vc[k] = load_bytes(t.v + e, count[k]);
                mb[k] = i < left ? ((const uint8_t DSLLM_GLOBAL *)t.m_scale)[e / 32] : 0;
                vb[k] = i < left ? ((const uint8_t DSLLM_GLOBAL *)t.v_scale)[e / 32] : 0;
            }
        }
#pragma unroll
        for (int k = 0; k < GROUPS; k++) {
            const uint32_t i = 256 * k + 4 * threadIdx.x;
            const uint64_t e = e0 + i;
            if constexpr (BITS == 8) {
                m[k] = fp8_values(mc[k]) * scale_value(mb[k]);
                v[k] = fp8_values(vc[k]) * scale_value(vb[k]);
            }
            update_moments(g[k] * scale, m[k], v[k], a);
            if constexpr (BITS == 32) {
                store_upto4<CKPT_F32>(t.m + 4 * e, m[k], count[k]);
                store_upto4<CKPT_F32>(t.v + 4 * e, v[k], count[k]);
            } else {
                const uint32_t mb = scale_byte<CKPT_MXFP8>(most_of_8(magnitude_bits(m[k]))), vb = scale_byte<CKPT_MXFP8>(most_of_8(magnitude_bits(v[k])));
                const f32x4 ym = m[k] * inverse_scale(mb), yv = v[k] * inverse_scale(vb);
                uint32_t mc, vc;
                if constexpr (STOCHASTIC) {
                    const uint64_t r = mix64(a.key + 8 * t.first_block + e / 4);
                    const uint32_t r_lo = uint32_t(r), r_hi = uint32_t(r >> 32);
                    const uint64_t backwards = uint64_t(__builtin_amdgcn_alignbit(r_lo, r_lo, 16)) << 32 | __builtin_amdgcn_alignbit(r_hi, r_hi, 16);      // the four fields, last first
                    mc = fp8_stochastic<false>(ym, m[k], r);
                    vc = fp8_stochastic<true, false>(yv, v[k], backwards);      // squares: never negative
                } else {
                    mc = fp8_nearest<false>(ym, m[k]);
                    vc = fp8_nearest<true>(yv, v[k]);
                }
                store_bytes(t.m + e, mc, count[k]);
                store_bytes(t.v + e, vc, count[k]);
                if ((threadIdx.x & 7) == 0 && (whole || i < left)) {
                    ((uint8_t DSLLM_GLOBAL *)t.m_scale)[e / 32] = uint8_t(mb);
                    ((uint8_t DSLLM_GLOBAL *)t.v_scale)[e / 32] = uint8_t(vb);
                }
            }
            const f32x4 next = updated(w[k], m[k], v[k], keep, a);
            store_upto4<CKPT_F32>(t.master + e, next, count[k]);
            if constexpr (PARAM != 0) store_upto4<PARAM>(t.param + 2 * e, next, count[k]);
        }
    };
    if (left >= kWave) work(std::true_type{});
    else work(std::false_type{});
}

constexpr uint32_t kGradsALaunch = 448;
struct GradList { const uint8_t *grad[kGradsALaunch]; };
__global__ __launch_bounds__(kGradsALaunch) void set_grads_kernel(TensorEntry *tensors, uint32_t count, GradList list) {
    if (threadIdx.x < count) tensors[threadIdx.x].grad = list.grad[threadIdx.x];
}

template <int GRAD, int PARAM>
void launch_adamw(const ckpt_optim *o, const StepArgs &a, bool stochastic, hipStream_t stream) {
    auto go = [&](auto kernel, unsigned groups, unsigned lds) {
        for (uint32_t first = 0;; first += kSpansALaunch) {
            const uint32_t here = std::min(o->n_full - first, kSpansALaunch);
            const bool last = first + here == o->n_full;
            const unsigned blocks = here * (kSpan / 256 / groups) + (last ? o->n_pieces : 0);
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64), blocks > kFreeBlocks ? lds : 0, stream, o->dev_tensors, o->dev_step_spans + first, here, o->dev_step_spans + o->n_full, a);
            if (last) break;
        }
    };
    if (o->cfg.state_bits == 32) go(adamw_kernel<GRAD, PARAM, 32, false, kGroups32>, kGroups32, 12800);
    else if (stochastic) go(adamw_kernel<GRAD, PARAM, 8, true, kGroups8>, kGroups8, 8192);
    else go(adamw_kernel<GRAD, PARAM, 8, false, kGroups8>, kGroups8, 8192);
}
template <int GRAD>
void launch_adamw(const ckpt_optim *o, const StepArgs &a, bool stochastic, hipStream_t stream) {
    switch (o->cfg.param_dtype) {
        case CKPT_BF16: return launch_adamw<GRAD, CKPT_BF16>(o, a, stochastic, stream);
        case CKPT_F16: return launch_adamw<GRAD, CKPT_F16>(o, a, stochastic, stream);
        default: return launch_adamw<GRAD, 0>(o, a, stochastic, stream);
    }
}

int wrong_device(const ckpt_optim *o) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); return refuse(CKPT_EHIP, "no current device"); }
    return dev == o->device ? CKPT_OK : refuse(CKPT_EINVAL, "the optimizer belongs to another device than the current one");
}

int create(const ckpt_optim_tensor *tensors, size_t n, const ckpt_optim_config *cfg, ckpt_optim **out) {
    if (!out) return refuse(CKPT_EINVAL, "null argument");
    *out = nullptr;
    if (!tensors || !cfg || n == 0 || n > 0xFFFFFFFFu) return refuse(CKPT_EINVAL, "null argument or empty tensor list");
    const uint32_t grad_bytes = element_bytes(cfg->grad_dtype);
    if (!grad_bytes) return refuse(CKPT_EINVAL, "grad_dtype must be CKPT_F32, CKPT_BF16 or CKPT_F16");
    if (cfg->param_dtype != 0 && cfg->param_dtype != CKPT_BF16 && cfg->param_dtype != CKPT_F16) return refuse(CKPT_EINVAL, "param_dtype must be CKPT_BF16, CKPT_F16 or 0");
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return refuse(CKPT_EINVAL, "state_bits must be 32 or 8");
    if (cfg->reserved) return refuse(CKPT_EINVAL, "reserved field not zero");
    std::unique_ptr<ckpt_optim> o(new ckpt_optim);
    o->cfg = *cfg;
    o->n = n;
    std::vector<TensorEntry> entries(n);
    std::vector<Span> spans, full, pieces;
    const uint32_t wave = 256 * (cfg->state_bits == 32 ? kGroups32 : kGroups8);
    DeviceRanges ranges;
    uint64_t blocks = 0, n_spans = 0;
    bool any = false;
    for (size_t k = 0; k < n; k++) {
        const ckpt_optim_tensor &t = tensors[k];
        auto bad = [&](const char *part, const char *why) { return refuse(CKPT_EINVAL, "tensor " + std::to_string(k) + ": " + part + ": " + why); };
        if (t.numel > 1ull << 48) return bad("numel", "too large");
        const bool state = t.dev_master != nullptr;
        if (t.numel) {
            if (any && state != o->has_state) return bad("dev_master", "given for some tensors only");
            any = true;
            o->has_state = state;
            struct { const char *name; const void *p; uint64_t bytes, align; } parts[] = {
                {"dev_grad", t.dev_grad, t.numel * grad_bytes, grad_bytes},
                {"dev_master", t.dev_master, state ? 4 * t.numel : 0, 4},
                {"dev_param", t.dev_param, state && cfg->param_dtype ? 2 * t.numel : 0, 2},
                {"dev_m", t.dev_m, !state ? 0 : cfg->state_bits == 32 ? 4 * t.numel : t.numel, cfg->state_bits == 32 ? 4u : 1u},
                {"dev_v", t.dev_v, !state ? 0 : cfg->state_bits == 32 ? 4 * t.numel : t.numel, cfg->state_bits == 32 ? 4u : 1u},
                {"dev_m_scale", t.dev_m_scale, state && cfg->state_bits == 8 ? (t.numel + 31) / 32 : 0, 1},
                {"dev_v_scale", t.dev_v_scale, state && cfg->state_bits == 8 ? (t.numel + 31) / 32 : 0, 1},
            };
            for (const auto &part : parts) {
                if (!part.bytes) continue;
                if (const char *why = ranges.wrong(part.p, part.bytes)) return bad(part.name, why);
                if (uint64_t(part.p) % part.align) return bad(part.name, "not aligned to its element");
            }
        }
        if (!(fabs(t.weight_decay) <= 1e30)) return bad("weight_decay", "not a finite number");
        entries[k] = TensorEntry{static_cast<const uint8_t *>(t.dev_grad), static_cast<uint8_t *>(t.dev_param), t.dev_master, static_cast<uint8_t *>(t.dev_m),
                                 static_cast<uint8_t *>(t.dev_v), static_cast<uint8_t *>(t.dev_m_scale), static_cast<uint8_t *>(t.dev_v_scale), blocks, t.weight_decay};
        o->numels.push_back(t.numel);
        blocks += (t.numel + 31) / 32;
        n_spans += (t.numel + kSpan - 1) / kSpan;
        if (n_spans > 1u << 24) return refuse(CKPT_EINVAL, "more than 2^36 elements");
        if (state && t.numel) {
            // 32-bit moments: the spans begin where the master weights begin a line, so that the waves' stores are whole lines (the moments' too, where all lie at the same distance from one, as in
            // flattened buffers: 85 M elements at any element's address 502 us, so 372). 8-bit ones begin with a block of 32.
            uint64_t at = 0;
            const uint64_t head = cfg->state_bits == 32 ? (128 - uint64_t(t.dev_master) % 128) % 128 / 4 : 0;
            auto piece = [&](uint64_t count) {
                pieces.push_back(Span{uint32_t(k), uint32_t(count), at});
                at += count;
            };
            if (head && t.numel >= kSpan) piece(head);
            for (; t.numel - at >= kSpan; at += kSpan) full.push_back(Span{uint32_t(k), kSpan, at});
            while (at < t.numel) piece(std::min(t.numel - at, uint64_t(wave)));
        }
        if (pieces.size() > 1u << 24) return refuse(CKPT_EINVAL, "too many tensors");
        for (uint64_t first = 0; first < t.numel; first += kSpan) spans.push_back(Span{uint32_t(k), uint32_t(t.numel - first < kSpan ? t.numel - first : kSpan), first});
    }
    o->n_spans = uint32_t(spans.size());
    o->n_full = uint32_t(full.size());
    o->n_pieces = uint32_t(pieces.size());
    full.insert(full.end(), pieces.begin(), pieces.end());
    auto failed = [&](hipError_t e) {
        (void)hipFree(o->dev_tensors); (void)hipFree(o->dev_spans); (void)hipFree(o->dev_step_spans); (void)hipFree(o->dev_scratch);
        (void)hipGetLastError();
        return refuse(e == hipErrorOutOfMemory ? CKPT_ENOMEM : CKPT_EHIP, std::string("optimizer set-up: ") + hipGetErrorString(e));
    };
    hipError_t e = hipGetDevice(&o->device);
    if (e == hipSuccess) e = hipMalloc(&o->dev_tensors, n * sizeof(TensorEntry));
    if (e == hipSuccess) e = hipMalloc(&o->dev_spans, (spans.size() + 1) * sizeof(Span));
    if (e == hipSuccess) e = hipMalloc(&o->dev_step_spans, (full.size() + 1) * sizeof(Span));
    if (e == hipSuccess) e = hipMalloc(&o->dev_scratch, sizeof(NormScratch));
    if (e == hipSuccess) e = hipMemcpy(o->dev_tensors, entries.data(), n * sizeof(TensorEntry), hipMemcpyHostToDevice);
    if (e == hipSuccess && !spans.empty()) e = hipMemcpy(o->dev_spans, spans.data(), spans.size() * sizeof(Span), hipMemcpyHostToDevice);
    if (e == hipSuccess && !full.empty()) e = hipMemcpy(o->dev_step_spans, full.data(), full.size() * sizeof(Span), hipMemcpyHostToDevice);
    const NormScratch zero{};
    if (e == hipSuccess) e = hipMemcpy(o->dev_scratch, &zero, sizeof zero, hipMemcpyHostToDevice);
    if (e != hipSuccess) return failed(e);
    *out = o.release();
    return CKPT_OK;
}

}  // namespace

extern "C" {

int ckpt_optim_create(const ckpt_optim_tensor *tensors, size_t n, const ckpt_optim_config *cfg, ckpt_optim **out) {
    return at_c_entry([&] { return create(tensors, n, cfg, out); });
}

int ckpt_optim_destroy(ckpt_optim *o) {
    return at_c_entry([&] {
        if (!o) return refuse(CKPT_EINVAL, "null argument");
        int current = o->device;      // the caller's may be another device than the one whose work is to be waited for
        (void)hipGetDevice(&current);
        hipError_t e = current == o->device ? hipSuccess : hipSetDevice(o->device);
        if (e == hipSuccess) e = hipDeviceSynchronize();
        (void)hipFree(o->dev_tensors);
        (void)hipFree(o->dev_spans);
        (void)hipFree(o->dev_step_spans);
        (void)hipFree(o->dev_scratch);
        if (current != o->device) (void)hipSetDevice(current);
        delete o;
        return e == hipSuccess ? CKPT_OK : refuse(CKPT_EHIP, hipGetErrorString(e));
    });
}

int ckpt_optim_set_grads(ckpt_optim *o, const void *const *dev_grads, size_t n, void *stream) {
    return at_c_entry([&] {
        if (!o || !dev_grads) return refuse(CKPT_EINVAL, "null argument");
        if (n != o->n) return refuse(CKPT_EINVAL, "the optimizer has " + std::to_string(o->n) + " tensors");
        if (int r = wrong_device(o)) return r;
        const uint32_t bytes = element_bytes(o->cfg.grad_dtype);
        DeviceRanges ranges;
        for (size_t k = 0; k < n; k++) {
            if (!o->numels[k]) continue;
            if (const char *why = ranges.wrong(dev_grads[k], o->numels[k] * bytes)) return refuse(CKPT_EINVAL, "tensor " + std::to_string(k) + ": " + why);
            if (uint64_t(dev_grads[k]) % bytes) return refuse(CKPT_EINVAL, "tensor " + std::to_string(k) + ": not aligned to its element");
        }
        GradList list;
        for (size_t first = 0; first < n; first += kGradsALaunch) {
            const uint32_t count = uint32_t(n - first < kGradsALaunch ? n - first : kGradsALaunch);
            for (uint32_t k = 0; k < count; k++) list.grad[k] = static_cast<const uint8_t *>(dev_grads[first + k]);
            hipLaunchKernelGGL(set_grads_kernel, dim3(1), dim3(kGradsALaunch), 0, static_cast<hipStream_t>(stream), o->dev_tensors + first, count, list);
        }
        return launched();
    });
}

int ckpt_optim_grad_norm(ckpt_optim *o, double max_norm, double grad_scale, ckpt_norm_result *dev_out, void *hip_stream) {
    return at_c_entry([&] {
        if (!o) return refuse(CKPT_EINVAL, "null argument");
        if (!(max_norm == max_norm) || !(grad_scale >= 0 && grad_scale <= 1e30)) return refuse(CKPT_EINVAL, "max_norm is not a number, or grad_scale negative or not one");
        if (int r = wrong_device(o)) return r;
        DeviceRanges ranges;
        if (const char *why = ranges.wrong(dev_out, sizeof *dev_out)) return refuse(CKPT_EINVAL, std::string("dev_out: ") + why);
        if (uint64_t(dev_out) % 8) return refuse(CKPT_EINVAL, "dev_out must be 8-byte aligned");
        auto go = [&](auto kernel, uint32_t threads, uint32_t most) {
            hipLaunchKernelGGL(kernel, dim3(norm_blocks(o->n_spans, most)), dim3(threads), 0, static_cast<hipStream_t>(hip_stream), o->dev_tensors, o->dev_spans, o->n_spans, o->dev_scratch, dev_out, max_norm, grad_scale);
        };
        switch (o->cfg.grad_dtype) {
            case CKPT_F32: go(norm_kernel<CKPT_F32, 256>, 256, 512); break;
            case CKPT_BF16: go(norm_kernel<CKPT_BF16, 512>, 512, 1024); break;
            default: go(norm_kernel<CKPT_F16, 512>, 512, 1024);
        }
        return launched();
    });
}

int ckpt_optim_adamw_step(ckpt_optim *o, const ckpt_adamw_args *p, void *hip_stream) {
    return at_c_entry([&] {
        if (!o || !p) return refuse(CKPT_EINVAL, "null argument");
        if (!o->has_state && o->n_spans) return refuse(CKPT_ESTATE, "the optimizer was created with gradients only");
        if (!(p->beta1 >= 0 && p->beta1 < 1 && p->beta2 >= 0 && p->beta2 < 1)) return refuse(CKPT_EINVAL, "beta1 and beta2 lie in [0, 1)");
        if (!(p->eps >= 1e-30 && p->eps <= 1e30) || !(fabs(p->lr) <= 1e30)) return refuse(CKPT_EINVAL, "eps must be at least 1e-30, lr a finite number");
        if (p->step == 0) return refuse(CKPT_EINVAL, "steps are counted from 1");
        if (p->rounding != CKPT_ROUND_NEAREST && p->rounding != CKPT_ROUND_STOCHASTIC) return refuse(CKPT_EINVAL, "rounding must be CKPT_ROUND_NEAREST or CKPT_ROUND_STOCHASTIC");
        if (p->reserved) return refuse(CKPT_EINVAL, "reserved field not zero");
        if (int r = wrong_device(o)) return r;
        DeviceRanges ranges;
        if (p->dev_norm) {
            if (const char *why = ranges.wrong(p->dev_norm, sizeof *p->dev_norm)) return refuse(CKPT_EINVAL, std::string("dev_norm: ") + why);
            if (uint64_t(p->dev_norm) % 8) return refuse(CKPT_EINVAL, "dev_norm must be 8-byte aligned");
        }
        if (!o->n_spans) return int(CKPT_OK);
        StepArgs a;
        a.beta1 = float(p->beta1);
        a.one_less_beta1 = float(1.0 - p->beta1);
        a.beta2 = float(p->beta2);
        a.one_less_beta2 = float(1.0 - p->beta2);
        a.eps = float(p->eps);
        a.lr = float(p->lr);
        a.lr64 = p->lr;
        a.inv_bc1 = float(1.0 / (1.0 - pow(p->beta1, double(p->step))));
        a.inv_bc2 = float((p->eps < kSmallEps ? 0x1p24 : 1.0) / (1.0 - pow(p->beta2, double(p->step))));
        a.root_back = p->eps < kSmallEps ? 0x1p-12f : 1.0f;
        a.key = mix64(mix64(p->seed) + p->step);
        a.norm = p->dev_norm;
        const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        const bool stochastic = p->rounding == CKPT_ROUND_STOCHASTIC;
        switch (o->cfg.grad_dtype) {
            case CKPT_F32: launch_adamw<CKPT_F32>(o, a, stochastic, stream); break;
            case CKPT_BF16: launch_adamw<CKPT_BF16>(o, a, stochastic, stream); break;
            default: launch_adamw<CKPT_F16>(o, a, stochastic, stream);
        }
        return launched();
    });
}

}  // extern "C"
