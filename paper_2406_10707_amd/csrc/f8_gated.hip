// The gated feed-forward block in 8 bits with a scale for each block of 128, forward and backward (include/ckpt_train.h).
#include <algorithm>
#include <type_traits>

#include "f8_forms.hpp"
#include "f8_rows.hpp"
#include "f8_tile.hpp"

using namespace dsllm;

namespace {

// ------------------------------------------------------------------ activations

// act(g) = g s with s = 1 / (1 + exp(-z)): z is g for SiLU, 2 sqrt(2 / pi) (g + 0.044715 g^3) for GELU (its tanh(x) is 2 / (1 + exp(-2 x)) - 1).
constexpr float kGelu = 1.5957691216057308f, kCubic = 0.044715f;
template <int ACT>
__device__ __forceinline__ float sigmoid_of(float g) {
    const float z = ACT == CKPT_GATE_SILU ? g : kGelu * g * __builtin_fmaf(kCubic * g, g, 1.0f);
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}
// act'(g) = s + act(g) (1 - s) dz/dg. 1 - s is off by up to 2^-23 where s nears 1; act(g) dz/dg is below 40 there (for larger g, s is 1 and the second term below 2^-18 left out): 5e-6 of the slope, where a code's half step is 2^-4. Where act(g) (1 - s) is zero dz/dg may be infinite.
template <int ACT>
__device__ __forceinline__ float slope_of(float g, float s, float act) {
    if constexpr (ACT == CKPT_GATE_SILU) return __builtin_fmaf(act, 1.0f - s, s);
    else {
        const float t = act * (1.0f - s);
        return t == 0 ? s : __builtin_fmaf(t, kGelu * __builtin_fmaf(3 * kCubic * g, g, 1.0f), s);
    }
}

// Which bytes of a word of four codes stay where `left` columns are left.
__device__ __forceinline__ uint32_t bytes_kept(int64_t left) { return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1; }

// ------------------------------------------------------------------ forward

struct GatedForward {
    F8Side x, w_gate, w_up;
    F8Held gate, up, h;      // gate, up: both or none
    int64_t tokens, ffn;
    uint32_t steps;
};

// A tile's columns are 128 of gate and the same 128 of up, in turn groups of 16 TNG, so that a lane has both factors of its elements. The rows' largest values of 128 columns are found among the lanes of a row (q), then
// through LDS among the WN waves. 4096 tokens, 4096 to 11008, all three matrices kept, 569 to 625 us from card to card in a row of calls (1.2 to 1.3 PFLOP/s; a trace's first ones up to 690): the sums (f8_tile.hpp), and some 30 us of rounds' ends.
template <class S, int ACT, bool SQUARE, int FA>
__device__ __forceinline__ void gated_forward_tile(const GatedForward &p, uint8_t *lds, int64_t row, int64_t col) {
    static_assert(S::PAIR && S::BN == 256, "a tile has a block of each");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, ar = lane & 15;
    const F8Loader<S> load(p.x, p.w_gate, p.w_up, p.steps, row, col, lane, wave);
    f32x4 acc[S::TM][S::TN];
    f8_sums<S, SQUARE, true, FA, 0>(acc, lds, load, 0, p.steps, lane, wm, wn);
    const bool keep = p.gate.codes;
    const int64_t my_col = col + 16 * S::TNG * wn + 4 * S::TNG * q, my_row = row + 16 * S::TM * wm + S::TM * ar;
    // columns behind the last are the last again, and change no largest value; their codes are zero (NaN times zero would be none)
    uint32_t kept[S::TNG];
#pragma unroll
    for (int j = 0; j < S::TNG; j++) kept[j] = bytes_kept(p.ffn - my_col - 4 * j);
    f32x4 h[S::TM][S::TNG];
    uint32_t *most = reinterpret_cast<uint32_t *>(lds);      // [3][BM][WN]
#pragma unroll
    for (int i = 0; i < S::TM; i++) {
        float most_h = 0, most_gate = 0, most_up = 0;
#pragma unroll
        for (int j = 0; j < S::TNG; j++) {
            const f32x4 g = acc[i][j], u = acc[i][S::TNG + j];
#pragma unroll
            for (int e = 0; e < 4; e++) h[i][j][e] = g[e] * sigmoid_of<ACT>(g[e]) * u[e];
            most_h = larger(most_h, h[i][j]);
            most_gate = larger(most_gate, g);
            most_up = larger(most_up, u);
        }
        const uint32_t of_h = most_of_quarters(bits_of(most_h)), of_gate = most_of_quarters(bits_of(most_gate)), of_up = most_of_quarters(bits_of(most_up));
        uint32_t *at = most + (16 * S::TM * wm + S::TM * ar + i) * S::WN + wn;
        if (q == 0) {
            at[0] = of_h;
            at[S::BM * S::WN] = of_gate;
            at[2 * S::BM * S::WN] = of_up;
        }
    }
    __syncthreads();
    // every row's scale once: a division is some twenty instructions
    float *inverses = reinterpret_cast<float *>(lds) + 3 * S::BM * S::WN;      // [3][BM]
    const int matrices = keep ? 3 : 1;
    for (int k = threadIdx.x; k < matrices * S::BM; k += S::THREADS) {
        uint32_t amax = 0;
#pragma unroll
        for (int w = 0; w < S::WN; w++) amax = max(amax, most[k * S::WN + w]);
        inverses[k] = f8_inverse(amax, f8_most(false));
        const F8Held &to = k < S::BM ? p.h : k < 2 * S::BM ? p.gate : p.up;
        const int64_t r = row + k % S::BM;
        if (r < p.tokens) ((float DSLLM_GLOBAL *)to.scales)[(col / 128) * to.scale_pitch + r] = f8_scale(amax, f8_most(false));
    }
    __syncthreads();
    auto out = [&](const F8Held &to, int which, auto value) {
#pragma unroll
        for (int i = 0; i < S::TM; i++) {
            const float inverse = inverses[which * S::BM + 16 * S::TM * wm + S::TM * ar + i];
            uint32_t codes[S::TNG];
#pragma unroll
            for (int j = 0; j < S::TNG; j++) codes[j] = f8_codes(value(i, j) * inverse, false) & kept[j];
            if (my_row + i < p.tokens) {
                uint8_t *at = to.codes + (my_row + i) * to.code_pitch + my_col;
                if constexpr (S::TNG == 4) *(u32x4 DSLLM_GLOBAL *)at = u32x4{codes[0], codes[1], codes[2], codes[3]};
                else *(u32x2 DSLLM_GLOBAL *)at = u32x2{codes[0], codes[1]};
            }
        }
    };
    out(p.h, 0, [&](int i, int j) { return h[i][j]; });
    if (!keep) return;
    out(p.gate, 1, [&](int i, int j) { return acc[i][j]; });
    out(p.up, 2, [&](int i, int j) { return acc[i][S::TNG + j]; });
}

template <class S, int ACT, bool SQUARE, int FA>
__global__ __launch_bounds__(S::THREADS, 2) void gated_forward_kernel(GatedForward p, TileOrder order) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::BYTES];
    const GemmTile t = gemm_tile(order);
    gated_forward_tile<S, ACT, SQUARE, FA>(p, lds, int64_t(t.tm) * S::BM, int64_t(t.tn) * 128);
}

// Tiles of 256 tokens up to the `whole`th block; behind them each two blocks take the halves of one, where the last round of blocks would leave half of the chip idle: 4096 tokens, 4096 to 11008, 5.4 rounds, 601 -> 569 us; 1024 tokens 204 -> 163.
template <int ACT, bool SQUARE, int FA>
__global__ __launch_bounds__(512, 2) void gated_forward_halves_kernel(GatedForward p, TileOrder order, uint32_t whole) {
    typedef F8GatedShape<0>::type S;
    typedef F8GatedShape<1>::type Half;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::BYTES];
    const uint32_t rest = (gridDim.x - whole) / 2, second = blockIdx.x >= whole + rest;
    const GemmTile t = gemm_tile(order, second ? blockIdx.x - rest : blockIdx.x);
    if (blockIdx.x < whole) gated_forward_tile<S, ACT, SQUARE, FA>(p, lds, int64_t(t.tm) * 256, int64_t(t.tn) * 128);
    else if (int64_t(t.tm) * 256 + 128 * second < p.tokens) gated_forward_tile<Half, ACT, SQUARE, FA>(p, lds, int64_t(t.tm) * 256 + 128 * second, int64_t(t.tn) * 128);
}

// ------------------------------------------------------------------ few tokens: values first

// Up to sixteen tokens. Rows of `pitch` floats, one for each token: h, then gate and up. No block has a whole block of 128 columns, so a second launch rounds them: 3 us of 21 to 23 for one token, 4096 to 11008 (90 MB; 16.5 to 18 us are this kernel's, 5 TB/s and more).
template <int WAVES, bool EIGHT, int ACT, int FA>
__global__ __launch_bounds__(64 * WAVES) void gated_few_kernel(GatedForward p, float *values, uint64_t pitch) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[F8Few<WAVES, 2, EIGHT>::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    f32x4 sum[2];
    F8Few<WAVES, 2, EIGHT>::template sums<FA, 0>(sum, p.x, p.w_gate, p.w_up, p.steps, n0, lds, lane, wave);
    if (wave > 0 || (lane & 15) >= p.tokens) return;
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; e++) h[e] = sum[0][e] * sigmoid_of<ACT>(sum[0][e]) * sum[1][e];
    float *at = values + (lane & 15) * pitch + n0 + 4 * (lane >> 4);
    *(f32x4 DSLLM_GLOBAL *)at = h;
    if (!p.gate.codes) return;
    *(f32x4 DSLLM_GLOBAL *)(at + p.tokens * pitch) = sum[0];
    *(f32x4 DSLLM_GLOBAL *)(at + 2 * p.tokens * pitch) = sum[1];
}

// Up to 64 tokens, values in the same rows: tiles of all tokens by 32 columns of gate and of up are four times as many as those with whole blocks of 128 (which of the two: gated_values_first).
template <int ACT, bool SQUARE, int FA>
__global__ __launch_bounds__(256, 2) void gated_values_kernel(GatedForward p, float *values, uint64_t pitch) {
    typedef F8GatedValuesShape S;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    const int64_t col = int64_t(blockIdx.x) * (S::BN / 2);
    const F8Loader<S> load(p.x, p.w_gate, p.w_up, p.steps, 0, col, lane, wave);
    f32x4 acc[S::TM][S::TN];
    f8_sums<S, SQUARE, true, FA, 0>(acc, lds, load, 0, p.steps, lane, wm, wn);
    const int row = 16 * S::TM * wm + S::TM * (lane & 15);
    float *at = values + row * pitch + col + 16 * wn + 4 * (lane >> 4);      // rows reach to a multiple of 128
#pragma unroll
    for (int i = 0; i < S::TM; i++, at += pitch) {
        if (row + i >= p.tokens) return;
        const f32x4 g = acc[i][0], u = acc[i][1];
        f32x4 h;
#pragma unroll
        for (int e = 0; e < 4; e++) h[e] = g[e] * sigmoid_of<ACT>(g[e]) * u[e];
        *(f32x4 DSLLM_GLOBAL *)at = h;
        if (!p.gate.codes) continue;
        *(f32x4 DSLLM_GLOBAL *)(at + p.tokens * pitch) = g;
        *(f32x4 DSLLM_GLOBAL *)(at + 2 * p.tokens * pitch) = u;
    }
}

__global__ __launch_bounds__(256) void gated_round_kernel(GatedForward p, const float *values, uint64_t pitch) {
    const F8Held &to = blockIdx.y == 0 ? p.h : blockIdx.y == 1 ? p.gate : p.up;
    const F8Source src{reinterpret_cast<const uint8_t *>(values + p.tokens * blockIdx.y * pitch), pitch, p.tokens, p.ffn, nullptr, 0, 0};
    f8_round_rows<CKPT_F32>(src, to, 16 * int64_t(blockIdx.z), 512 * int64_t(blockIdx.x));
}

// ------------------------------------------------------------------ backward

struct GatedBackward {
    F8Side dy, w_down;
    F8Held gate, up, dgate, dup, dgate_by_col, dup_by_col, h_by_col;
    int64_t tokens, ffn;
    uint32_t steps;
};

// A tile is 128 tokens by 128 columns, a block of each of the forms that are written, and its dh never leaves the registers: dgate, dup and h take their place. A lane has four consecutive rows (TM) of
// sixteen consecutive columns (TNG): 16 bytes of a row's codes, 4 of a column's. Largest values of rows are found among the lanes of a row (q) and, through LDS, two waves; those of columns among sixteen lanes and two waves.
// Two blocks share a compute unit, so that the vector work behind a tile's sums runs beside the other's matrix instructions. 4096 tokens, 4096 to 11008, all five forms 391 to 407 us: some 290 are the sums, the rest is the vector work, 2750 instructions a wave
// for 64 elements a lane, and 0.23 GB of stores.
// One body for whole and ragged tiles (two are 80 KB of code, more than the instruction cache holds): rows and columns past the end are the last ones again. Those columns change no largest value of a row; those rows get factors of zero, and
// are NaN only where the last row is.
template <int ACT, bool SQUARE, int FA, bool E5M2>
__global__ __launch_bounds__(256, 2) void gated_backward_kernel(GatedBackward p, TileOrder order) {
    typedef F8BackwardShape S;
    // largest magnitudes, [640][2]: 128 rows of dgate, of dup, 128 columns of dgate, of dup, of h, each as two waves have seen it; what they are multiplied with, [640]; gate's and up's codes, [32][256]
    constexpr int DGATE = 0, DUP = 128, DGATE_BY_COL = 256, DUP_BY_COL = 384, H_BY_COL = 512, EVERY = 640;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::BYTES];
    static_assert(12 * EVERY + 32 * 1024 <= S::BYTES, "");
    uint32_t *most = reinterpret_cast<uint32_t *>(lds), *parked = most + 3 * EVERY;
    float *inverses = reinterpret_cast<float *>(lds) + 2 * EVERY;
    const GemmTile t = gemm_tile(order);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, ar = lane & 15;
    const int64_t row = int64_t(t.tm) * 128, col = int64_t(t.tn) * 128;
    const F8Loader<S> load(p.dy, p.w_down, p.w_down, p.steps, row, col, lane, wave);
    f32x4 dgate[4][4], dup[4][4], h[4][4];
    const int64_t my_row = row + 64 * wm + 4 * ar, my_col = col + 64 * wn + 16 * q;
    u32x4 gates[4], ups[4];
    float gate_scale[4], up_scale[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t r = min(my_row + i, p.tokens - 1);
        gates[i] = *(const u32x4 DSLLM_GLOBAL *)(p.gate.codes + r * p.gate.code_pitch + my_col);
        ups[i] = *(const u32x4 DSLLM_GLOBAL *)(p.up.codes + r * p.up.code_pitch + my_col);
        gate_scale[i] = ((const float DSLLM_GLOBAL *)p.gate.scales)[t.tn * p.gate.scale_pitch + r];
        up_scale[i] = ((const float DSLLM_GLOBAL *)p.up.scales)[t.tn * p.up.scale_pitch + r];
    }
    f8_sums<S, SQUARE, true, FA, 0>(dgate, lds, load, 0, p.steps, lane, wm, wn);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (my_row + i >= p.tokens) gate_scale[i] = up_scale[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {      // there are no registers for them any more
            parked[(8 * j + i) * 256 + threadIdx.x] = gates[i][j];
            parked[(8 * j + 4 + i) * 256 + threadIdx.x] = ups[i][j];
        }
    }
    float most_dgate[4] = {}, most_dup[4] = {};
    uint32_t of_column[3] = {};      // of column 16 q + ar of the wave's, of dgate, dup and h
#pragma unroll
    for (int j = 0; j < 4; j++) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const f32x4 g = fp8_values(parked[(8 * j + i) * 256 + threadIdx.x]) * gate_scale[i], u = fp8_values(parked[(8 * j + 4 + i) * 256 + threadIdx.x]) * up_scale[i];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float s = sigmoid_of<ACT>(g[e]), act = g[e] * s, dh = dgate[i][j][e];
                dgate[i][j][e] = dh * u[e] * slope_of<ACT>(g[e], s, act);
                dup[i][j][e] = dh * act;
                h[i][j][e] = act * u[e];
            }
            // these four now: put off, as the compiler would, they need what they are made of as well, and spill
            asm volatile("" : "+v"(dgate[i][j]), "+v"(dup[i][j]), "+v"(h[i][j]));
            most_dgate[i] = larger(most_dgate[i], dgate[i][j]);
            most_dup[i] = larger(most_dup[i], dup[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        uint32_t found[12];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            auto column = [&](const f32x4 (&v)[4][4]) { return bits_of(larger(0, f32x4{v[0][j][e], v[1][j][e], v[2][j][e], v[3][j][e]})); };
            found[3 * e] = column(dgate);
            found[3 * e + 1] = column(dup);
            found[3 * e + 2] = column(h);
        }
        most_of_16(found);
#pragma unroll
        for (int k = 0; k < 12; k++) of_column[k % 3] = ar == 4 * j + k / 3 ? found[k] : of_column[k % 3];
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int k = 0; k < 3; k++) most[(DGATE_BY_COL + 128 * k + 64 * wn + 16 * q + ar) * 2 + wm] = of_column[k];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t of_dgate = most_of_quarters(bits_of(most_dgate[i])), of_dup = most_of_quarters(bits_of(most_dup[i]));
        if (q == 0) {
            most[(DGATE + 64 * wm + 4 * ar + i) * 2 + wn] = of_dgate;
            most[(DUP + 64 * wm + 4 * ar + i) * 2 + wn] = of_dup;
        }
    }
    __syncthreads();
    // every scale once: a division is some twenty instructions
    for (int k = threadIdx.x; k < EVERY; k += 256) {
        const F8Held &to = k < DUP ? p.dgate : k < DGATE_BY_COL ? p.dup : k < DUP_BY_COL ? p.dgate_by_col : k < H_BY_COL ? p.dup_by_col : p.h_by_col;
        const float largest = f8_most(E5M2 && k < H_BY_COL);
        const uint32_t amax = max(most[2 * k], most[2 * k + 1]);
        inverses[k] = f8_inverse(amax, largest);
        const int64_t block = k < DGATE_BY_COL ? t.tn : t.tm, of = (k < DGATE_BY_COL ? row : col) + k % 128;
        if (to.scales && of < to.rows) ((float DSLLM_GLOBAL *)to.scales)[block * to.scale_pitch + of] = f8_scale(amax, largest);
    }
    __syncthreads();
    // codes behind the last element are zero (NaN times zero would be none)
    uint32_t kept[4];
#pragma unroll
    for (int j = 0; j < 4; j++) kept[j] = bytes_kept(p.ffn - my_col - 4 * j);
    auto by_row = [&](const F8Held &to, int first, const f32x4 (&v)[4][4]) {
        if (!to.codes) return;
        uint8_t *at = to.codes + my_row * to.code_pitch + my_col;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float inverse = inverses[first + 64 * wm + 4 * ar + i];
            u32x4 codes;
#pragma unroll
            for (int j = 0; j < 4; j++) codes[j] = f8_codes(v[i][j] * inverse, E5M2) & kept[j];
            if (my_row + i < p.tokens) *(u32x4 DSLLM_GLOBAL *)(at + i * to.code_pitch) = codes;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const uint32_t rows_kept = bytes_kept(p.tokens - my_row);
    // a column past the end lies past the descriptor's end, and is not stored
    const uint32_t columns = uint32_t(min(p.ffn - col, int64_t(128)));
    auto by_col = [&](const F8Held &to, int first, const f32x4 (&v)[4][4], bool e5m2) {
        if (!to.codes) return;
        const uint32_t pitch = uint32_t(to.code_pitch);
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(to.codes + col * to.code_pitch + row, 0, (columns - 1) * pitch + 128, 0x00020000);
        uint32_t at = (64 * wn + 16 * q) * pitch + uint32_t(my_row - row);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const f32x4 inverse = *reinterpret_cast<const f32x4 *>(inverses + first + 64 * wn + 16 * q + 4 * j);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                __builtin_amdgcn_raw_buffer_store_b32(f8_codes(f32x4{v[0][j][e], v[1][j][e], v[2][j][e], v[3][j][e]} * inverse[e], e5m2) & rows_kept, rsrc, at, 0, 0);
                at += pitch;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    by_row(p.dgate, DGATE, dgate);
    by_row(p.dup, DUP, dup);
    by_col(p.dgate_by_col, DGATE_BY_COL, dgate, E5M2);
    by_col(p.dup_by_col, DUP_BY_COL, dup, E5M2);
    by_col(p.h_by_col, H_BY_COL, h, false);
}

// ------------------------------------------------------------------ host

template <class F>
void with_kinds(int32_t activation, bool e5m2, bool square, F f) {
    auto with_square = [&](auto act, auto fa) {
        if (square) f(act, fa, std::true_type());
        else f(act, fa, std::false_type());
    };
    auto with_format = [&](auto act) {
        if (e5m2) with_square(act, std::integral_constant<int, 1>());
        else with_square(act, std::integral_constant<int, 0>());
    };
    if (activation == CKPT_GATE_SILU) with_format(std::integral_constant<int, CKPT_GATE_SILU>());
    else with_format(std::integral_constant<int, CKPT_GATE_GELU>());
}

// Sides are at most 2^31 - 1. Fewer than 2^22 tiles, of up to 512 threads (and half a round of halves): a grid has fewer than 2^32 work-items.
bool fits_grid(int64_t down, int64_t across) { return down * across < 1 << 22; }
constexpr const char *kTooManyTiles = "2^22 tiles of tokens and columns or more";

// What the values of few tokens take, 0 where they are rounded in one launch.
uint64_t values_pitch(int64_t ffn) { return f8_padded(ffn); }
uint64_t values_bytes(int64_t tokens, int64_t ffn) { return uint64_t(tokens) <= kF8Few || gated_values_first(uint64_t(tokens), uint64_t(ffn)) ? 3 * tokens * values_pitch(ffn) * sizeof(float) : 0; }

int forward(const ckpt_f8_matrix *x, const ckpt_f8_matrix *w_gate, const ckpt_f8_matrix *w_up, int32_t activation, const ckpt_f8_matrix *gate, const ckpt_f8_matrix *up, const ckpt_f8_matrix *h,
            void *workspace, uint64_t workspace_bytes, hipStream_t stream) {
    if (!x || !w_gate || !w_up || !h) return refuse(CKPT_EINVAL, "null argument");
    if (!gate != !up) return refuse(CKPT_EINVAL, "gate and up are kept both or not at all");
    if (activation != CKPT_GATE_SILU && activation != CKPT_GATE_GELU) return refuse(CKPT_EINVAL, "activation must be CKPT_GATE_SILU or CKPT_GATE_GELU");
    DeviceRanges ranges;
    struct { const char *name; const ckpt_f8_matrix *m; } const every[] = {{"x: ", x}, {"w_gate: ", w_gate}, {"w_up: ", w_up}, {"gate: ", gate}, {"up: ", up}, {"h: ", h}};
    for (const auto &e : every)
        if (e.m)
            if (const char *why = wrong_f8_matrix(e.m, ranges)) return refuse(CKPT_EINVAL, std::string(e.name) + why);
    for (int i = 0; i < 3; i++)
        if (const char *why = wrong_f8_contraction(every[i].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + why);
    if (w_gate->format != CKPT_F8_E4M3 || w_up->format != CKPT_F8_E4M3) return refuse(CKPT_EINVAL, "w_gate and w_up must be CKPT_F8_E4M3");
    if (w_gate->block_rows != w_up->block_rows || w_gate->rows != w_up->rows) return refuse(CKPT_EINVAL, "w_gate and w_up differ in block_rows or rows");
    if (w_gate->cols != x->cols || w_up->cols != x->cols) return refuse(CKPT_EINVAL, "x and the weights differ in their columns");
    const int64_t tokens = x->rows, ffn = w_gate->rows;
    if (tokens > 0x7FFFFFFF || ffn > 0x7FFFFFFF) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1");
    for (int i = 3; i < 6; i++)
        if (every[i].m) {
            if (every[i].m->rows != tokens || every[i].m->cols != ffn) return refuse(CKPT_EINVAL, std::string(every[i].name) + "not tokens x ffn");
            if (every[i].m->block_rows != 1 || every[i].m->format != CKPT_F8_E4M3) return refuse(CKPT_EINVAL, std::string(every[i].name) + "must be CKPT_F8_E4M3 with block_rows 1");
            if (overlaps_itself(*every[i].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + "codes and scales overlap");
            for (int k = 0; k < i; k++)
                if (every[k].m && overlap(*every[i].m, *every[k].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + "overlaps another matrix");
        }
    if (tokens == 0 || ffn == 0) return CKPT_OK;
    const uint32_t steps = f8_steps(uint64_t(x->cols));
    const GatedForward p{f8_side(x), f8_side(w_gate), f8_side(w_up), F8Held(gate), F8Held(up), F8Held(h), tokens, ffn, steps};
    const bool x_e5m2 = x->format == CKPT_F8_E5M2;
    const int64_t across = (ffn + 127) / 128;
    const uint64_t bytes = values_bytes(tokens, ffn);
    if (bytes && steps && workspace && workspace_bytes >= bytes && across < 1 << 20) {
        if (uint64_t(workspace) % 16) return refuse(CKPT_EINVAL, "workspace must be 16-byte aligned");
        if (const char *why = ranges.wrong(workspace, bytes)) return refuse(CKPT_EINVAL, std::string("workspace: ") + why);
        for (const auto &e : every)
            if (e.m && overlap(*e.m, Rows{uint64_t(workspace), bytes, bytes, 1})) return refuse(CKPT_EINVAL, std::string(e.name) + "overlaps the workspace");
        float *values = static_cast<float *>(workspace);
        const uint64_t pitch = values_pitch(ffn);
        if (uint64_t(tokens) > kF8Few)
            with_kinds(activation, x_e5m2, p.w_gate.shift, [&](auto act, auto fa, auto square) { hipLaunchKernelGGL((gated_values_kernel<act, square, fa>), dim3(unsigned((ffn + 31) / 32)), dim3(256), 0, stream, p, values, pitch); });
        else
            with_kinds(activation, x_e5m2, true, [&](auto act, auto fa, auto) {
                auto launch = [&](auto waves, auto eight) { hipLaunchKernelGGL((gated_few_kernel<waves, eight, act, fa>), dim3(unsigned((ffn + 15) / 16)), dim3(64 * waves), 0, stream, p, values, pitch); };
                if (f8_few_waves(uint64_t(ffn), steps) == 2) tokens <= 8 ? launch(std::integral_constant<int, 2>(), std::true_type()) : launch(std::integral_constant<int, 2>(), std::false_type());
                else tokens <= 8 ? launch(std::integral_constant<int, 4>(), std::true_type()) : launch(std::integral_constant<int, 4>(), std::false_type());
            });
        hipLaunchKernelGGL(gated_round_kernel, dim3(unsigned((ffn + 511) / 512), gate ? 3 : 1, unsigned((tokens + 15) / 16)), dim3(256), 0, stream, p, values, pitch);
        return launched();
    }
    auto tiles = [&](auto shape) {
        typedef decltype(shape) S;
        const int64_t down = (tokens + S::BM - 1) / S::BM;
        if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooManyTiles);
        const dim3 grid(unsigned(down * across)), block(S::THREADS);
        const TileOrder order(uint32_t(down), uint32_t(across), true);
        with_kinds(activation, x_e5m2, p.w_gate.shift, [&](auto act, auto fa, auto square) { hipLaunchKernelGGL((gated_forward_kernel<S, act, square, fa>), grid, block, 0, stream, p, order); });
        return launched();
    };
    switch (gated_form(uint64_t(tokens), uint64_t(across), steps)) {
        case kGatedHalves: {
            const int64_t down = (tokens + 255) / 256, count = down * across, rest = count % kF8Units;
            if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooManyTiles);
            with_kinds(activation, x_e5m2, p.w_gate.shift, [&](auto act, auto fa, auto square) {
                hipLaunchKernelGGL((gated_forward_halves_kernel<act, square, fa>), dim3(unsigned(count + rest)), dim3(512), 0, stream, p, TileOrder(uint32_t(down), uint32_t(across), true), uint32_t(count - rest));
            });
            return launched();
        }
        case 0: return tiles(F8GatedShape<0>::type());
        case 1: return tiles(F8GatedShape<1>::type());
        default: return tiles(F8GatedShape<2>::type());
    }
}

int backward(const ckpt_f8_matrix *dy, const ckpt_f8_matrix *w_down, const ckpt_f8_matrix *gate, const ckpt_f8_matrix *up, int32_t activation, const ckpt_gated_grads *grads, hipStream_t stream) {
    if (!dy || !w_down || !gate || !up || !grads) return refuse(CKPT_EINVAL, "null argument");
    if (activation != CKPT_GATE_SILU && activation != CKPT_GATE_GELU) return refuse(CKPT_EINVAL, "activation must be CKPT_GATE_SILU or CKPT_GATE_GELU");
    DeviceRanges ranges;
    struct { const char *name; const ckpt_f8_matrix *m; } const every[] = {{"dy: ", dy}, {"w_down_by_col: ", w_down}, {"gate: ", gate}, {"up: ", up}, {"dgate: ", grads->dgate}, {"dup: ", grads->dup},
                                                                         {"dgate_by_col: ", grads->dgate_by_col}, {"dup_by_col: ", grads->dup_by_col}, {"h_by_col: ", grads->h_by_col}};
    bool any = false;
    for (int i = 0; i < 9; i++)
        if (every[i].m) {
            any |= i >= 4;
            if (const char *why = wrong_f8_matrix(every[i].m, ranges)) return refuse(CKPT_EINVAL, std::string(every[i].name) + why);
        }
    if (!any) return refuse(CKPT_EINVAL, "nothing is asked for");
    for (int i = 0; i < 2; i++)
        if (const char *why = wrong_f8_contraction(every[i].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + why);
    if (w_down->format != CKPT_F8_E4M3) return refuse(CKPT_EINVAL, "w_down_by_col must be CKPT_F8_E4M3");
    int32_t format = 0;
    for (int i = 6; i < 9; i++)
        if (every[i].m && every[i].m->code_pitch > uint64_t(kF8LongestRow)) return refuse(CKPT_EINVAL, std::string(every[i].name) + "a pitch of at most 2^23 is wanted");
    for (int i = 4; i < 8; i++)
        if (every[i].m) {
            if (format && every[i].m->format != format) return refuse(CKPT_EINVAL, "the gradients differ in their format");
            format = every[i].m->format;
        }
    const bool e5m2 = format == CKPT_F8_E5M2;
    if (dy->cols != w_down->cols) return refuse(CKPT_EINVAL, "dy and w_down_by_col differ in their columns");
    const int64_t tokens = dy->rows, ffn = w_down->rows;
    if (tokens > 0x7FFFFFFF || ffn > 0x7FFFFFFF) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1");
    for (int i = 2; i < 9; i++)
        if (every[i].m) {
            if (every[i].m->rows != (i < 6 ? tokens : ffn) || every[i].m->cols != (i < 6 ? ffn : tokens)) return refuse(CKPT_EINVAL, std::string(every[i].name) + (i < 6 ? "not tokens x ffn" : "not ffn x tokens"));
            if (every[i].m->block_rows != 1) return refuse(CKPT_EINVAL, std::string(every[i].name) + "block_rows must be 1");
            if ((i < 4 || i == 8) && every[i].m->format != CKPT_F8_E4M3) return refuse(CKPT_EINVAL, std::string(every[i].name) + "must be CKPT_F8_E4M3");
            if (i >= 4 && overlaps_itself(*every[i].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + "codes and scales overlap");
            for (int k = 0; i >= 4 && k < i; k++)
                if (every[k].m && overlap(*every[i].m, *every[k].m)) return refuse(CKPT_EINVAL, std::string(every[i].name) + "overlaps another matrix");
        }
    if (tokens == 0 || ffn == 0) return CKPT_OK;
    const GatedBackward p{f8_side(dy), f8_side(w_down), F8Held(gate), F8Held(up), F8Held(grads->dgate), F8Held(grads->dup), F8Held(grads->dgate_by_col), F8Held(grads->dup_by_col), F8Held(grads->h_by_col),
                          tokens, ffn, f8_steps(uint64_t(dy->cols))};
    const int64_t down = (tokens + 127) / 128, across = (ffn + 127) / 128;
    if (!fits_grid(down, across)) return refuse(CKPT_EINVAL, kTooManyTiles);
    const dim3 grid(unsigned(down * across));
    const TileOrder order(uint32_t(down), uint32_t(across), true);
    with_kinds(activation, dy->format == CKPT_F8_E5M2, p.w_down.shift, [&](auto act, auto fa, auto square) {
        if (e5m2) hipLaunchKernelGGL((gated_backward_kernel<act, square, fa, true>), grid, dim3(256), 0, stream, p, order);
        else hipLaunchKernelGGL((gated_backward_kernel<act, square, fa, false>), grid, dim3(256), 0, stream, p, order);
    });
    return launched();
}

}  // namespace

extern "C" {

int ckpt_gated_workspace(int64_t tokens, int64_t ffn, int64_t hidden, uint64_t *bytes) {
    return at_c_entry([&] {
        if (!bytes || tokens < 0 || ffn < 0 || hidden < 0) return refuse(CKPT_EINVAL, "null argument or negative size");
        *bytes = 0;
        if (tokens > 0x7FFFFFFF || ffn > 0x7FFFFFFF || hidden > kF8LongestRow) return refuse(CKPT_EINVAL, "a side is over 2^31 - 1, or what is contracted over 2^23");
        if (tokens && ffn && hidden) *bytes = values_bytes(tokens, ffn);
        return int(CKPT_OK);
    });
}

int ckpt_gated_forward(const ckpt_f8_matrix *x, const ckpt_f8_matrix *w_gate, const ckpt_f8_matrix *w_up, int32_t activation, const ckpt_f8_matrix *gate, const ckpt_f8_matrix *up,
                       const ckpt_f8_matrix *h, void *workspace, uint64_t workspace_bytes, void *stream) {
    return at_c_entry([&] { return forward(x, w_gate, w_up, activation, gate, up, h, workspace, workspace_bytes, static_cast<hipStream_t>(stream)); });
}

int ckpt_gated_backward(const ckpt_f8_matrix *dy, const ckpt_f8_matrix *w_down_by_col, const ckpt_f8_matrix *gate, const ckpt_f8_matrix *up, int32_t activation, const ckpt_gated_grads *grads,
                        void *stream) {
    return at_c_entry([&] { return backward(dy, w_down_by_col, gate, up, activation, grads, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
