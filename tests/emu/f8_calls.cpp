// The host side of the operators with 8-bit matrices in blocks of 128, on the runtime of train_calls.cpp: what is refused, before anything is launched, and the launches of products and blocks of every size.
#define main main_of_train_calls
#include "train_calls.cpp"
#undef main

#include "../../paper_2406_10707_amd/csrc/f8_forms.hpp"
#include "../../paper_2406_10707_amd/csrc/f8_loader.hpp"

namespace {

struct Product {      // as f8_gemm.hip has it
    dsllm::F8Side a, b;
    void *c;
    int64_t ldc, m, n;
    uint32_t steps, steps_a_split;
    int64_t c_split;
    int32_t accumulate, dtype;
};

ckpt_f8_matrix matrix(int32_t format, int64_t rows, int64_t cols, int32_t block_rows = 1, int device = 0) {
    ckpt_f8_matrix m;
    REQUIRE(ckpt_f8_layout(format, block_rows, rows, cols, &m) == CKPT_OK);
    if (rows && cols) {
        m.codes = allocate(uint64_t(rows) * m.code_pitch, device);
        m.scales = static_cast<float *>(allocate(4 * (m.code_pitch / 128) * m.scale_pitch, device));
    }
    return m;
}

// A call that is refused, with a text, and launches nothing.
#define REFUSED(call) do { launches.clear(); dsllm::g_last_error.clear(); REQUIRE((call) == CKPT_EINVAL); REQUIRE(launches.empty() && !dsllm::g_last_error.empty()); printf("# %s\n", dsllm::g_last_error.c_str()); } while (0)
#define TAKEN(call) do { launches.clear(); REQUIRE((call) == CKPT_OK); REQUIRE(!launches.empty()); } while (0)
#define NOTHING(call) do { launches.clear(); REQUIRE((call) == CKPT_OK); REQUIRE(launches.empty()); } while (0)

template <class F>
ckpt_f8_matrix but(ckpt_f8_matrix m, F change) {
    change(m);
    return m;
}

// Every way a matrix can be malformed, as an argument of `call`.
template <class F>
void malformed(const ckpt_f8_matrix &m, F call) {
    const ckpt_f8_matrix wrong[] = {
        but(m, [](auto &x) { x.format = 1; }), but(m, [](auto &x) { x.format = 5; }), but(m, [](auto &x) { x.block_rows = 0; }), but(m, [](auto &x) { x.block_rows = 64; }), but(m, [](auto &x) { x.rows = -1; }),
        but(m, [](auto &x) { x.cols = -1; }), but(m, [](auto &x) { x.rows = 1ll << 41; }), but(m, [](auto &x) { x.cols = 1ll << 62; }), but(m, [](auto &x) { x.code_pitch += 8; }), but(m, [](auto &x) { x.code_pitch -= 128; }),
        but(m, [](auto &x) { x.code_pitch = 1ull << 60; }), but(m, [](auto &x) { x.codes = static_cast<char *>(x.codes) + 1; }), but(m, [](auto &x) { x.codes = nullptr; }), but(m, [](auto &x) { x.scales = nullptr; }),
        but(m, [](auto &x) { x.scales = reinterpret_cast<float *>(uint64_t(x.scales) + 2); }), but(m, [](auto &x) { x.scale_pitch -= 1; }), but(m, [](auto &x) { x.scale_pitch = 1ull << 62; }), but(m, [](auto &x) { x.rows += 100000000; x.scale_pitch += 100000000; }),
        but(m, [](auto &x) { x.codes = static_cast<char *>(x.codes) + 16; }), but(m, [](auto &x) { x.codes = reinterpret_cast<void *>(4096); }), but(m, [](auto &x) { x.scales += 1; })};
    for (const ckpt_f8_matrix &w : wrong) REFUSED(call(&w));
}

void refusals() {
    ckpt_f8_matrix out;
    REFUSED(ckpt_f8_layout(CKPT_F8_E4M3, 1, 3, 3, nullptr));
    REFUSED(ckpt_f8_layout(CKPT_MXFP8, 1, 3, 3, &out));
    REFUSED(ckpt_f8_layout(CKPT_F8_E4M3, 2, 3, 3, &out));
    REFUSED(ckpt_f8_layout(CKPT_F8_E4M3, 1, -3, 3, &out));
    // conversion
    const auto row = matrix(CKPT_F8_E4M3, 300, 200), col = matrix(CKPT_F8_E4M3, 200, 300), row128 = matrix(CKPT_F8_E4M3, 300, 200, 128), col128 = matrix(CKPT_F8_E4M3, 200, 300, 128), col_e5m2 = matrix(CKPT_F8_E5M2, 200, 300),
               col128_e5m2 = matrix(CKPT_F8_E5M2, 200, 300, 128), there = matrix(CKPT_F8_E4M3, 300, 200, 1, 1);
    void *src = allocate(4 * 300 * 210), *elsewhere = allocate(4 * 300 * 210, 1);
    TAKEN(ckpt_f8_quantize(src, CKPT_F32, 210, &row, &col, nullptr));
    TAKEN(ckpt_f8_quantize(src, CKPT_F32, 210, &row, &col_e5m2, nullptr));
    TAKEN(ckpt_f8_quantize(src, CKPT_BF16, 210, &row128, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 210, nullptr, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_U8, 210, &row, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 199, &row, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 1ll << 60, &row, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 400, &row, nullptr, nullptr));                       // past the end of src
    REFUSED(ckpt_f8_quantize(nullptr, CKPT_F32, 210, &row, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(static_cast<char *>(src) + 1, CKPT_BF16, 210, &row, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(elsewhere, CKPT_F32, 210, &row, nullptr, nullptr));                 // another device's memory
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 210, &there, nullptr, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 210, &row, &row, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 210, &row, &col128, nullptr));
    REFUSED(ckpt_f8_quantize(src, CKPT_F32, 210, &row128, &col128_e5m2, nullptr));
    malformed(row, [&](const ckpt_f8_matrix *m) { return ckpt_f8_quantize(src, CKPT_F32, 210, m, nullptr, nullptr); });
    malformed(col128, [&](const ckpt_f8_matrix *m) { return ckpt_f8_quantize(src, CKPT_F32, 210, nullptr, m, nullptr); });
    const auto none = matrix(CKPT_F8_E4M3, 0, 200), none_col = matrix(CKPT_F8_E4M3, 200, 0);
    NOTHING(ckpt_f8_quantize(nullptr, CKPT_F32, 200, &none, &none_col, nullptr));
    TAKEN(ckpt_f8_columns(&row, &col, nullptr));
    TAKEN(ckpt_f8_columns(&row, &col_e5m2, nullptr));
    TAKEN(ckpt_f8_columns(&row128, &col128, nullptr));
    REFUSED(ckpt_f8_columns(&row, nullptr, nullptr));
    REFUSED(ckpt_f8_columns(nullptr, &col, nullptr));
    REFUSED(ckpt_f8_columns(&row, &row, nullptr));
    REFUSED(ckpt_f8_columns(&row128, &col, nullptr));
    REFUSED(ckpt_f8_columns(&row128, &col128_e5m2, nullptr));
    NOTHING(ckpt_f8_columns(&none, &none_col, nullptr));
    malformed(row, [&](const ckpt_f8_matrix *m) { return ckpt_f8_columns(m, &col, nullptr); });
    malformed(col, [&](const ckpt_f8_matrix *m) { return ckpt_f8_columns(&row, m, nullptr); });
    TAKEN(ckpt_f8_dequantize(&row128, src, CKPT_F32, 210, nullptr));
    REFUSED(ckpt_f8_dequantize(nullptr, src, CKPT_F32, 210, nullptr));
    REFUSED(ckpt_f8_dequantize(&row, nullptr, CKPT_F32, 210, nullptr));
    REFUSED(ckpt_f8_dequantize(&row, src, 77, 210, nullptr));
    REFUSED(ckpt_f8_dequantize(&row, src, CKPT_F32, 100, nullptr));
    REFUSED(ckpt_f8_dequantize(&row, src, CKPT_F32, 300, nullptr));
    REFUSED(ckpt_f8_dequantize(&row, static_cast<char *>(src) + 2, CKPT_F32, 200, nullptr));
    malformed(row, [&](const ckpt_f8_matrix *m) { return ckpt_f8_dequantize(m, src, CKPT_F32, 210, nullptr); });
    // product
    uint64_t bytes;
    REFUSED(ckpt_f8_gemm_workspace(-1, 1, 1, &bytes));
    REFUSED(ckpt_f8_gemm_workspace(1, 1, 1, nullptr));
    REFUSED(ckpt_f8_gemm_workspace(1ll << 31, 1, 1, &bytes));
    REFUSED(ckpt_f8_gemm_workspace(1, 1, (1 << 23) + 1, &bytes));
    const auto a = matrix(CKPT_F8_E5M2, 300, 200), b = matrix(CKPT_F8_E4M3, 500, 200, 128), other = matrix(CKPT_F8_E4M3, 500, 201), wide = matrix(CKPT_F8_E4M3, 3, (1 << 23) + 1);
    void *c = allocate(4 * 300 * 500);
    TAKEN(ckpt_f8_gemm(&a, &b, c, CKPT_F32, 500, 1, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(nullptr, &b, c, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, nullptr, c, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &other, c, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&wide, &wide, c, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &b, c, CKPT_U8, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &b, c, CKPT_F32, 499, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &b, c, CKPT_F32, 600, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &b, nullptr, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    REFUSED(ckpt_f8_gemm(&a, &b, static_cast<char *>(c) + 2, CKPT_F32, 400, 0, nullptr, 0, nullptr));
    malformed(a, [&](const ckpt_f8_matrix *m) { return ckpt_f8_gemm(m, &b, c, CKPT_F32, 500, 0, nullptr, 0, nullptr); });
    malformed(b, [&](const ckpt_f8_matrix *m) { return ckpt_f8_gemm(&a, m, c, CKPT_F32, 500, 0, nullptr, 0, nullptr); });
    const auto long_a = matrix(CKPT_F8_E4M3, 64, 16384), long_b = matrix(CKPT_F8_E4M3, 64, 16384);
    REQUIRE(ckpt_f8_gemm_workspace(64, 64, 16384, &bytes) == CKPT_OK && bytes > 0);
    char *ws = static_cast<char *>(allocate(bytes));
    TAKEN(ckpt_f8_gemm(&long_a, &long_b, c, CKPT_F32, 64, 0, ws, bytes, nullptr));
    REQUIRE(launches.size() == 2);
    TAKEN(ckpt_f8_gemm(&long_a, &long_b, c, CKPT_F32, 64, 0, nullptr, 0, nullptr));
    REQUIRE(launches.size() == 1);
    REFUSED(ckpt_f8_gemm(&long_a, &long_b, c, CKPT_F32, 64, 0, ws + 4, bytes - 4, nullptr));
    REFUSED(ckpt_f8_gemm(&long_a, &long_b, c, CKPT_F32, 64, 0, reinterpret_cast<void *>(8192), bytes, nullptr));
    REFUSED(ckpt_f8_gemm(&long_a, &long_b, c, CKPT_F32, 64, 0, ws + (1 << 21), bytes, nullptr));
    const auto no_k = matrix(CKPT_F8_E4M3, 64, 0);
    TAKEN(ckpt_f8_gemm(&no_k, &no_k, c, CKPT_F32, 64, 0, nullptr, 0, nullptr));
    NOTHING(ckpt_f8_gemm(&no_k, &no_k, c, CKPT_F32, 64, 1, nullptr, 0, nullptr));
    NOTHING(ckpt_f8_gemm(&none, &b, nullptr, CKPT_F32, 500, 0, nullptr, 0, nullptr));
    // the gated block
    REFUSED(ckpt_gated_workspace(1, 1, 1, nullptr));
    REFUSED(ckpt_gated_workspace(1, -1, 1, &bytes));
    REFUSED(ckpt_gated_workspace(1, 1, 1ll << 40, &bytes));
    const auto x = matrix(CKPT_F8_E5M2, 40, 200), wg = matrix(CKPT_F8_E4M3, 300, 200, 128), wu = matrix(CKPT_F8_E4M3, 300, 200, 128), wu1 = matrix(CKPT_F8_E4M3, 300, 200), w5 = matrix(CKPT_F8_E5M2, 300, 200, 128), ws2 = matrix(CKPT_F8_E4M3, 299, 200, 128),
               gate = matrix(CKPT_F8_E4M3, 40, 300), up = matrix(CKPT_F8_E4M3, 40, 300), h = matrix(CKPT_F8_E4M3, 40, 300), h5 = matrix(CKPT_F8_E5M2, 40, 300), h128 = matrix(CKPT_F8_E4M3, 40, 300, 128), small = matrix(CKPT_F8_E4M3, 39, 300);
    auto forward = [&](const ckpt_f8_matrix *x, const ckpt_f8_matrix *g, const ckpt_f8_matrix *u, int act, const ckpt_f8_matrix *kg, const ckpt_f8_matrix *ku, const ckpt_f8_matrix *h) {
        return ckpt_gated_forward(x, g, u, act, kg, ku, h, nullptr, 0, nullptr);
    };
    TAKEN(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h));
    TAKEN(forward(&x, &wg, &wu, CKPT_GATE_GELU, nullptr, nullptr, &h));
    REFUSED(forward(nullptr, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&x, nullptr, &wu, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, nullptr));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, nullptr, &h));
    REFUSED(forward(&x, &wg, &wu, 0, &gate, &up, &h));
    REFUSED(forward(&x, &wg, &wu, 3, &gate, &up, &h));
    REFUSED(forward(&x, &wg, &wu1, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&x, &w5, &w5, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&x, &wg, &ws2, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&row, &gate, &up, CKPT_GATE_SILU, &gate, &up, &h));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h5));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h128));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &small));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &h, &up, &h));             // one matrix written twice
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &gate, &h));
    malformed(x, [&](const ckpt_f8_matrix *m) { return forward(m, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h); });
    malformed(wg, [&](const ckpt_f8_matrix *m) { return forward(&x, m, &wu, CKPT_GATE_SILU, &gate, &up, &h); });
    malformed(gate, [&](const ckpt_f8_matrix *m) { return forward(&x, &wg, &wu, CKPT_GATE_SILU, m, &up, &h); });
    malformed(h, [&](const ckpt_f8_matrix *m) { return forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, m); });
    // halves of one wider matrix, side by side, do not overlap; halves that begin too near do
    const auto both = matrix(CKPT_F8_E4M3, 40, 768);
    auto half = [&](int64_t at) { return ckpt_f8_matrix{CKPT_F8_E4M3, 1, 40, 300, static_cast<char *>(both.codes) + at, both.code_pitch, both.scales + at / 128 * both.scale_pitch, both.scale_pitch}; };
    const auto left = half(0), right = half(384), near = half(256);
    TAKEN(forward(&x, &wg, &wu, CKPT_GATE_SILU, &left, &right, &h));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &left, &near, &h));
    REFUSED(forward(&x, &wg, &wu, CKPT_GATE_SILU, &near, &left, &h));
    const auto x1 = matrix(CKPT_F8_E4M3, 16, 200), h1 = matrix(CKPT_F8_E4M3, 16, 300);
    REQUIRE(ckpt_gated_workspace(16, 300, 200, &bytes) == CKPT_OK && bytes > 0);
    char *fws = static_cast<char *>(allocate(bytes));
    TAKEN(ckpt_gated_forward(&x1, &wg, &wu, CKPT_GATE_SILU, nullptr, nullptr, &h1, fws, bytes, nullptr));
    REQUIRE(launches.size() == 2);
    TAKEN(ckpt_gated_forward(&x1, &wg, &wu, CKPT_GATE_SILU, nullptr, nullptr, &h1, fws, bytes - 1, nullptr));
    REQUIRE(launches.size() == 1);
    const auto x64 = matrix(CKPT_F8_E4M3, 64, 200), w4096 = matrix(CKPT_F8_E4M3, 4096, 200, 128), u4096 = matrix(CKPT_F8_E4M3, 4096, 200, 128), h64 = matrix(CKPT_F8_E4M3, 64, 4096), g64 = matrix(CKPT_F8_E4M3, 64, 4096),
               p64 = matrix(CKPT_F8_E4M3, 64, 4096);
    uint64_t values;
    REQUIRE(ckpt_gated_workspace(64, 4096, 200, &values) == CKPT_OK && values == 3ull * 64 * 4096 * 4);
    char *vws = static_cast<char *>(allocate(values));
    for (const ckpt_f8_matrix *gate64 : {static_cast<const ckpt_f8_matrix *>(nullptr), &g64}) {
        TAKEN(ckpt_gated_forward(&x64, &w4096, &u4096, CKPT_GATE_SILU, gate64, gate64 ? &p64 : nullptr, &h64, vws, values, nullptr));
        REQUIRE(launches.size() == 2);
        TAKEN(ckpt_gated_forward(&x64, &w4096, &u4096, CKPT_GATE_SILU, gate64, gate64 ? &p64 : nullptr, &h64, vws, values - 1, nullptr));
        REQUIRE(launches.size() == 1);
    }
    REFUSED(ckpt_gated_forward(&x64, &w4096, &u4096, CKPT_GATE_SILU, nullptr, nullptr, &h64, vws + 8, values, nullptr));
    REFUSED(ckpt_gated_forward(&x64, &w4096, &u4096, CKPT_GATE_SILU, nullptr, nullptr, &h64, vws + 16, values, nullptr));
    REFUSED(ckpt_gated_forward(&x1, &wg, &wu, CKPT_GATE_SILU, nullptr, nullptr, &h1, fws + 4, bytes, nullptr));
    REFUSED(ckpt_gated_forward(&x1, &wg, &wu, CKPT_GATE_SILU, nullptr, nullptr, &h1, fws + (1 << 21), bytes, nullptr));
    // backward
    const auto dy = matrix(CKPT_F8_E5M2, 40, 200), wd = matrix(CKPT_F8_E4M3, 300, 200, 128), dgate = matrix(CKPT_F8_E5M2, 40, 300), dup = matrix(CKPT_F8_E5M2, 40, 300), dup4 = matrix(CKPT_F8_E4M3, 40, 300), dgc = matrix(CKPT_F8_E5M2, 300, 40),
               hc = matrix(CKPT_F8_E4M3, 300, 40), hc5 = matrix(CKPT_F8_E5M2, 300, 40);
    auto backward = [&](const ckpt_f8_matrix *dy, const ckpt_f8_matrix *wd, const ckpt_f8_matrix *g, const ckpt_f8_matrix *u, int act, ckpt_gated_grads grads) { return ckpt_gated_backward(dy, wd, g, u, act, &grads, nullptr); };
    TAKEN(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {&dgate, &dup, &dgc, nullptr, &hc}));
    TAKEN(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, nullptr, nullptr, &hc}));
    REFUSED(ckpt_gated_backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, nullptr, nullptr));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {}));
    REFUSED(backward(nullptr, &wd, &gate, &up, CKPT_GATE_SILU, {&dgate}));
    REFUSED(backward(&dy, &wd, &gate, nullptr, CKPT_GATE_SILU, {&dgate}));
    REFUSED(backward(&dy, &wd, &gate, &up, 9, {&dgate}));
    REFUSED(backward(&dy, &w5, &gate, &up, CKPT_GATE_SILU, {&dgate}));
    REFUSED(backward(&dy, &wd, &h5, &up, CKPT_GATE_SILU, {&dgate}));
    REFUSED(backward(&dy, &wd, &h128, &up, CKPT_GATE_SILU, {&dgate}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {&dgate, &dup4}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {&dgc}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, &dgate}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, nullptr, nullptr, &hc5}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {&dgate, &dgate}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {&gate}));                  // in the place of what is read
    REFUSED(backward(&dy, &ws2, &gate, &up, CKPT_GATE_SILU, {&dgate}));
    auto pitched = [&](uint64_t pitch) { return but(dgc, [&](auto &x) { x.code_pitch = pitch; x.codes = allocate(300 * pitch); }); };
    const auto longest = pitched(1 << 23), longer = pitched((1 << 23) + 16);
    TAKEN(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, &longest}));
    REFUSED(backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, &longer}));
    malformed(dy, [&](const ckpt_f8_matrix *m) { return backward(m, &wd, &gate, &up, CKPT_GATE_SILU, {&dgate}); });
    malformed(gate, [&](const ckpt_f8_matrix *m) { return backward(&dy, &wd, m, &up, CKPT_GATE_SILU, {&dgate}); });
    malformed(dgc, [&](const ckpt_f8_matrix *m) { return backward(&dy, &wd, &gate, &up, CKPT_GATE_SILU, {nullptr, nullptr, m}); });
}

// Every element of C is some launch's, once, and every launch reads the rows and scales of A and B that go with its part.
void products_beyond_a_grid() {
    struct { int64_t m, n, k; int32_t blocks; } sizes[] = {{1, (1ll << 29) + 5, 256, 128}, {16, (1ll << 28) + 77, 128, 1}, {1, (1ll << 31) - 1, 100, 128}, {5000000, 3, 0, 1}, {17, (1ll << 30) + 9, 0, 128}, {(1ll << 31) - 1, 1, 0, 1},
                                                           {17, (1ll << 31) - 1, 130, 128}, {3000000, 700, 128, 128}, {300000, 300000, 128, 1}, {3, 5, 0, 1}, {4097, 3, 40, 128}};
    for (const auto &s : sizes)
        for (int dtype : {int(CKPT_BF16), int(CKPT_F32)}) {
            const uint64_t size = dtype == CKPT_F32 ? 4 : 2;
            const auto a = matrix(CKPT_F8_E4M3, s.m, s.k, s.blocks), b = matrix(CKPT_F8_E4M3, s.n, s.k, s.blocks);
            const int64_t ldc = s.n + 3;
            char *c = static_cast<char *>(allocate(uint64_t(s.m) * ldc * size));
            first_argument_bytes = sizeof(Product);
            launches.clear();
            const int rc = ckpt_f8_gemm(&a, &b, c, dtype, ldc, 0, nullptr, 0, nullptr);
            printf("# %lld x %lld x %lld, %llu bytes an element: %d, %zu launches\n", (long long)s.m, (long long)s.n, (long long)s.k, (unsigned long long)size, rc, launches.size());
            REQUIRE(rc == CKPT_OK && !launches.empty());
            uint64_t covered = 0;
            for (const Launch &l : launches) {
                Product p;
                memcpy(&p, l.first.data(), sizeof p);
                const uint64_t at = (static_cast<char *>(p.c) - c) / size, row = at / ldc, col = at % ldc;
                REQUIRE(p.m > 0 && p.n > 0 && int64_t(row) + p.m <= s.m && int64_t(col) + p.n <= s.n && p.ldc == ldc && p.a.rows == p.m && p.b.rows == p.n && p.dtype == dtype);
                if (s.k) {
                    REQUIRE(p.a.codes == static_cast<uint8_t *>(a.codes) + row * a.code_pitch && p.a.scales == a.scales + row / s.blocks && row % s.blocks == 0);
                    REQUIRE(p.b.codes == static_cast<uint8_t *>(b.codes) + col * b.code_pitch && p.b.scales == b.scales + col / s.blocks && col % s.blocks == 0);
                }
                covered += uint64_t(p.m) * p.n;
                if (l.kernel.find("few") != std::string::npos) REQUIRE(l.grid.x == uint64_t(p.n + 15) / 16 && p.m <= 16);
                else REQUIRE(l.grid.x <= dsllm::kF8MostTiles);
            }
            REQUIRE(covered == uint64_t(s.m) * s.n);
            allocations.clear();
        }
}

// The blocks of the gated block's launches: enough for every tile, also where those of the last round are halves.
void tiles_of_blocks() {
    first_argument_bytes = 8;
    const auto w = matrix(CKPT_F8_E4M3, 11008, 256, 128), w2 = matrix(CKPT_F8_E4M3, 11008, 256, 128);
    bool halves = false;
    for (int64_t tokens : {17, 64, 65, 256, 700, 1024, 2048, 4000, 4096, 8192}) {
        const auto x = matrix(CKPT_F8_E4M3, tokens, 256), h = matrix(CKPT_F8_E4M3, tokens, 11008);
        TAKEN(ckpt_gated_forward(&x, &w, &w2, CKPT_GATE_SILU, nullptr, nullptr, &h, nullptr, 0, nullptr));
        REQUIRE(launches.size() == 1);
        const Launch &l = launches[0];
        const bool half = l.kernel.find("halves") != std::string::npos;
        const int form = dsllm::gated_form(uint64_t(tokens), 86, 2);
        REQUIRE(half == (form == dsllm::kGatedHalves));
        halves |= half;
        const int64_t rows = half || form == 0 ? 256 : form == 1 ? 128 : 64, count = (tokens + rows - 1) / rows * 86;
        REQUIRE(int64_t(l.grid.x) == (half ? count + count % 256 : count));
        printf("# %lld tokens: %u blocks, form %d\n", (long long)tokens, l.grid.x, form);
    }
    REQUIRE(halves);
    const auto x = matrix(CKPT_F8_E4M3, 1ll << 24, 128), wl = matrix(CKPT_F8_E4M3, 16384, 128), h = matrix(CKPT_F8_E4M3, 1ll << 24, 16384);
    REFUSED(ckpt_gated_forward(&x, &wl, &wl, CKPT_GATE_SILU, nullptr, nullptr, &h, nullptr, 0, nullptr));      // 2^23 tiles of 256 tokens
}

}  // namespace

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "refusals") refusals();
    else if (what == "grids") products_beyond_a_grid();
    else if (what == "blocks") tiles_of_blocks();
    else return 2;
    printf("ok\n");
}
