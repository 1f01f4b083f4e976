// What a call writes may share no byte with anything else that it reads or writes, codes, scales, plain matrices and workspace alike: on the runtime of train_calls.cpp, each is moved onto the last bytes of every other
// one, which is refused before anything is launched, and right behind them, which is not. Rows that lie between another's rows share nothing.
#define main main_of_train_calls
#include "train_calls.cpp"
#undef main

#include <functional>
#include <random>

#include "../../paper_2406_10707_amd/csrc/f8_forms.hpp"
#include "../../paper_2406_10707_amd/csrc/f8_util.hpp"

#define TAKEN(call) do { launches.clear(); REQUIRE((call) == CKPT_OK); REQUIRE(!launches.empty()); } while (0)
#define OVERLAPS(call) do { launches.clear(); dsllm::g_last_error.clear(); REQUIRE((call) == CKPT_EINVAL); REQUIRE(launches.empty() && dsllm::g_last_error.find("overlap") != std::string::npos); } while (0)

namespace {

struct Piece { uint64_t bytes, aligned; bool written; };
void add(std::vector<Piece> &pieces, const ckpt_f8_matrix &m, bool written) {
    pieces.push_back({uint64_t(m.rows - 1) * m.code_pitch + (uint64_t(m.cols) + 127) / 128 * 128, 16, written});
    pieces.push_back({4 * (((uint64_t(m.cols) + 127) / 128 - 1) * m.scale_pitch + (uint64_t(m.rows) + m.block_rows - 1) / m.block_rows), 4, written});
}
ckpt_f8_matrix shape(int32_t format, int64_t rows, int64_t cols, int32_t block_rows = 1) {
    ckpt_f8_matrix m;
    REQUIRE(ckpt_f8_layout(format, block_rows, rows, cols, &m) == CKPT_OK);
    return m;
}

ckpt_f8_matrix matrix(int64_t rows, int64_t cols) {
    ckpt_f8_matrix m = shape(CKPT_F8_E4M3, rows, cols);
    m.codes = allocate(uint64_t(rows) * m.code_pitch);
    m.scales = static_cast<float *>(allocate(4 * (m.code_pitch / 128) * m.scale_pitch));
    return m;
}
template <class F>
ckpt_f8_matrix but(ckpt_f8_matrix m, F change) {
    change(m);
    return m;
}

// `call` is given the address of every piece.
void every_pair(const char *name, const std::vector<Piece> &pieces, const std::function<int(const std::vector<uint64_t> &)> &call) {
    uint64_t most = 0;
    for (const Piece &p : pieces) most = std::max(most, p.bytes);
    const uint64_t apart = (3 * most + 4095) / 4096 * 4096, room = uint64_t(allocate(apart * pieces.size()));
    std::vector<uint64_t> apart_all;
    for (size_t i = 0; i < pieces.size(); i++) apart_all.push_back(room + apart * i);
    TAKEN(call(apart_all));
    for (size_t i = 0; i < pieces.size(); i++)
        for (size_t k = 0; k < pieces.size(); k++) {
            if (i == k || !(pieces[i].written || pieces[k].written)) continue;
            std::vector<uint64_t> at = apart_all;
            const uint64_t end = apart_all[k] + pieces[k].bytes;
            printf("# %s: %zu on %zu\n", name, i, k);
            at[i] = (end - 1) / pieces[i].aligned * pieces[i].aligned;
            OVERLAPS(call(at));
            at[i] = (end + pieces[i].aligned - 1) / pieces[i].aligned * pieces[i].aligned;
            TAKEN(call(at));
        }
    allocations.clear();
}

ckpt_f8_matrix placed(ckpt_f8_matrix m, const std::vector<uint64_t> &at, size_t &next) {
    m.codes = reinterpret_cast<void *>(at[next++]);
    m.scales = reinterpret_cast<float *>(at[next++]);
    return m;
}

void every_call() {
    for (int32_t block_rows : {1, 128}) {
        const ckpt_f8_matrix by_row = shape(CKPT_F8_E4M3, 300, 200, block_rows), by_col = shape(CKPT_F8_E4M3, 200, 300, block_rows);
        std::vector<Piece> pieces{{(299 * 210 + 200) * 2, 2, false}};
        add(pieces, by_row, true);
        add(pieces, by_col, true);
        every_pair("quantize", pieces, [&](const std::vector<uint64_t> &at) {
            size_t next = 1;
            const auto r = placed(by_row, at, next), c = placed(by_col, at, next);
            return ckpt_f8_quantize(reinterpret_cast<void *>(at[0]), CKPT_BF16, 210, &r, &c, nullptr);
        });
        pieces.clear();
        add(pieces, by_row, false);
        add(pieces, by_col, true);
        every_pair("columns", pieces, [&](const std::vector<uint64_t> &at) {
            size_t next = 0;
            const auto r = placed(by_row, at, next), c = placed(by_col, at, next);
            return ckpt_f8_columns(&r, &c, nullptr);
        });
        pieces = {{(299 * 210 + 200) * 4, 4, true}};
        add(pieces, by_row, false);
        every_pair("dequantize", pieces, [&](const std::vector<uint64_t> &at) {
            size_t next = 1;
            const auto r = placed(by_row, at, next);
            return ckpt_f8_dequantize(&r, reinterpret_cast<void *>(at[0]), CKPT_F32, 210, nullptr);
        });
    }
    for (int64_t m : {3, 64}) {      // unsplit, and in parts
        const ckpt_f8_matrix a = shape(CKPT_F8_E4M3, m, 16384), b = shape(CKPT_F8_E4M3, 64, 16384, 128);
        uint64_t bytes;
        REQUIRE(ckpt_f8_gemm_workspace(m, 64, 16384, &bytes) == CKPT_OK && (m == 3) == (bytes == 0));
        if (bytes) bytes = dsllm::f8_part_bytes(m, 64) * dsllm::f8_choice(m, 64, 16384, true, false, bytes).splits;      // what this product takes of it
        std::vector<Piece> pieces{{(uint64_t(m - 1) * 70 + 64) * 4, 4, true}};
        if (bytes) pieces.push_back({bytes, 16, true});
        add(pieces, a, false);
        add(pieces, b, false);
        every_pair("product", pieces, [&](const std::vector<uint64_t> &at) {
            size_t next = bytes ? 2 : 1;
            const auto x = placed(a, at, next), y = placed(b, at, next);
            return ckpt_f8_gemm(&x, &y, reinterpret_cast<void *>(at[0]), CKPT_F32, 70, 1, bytes ? reinterpret_cast<void *>(at[1]) : nullptr, bytes, nullptr);
        });
    }
    for (int64_t tokens : {3, 40, 300}) {
        const int64_t ffn = tokens == 40 ? 4100 : 300;
        const ckpt_f8_matrix x = shape(CKPT_F8_E5M2, tokens, 200), w = shape(CKPT_F8_E4M3, ffn, 200, 128), kept = shape(CKPT_F8_E4M3, tokens, ffn);
        uint64_t bytes;
        REQUIRE(ckpt_gated_workspace(tokens, ffn, 200, &bytes) == CKPT_OK && (tokens == 300) == (bytes == 0));
        std::vector<Piece> pieces;
        if (bytes) pieces.push_back({bytes, 16, true});
        for (int i = 0; i < 6; i++) add(pieces, i == 0 ? x : i < 3 ? w : kept, i >= 3);
        every_pair("forward", pieces, [&](const std::vector<uint64_t> &at) {
            size_t next = bytes ? 1 : 0;
            const auto mx = placed(x, at, next), wg = placed(w, at, next), wu = placed(w, at, next), gate = placed(kept, at, next), up = placed(kept, at, next), h = placed(kept, at, next);
            return ckpt_gated_forward(&mx, &wg, &wu, CKPT_GATE_GELU, &gate, &up, &h, bytes ? reinterpret_cast<void *>(at[0]) : nullptr, bytes, nullptr);
        });
    }
    const ckpt_f8_matrix dy = shape(CKPT_F8_E5M2, 200, 200), wd = shape(CKPT_F8_E4M3, 300, 200, 128), kept = shape(CKPT_F8_E4M3, 200, 300), grad = shape(CKPT_F8_E5M2, 200, 300), grad_by_col = shape(CKPT_F8_E5M2, 300, 200),
                         h_by_col = shape(CKPT_F8_E4M3, 300, 200);
    std::vector<Piece> pieces;
    for (const auto *m : {&dy, &wd, &kept, &kept}) add(pieces, *m, false);
    for (const auto *m : {&grad, &grad, &grad_by_col, &grad_by_col, &h_by_col}) add(pieces, *m, true);
    every_pair("backward", pieces, [&](const std::vector<uint64_t> &at) {
        size_t next = 0;
        const auto d = placed(dy, at, next), w = placed(wd, at, next), gate = placed(kept, at, next), up = placed(kept, at, next), dgate = placed(grad, at, next), dup = placed(grad, at, next), dgate_c = placed(grad_by_col, at, next),
                   dup_c = placed(grad_by_col, at, next), h_c = placed(h_by_col, at, next);
        const ckpt_gated_grads grads{&dgate, &dup, &dgate_c, &dup_c, &h_c};
        return ckpt_gated_backward(&d, &w, &gate, &up, CKPT_GATE_SILU, &grads, nullptr);
    });
}

// Rows between one another's rows: taken, and refused as soon as one byte is shared.
void between_rows() {
    const auto x = matrix(300, 200), wg = matrix(300, 200), wu = matrix(300, 200), gate = matrix(300, 300), up = matrix(300, 300), h = matrix(300, 300);
    auto forward = [&](const ckpt_f8_matrix &gate, const ckpt_f8_matrix &up) { return ckpt_gated_forward(&x, &wg, &wu, CKPT_GATE_SILU, &gate, &up, &h, nullptr, 0, nullptr); };
    float *scales = static_cast<float *>(allocate(4 * 10000));
    auto with_scales = [&](const ckpt_f8_matrix &m, int64_t first, uint64_t pitch) { return but(m, [&](auto &v) { v.scales = scales + first; v.scale_pitch = pitch; }); };
    TAKEN(forward(with_scales(gate, 0, 600), with_scales(up, 300, 600)));
    TAKEN(forward(with_scales(gate, 300, 600), with_scales(up, 0, 600)));
    OVERLAPS(forward(with_scales(gate, 0, 600), with_scales(up, 299, 600)));
    OVERLAPS(forward(with_scales(gate, 0, 600), with_scales(up, 301, 600)));
    TAKEN(forward(with_scales(gate, 0, 2000), with_scales(up, 300, 700)));         // [0, 300) [2000, 2300) [4000, 4300) and [300, 600) [1000, 1300) [1700, 2000)
    OVERLAPS(forward(with_scales(gate, 0, 2000), with_scales(up, 301, 700)));
    OVERLAPS(forward(with_scales(gate, 0, 2000), with_scales(up, 299, 700)));
    char *codes = static_cast<char *>(allocate(300 * 2048));
    auto with_codes = [&](const ckpt_f8_matrix &m, int64_t first, uint64_t pitch) { return but(m, [&](auto &v) { v.codes = codes + first; v.code_pitch = pitch; }); };
    TAKEN(forward(with_codes(gate, 0, 1024), with_codes(up, 384, 1024)));
    TAKEN(forward(with_codes(gate, 0, 1024), with_codes(up, 384, 2048)));          // every second gap
    OVERLAPS(forward(with_codes(gate, 0, 1024), with_codes(up, 384 - 16, 2048)));
    OVERLAPS(forward(with_codes(gate, 0, 1024), with_codes(up, 640 + 16, 2048)));
    // scales in the gaps of the codes' rows: three rows of 1200 bytes behind codes of 384
    TAKEN(forward(but(with_codes(gate, 0, 2048), [&](auto &v) { v.scales = reinterpret_cast<float *>(codes + 384); v.scale_pitch = 512; }), up));
    OVERLAPS(forward(but(with_codes(gate, 0, 2048), [&](auto &v) { v.scales = reinterpret_cast<float *>(codes + 380); v.scale_pitch = 512; }), up));
    OVERLAPS(forward(but(with_codes(gate, 0, 2048), [&](auto &v) { v.scales = reinterpret_cast<float *>(codes + 384); v.scale_pitch = 500; }), up));
}

// Against bytes that are marked.
void marked() {
    std::mt19937 rng(1);
    auto up_to = [&](uint64_t n) { return rng() % n; };
    for (int turn = 0, met = 0; turn < 200000; turn++) {
        dsllm::Rows r[2];
        std::vector<unsigned char> seen(600);
        bool shared = false;
        for (int i = 0; i < 2; i++) {
            r[i].width = 1 + up_to(12);
            r[i].pitch = i && up_to(2) ? r[0].pitch : r[i].width + up_to(25);
            if (r[i].pitch < r[i].width) r[i].width = r[i].pitch;
            r[i].rows = 1 + up_to(10);
            r[i].at = up_to(200);
            for (uint64_t k = 0; k < r[i].rows; k++)
                for (uint64_t b = 0; b < r[i].width; b++) {
                    unsigned char &s = seen[r[i].at + k * r[i].pitch + b];
                    shared |= i && s;
                    s |= !i;
                }
        }
        REQUIRE(dsllm::share_bytes(r[0], r[1]) == shared && dsllm::share_bytes(r[1], r[0]) == shared);
        met += shared;
        REQUIRE(turn != 199999 || (met > 20000 && met < 180000));
    }
    // far more rows than are looked at one by one
    const dsllm::Rows a{1ull << 40, 128, 1 << 20, 1ull << 30}, b{(1ull << 40) + 128, 256, 1 << 20, 1ull << 30}, c{(1ull << 40) + 256, 256, 1 << 20, 1ull << 30}, far{(1ull << 40) + (1ull << 50), 16, 16, 1ull << 30};
    REQUIRE(!dsllm::share_bytes(a, b) && dsllm::share_bytes(b, c) && !dsllm::share_bytes(a, far));
}

}  // namespace

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "calls") every_call();
    else if (what == "rows") between_rows();
    else if (what == "marked") marked();
    else return 2;
    printf("ok\n");
}
