// The host side of the training operators on a HIP runtime of this file's own: two devices, allocations by decree (nothing is behind their addresses), a record of every call and launch.
// The sources are compiled for the host alone, so a launch comes here with its grid and its arguments.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/ckpt.h"
#include "../../include/ckpt_train.h"
#include "../../paper_2406_10707_amd/csrc/mx_gemm_loader.hpp"

namespace dsllm { thread_local std::string g_last_error; }

static int current;                              // device
static std::vector<std::string> calls;           // what was called, with the device that was current
struct Allocation { uint64_t base, bytes; int device; };
static std::vector<Allocation> allocations;
struct Launch { std::string kernel; dim3 grid, block; std::vector<unsigned char> first; };
static std::vector<Launch> launches;
static size_t first_argument_bytes;              // of a launch, to be kept

static void note(const char *what) { calls.push_back(std::string(what) + " on " + std::to_string(current)); }
static const Allocation *allocation_of(const void *p) {
    for (const Allocation &a : allocations)
        if (uint64_t(p) >= a.base && uint64_t(p) < a.base + a.bytes) return &a;
    return nullptr;
}

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
static std::vector<std::pair<const void *, std::string>> &kernels() { static std::vector<std::pair<const void *, std::string>> k; return k; }
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *, int *) { kernels().push_back({host, name}); }
void __hipRegisterVar(void **, void *, char *, const char *, int, size_t, int, int) {}
static dim3 pushed_grid, pushed_block;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) { pushed_grid = grid; pushed_block = block; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) { *grid = pushed_grid; *block = pushed_block; *lds = 0; *stream = nullptr; return hipSuccess; }
static hipError_t last_error = hipSuccess;
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t, hipStream_t) {
    // as the runtime does: fewer than 2^32 work-items along each axis
    if (!grid.x || !grid.y || uint64_t(grid.x) * block.x >> 32 || uint64_t(grid.y) * block.y >> 32 || grid.y > 65535) return last_error = hipErrorInvalidConfiguration;
    std::string name = "?";
    for (const auto &k : kernels()) if (k.first == f) name = k.second;
    const unsigned char *a = static_cast<unsigned char *>(args[0]);
    launches.push_back({name, grid, block, std::vector<unsigned char>(a, a + first_argument_bytes)});
    return hipSuccess;
}
hipError_t hipGetLastError() { const hipError_t e = last_error; last_error = hipSuccess; return e; }
const char *hipGetErrorString(hipError_t e) { return e == hipSuccess ? "no error" : "an error"; }
hipError_t hipGetDevice(int *d) { *d = current; return hipSuccess; }
hipError_t hipSetDevice(int d) { current = d; return hipSuccess; }
hipError_t hipDeviceSynchronize() { note("wait"); return hipSuccess; }
hipError_t hipMalloc(void **p, size_t) { *p = malloc(16); note("malloc"); return hipSuccess; }
hipError_t hipFree(void *p) { free(p); note("free"); return hipSuccess; }
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { note("copy"); return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *a, const void *p) {
    const Allocation *of = allocation_of(p);
    if (!of) return hipErrorInvalidValue;
    a->type = hipMemoryTypeDevice;
    a->device = of->device;
    return hipSuccess;
}
hipError_t hipMemGetAddressRange(hipDeviceptr_t *base, size_t *size, hipDeviceptr_t p) {
    const Allocation *of = allocation_of(p);
    if (!of) return hipErrorInvalidValue;
    *base = reinterpret_cast<hipDeviceptr_t>(of->base);
    *size = of->bytes;
    return hipSuccess;
}
}

static void *allocate(uint64_t bytes, int device = 0) {
    static uint64_t next = 1ull << 44;
    allocations.push_back({next, bytes, device});
    next += (bytes + (1ull << 21)) >> 21 << 21;
    return reinterpret_cast<void *>(allocations.back().base);
}

#define REQUIRE(x) do { if (!(x)) { printf("%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, dsllm::g_last_error.c_str()); exit(1); } } while (0)

// A handle is destroyed on the device it belongs to, and the caller's stays current.
static void destroy_on_another_device() {
    current = 1;
    ckpt_optim_tensor t{};
    t.numel = 100;
    t.dev_grad = allocate(400, 1);
    const ckpt_optim_config cfg{CKPT_F32, 0, 32, 0};
    ckpt_optim *o = nullptr;
    REQUIRE(ckpt_optim_create(&t, 1, &cfg, &o) == CKPT_OK);
    current = 0;
    calls.clear();
    REQUIRE(ckpt_optim_destroy(o) == CKPT_OK && current == 0);
    REQUIRE(calls.size() == 5 && calls[0] == "wait on 1");
    for (size_t i = 1; i < calls.size(); i++) REQUIRE(calls[i] == "free on 1");
}

// Every element of C is some launch's, once, and every launch reads the rows of A and B that go with its part: products of more rows or columns than one grid has places for.
static void sizes_beyond_a_grid() {
    struct { int64_t m, n, k; } sizes[] = {{1, (1ll << 29) + 5, 256}, {16, (1ll << 28) + 77, 8192}, {1, (1ll << 31) - 1, 100}, {5000000, 3, 0}, {17, (1ll << 30) + 9, 0}, {(1ll << 31) - 1, 1, 0},
                   {5000000, 70, 1ll << 25}, {3, 5, 0}, {40, 40, 1ll << 25}};
    for (const auto &s : sizes)
        for (int dtype : {int(CKPT_BF16), int(CKPT_F32)}) {
            const uint64_t size = dtype == CKPT_F32 ? 4 : 2;
            ckpt_mx_matrix a, b;
            REQUIRE(ckpt_mx_layout(CKPT_MXFP4, s.m, s.k, &a) == CKPT_OK && ckpt_mx_layout(CKPT_MXFP4, s.n, s.k, &b) == CKPT_OK);
            for (ckpt_mx_matrix *x : {&a, &b})
                if (s.k) {
                    x->codes = allocate(x->rows * x->code_pitch);
                    x->scales = allocate(x->rows * x->scale_pitch);
                }
            const int64_t ldc = s.n + 3;
            unsigned char *c = static_cast<unsigned char *>(allocate((s.m * ldc) * size));
            launches.clear();
            first_argument_bytes = sizeof(dsllm::GemmArgs);
            const int rc = ckpt_mx_gemm(&a, &b, c, dtype, ldc, 0, nullptr, 0, nullptr);
            printf("# %lld x %lld x %lld, %llu bytes an element: %d, %zu launches\n", (long long)s.m, (long long)s.n, (long long)s.k, (unsigned long long)size, rc, launches.size());
            REQUIRE(rc == CKPT_OK && !launches.empty());
            uint64_t covered = 0;
            std::vector<std::pair<uint64_t, std::pair<int64_t, int64_t>>> places;
            for (const Launch &l : launches) {
                dsllm::GemmArgs p;
                memcpy(&p, l.first.data(), sizeof p);
                const uint64_t at = (static_cast<unsigned char *>(p.c) - c) / size, row = at / ldc, col = at % ldc;
                REQUIRE(p.m > 0 && p.n > 0 && int64_t(row) + p.m <= s.m && int64_t(col) + p.n <= s.n && p.ldc == ldc);
                REQUIRE(p.a == static_cast<uint8_t *>(a.codes) + row * a.code_pitch && p.a_scale == static_cast<uint8_t *>(a.scales) + row * a.scale_pitch);
                REQUIRE(p.b == static_cast<uint8_t *>(b.codes) + col * b.code_pitch && p.b_scale == static_cast<uint8_t *>(b.scales) + col * b.scale_pitch);
                for (const auto &q : places) REQUIRE(q.first != at);
                places.push_back({at, {p.m, p.n}});
                covered += uint64_t(p.m) * p.n;
                if (l.kernel.find("few") != std::string::npos) REQUIRE(l.grid.x == uint64_t(p.n + 15) / 16 && l.grid.y == 1);
                else if (l.kernel.find("long") != std::string::npos) REQUIRE(l.grid.x == uint64_t(p.n + 63) / 64 && l.grid.y == uint64_t(p.m + 63) / 64);
                else REQUIRE(launches.size() == 1);
            }
            REQUIRE(covered == uint64_t(s.m) * s.n);
            allocations.clear();
        }
}

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "destroy") destroy_on_another_device();
    else if (what == "grids") sizes_beyond_a_grid();
    else return 2;
    printf("ok\n");
}
