// The host side of the training operators on a HIP runtime of this file's own: two devices, allocations by decree (nothing is behind their addresses), a record of every call and launch.
// The sources are compiled for the host alone, so a launch comes here with its grid and its arguments.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/ckpt.h"
#include "../../include/ckpt_train.h"

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
char __hip_fatbin[1], __hip_fatbin_optim[1];
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

int main(int argc, char **argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "destroy") destroy_on_another_device();
    else return 2;
    printf("ok\n");
}
