// Loads the built library without a GPU and prints the launches that the sequence
// operators make, as launch_drive.cpp does of the other calls: the HIP entry points
// below stand in for the runtime's, and refuse what the device does not take.  No
// pointer given to the library is dereferenced on the host.
// Usage: sequence_launch_drive LIB, then lines "OP TYPE B D L N G" on stdin, OP conv,
// conv_back, conv_step, scan, scan_back, scan_step, norm, norm8, norm_back (B rows of
// D) or dropout, N the taps or the states; per line one output line
// "rc;kernel,grid x,y,z,threads,lds;..." (the kernel's mangled name).
// Test infrastructure: built and run by tests/test_sequence_launches_cpu.py.
#include <dlfcn.h>
#include <hip/hip_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <map>
#include <string>

#include "finc.h"

static std::map<const void *, std::string> &names() {
    static std::map<const void *, std::string> m;
    return m;
}
static std::string launches;
static hipError_t last = hipSuccess;
static struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} pushed;

extern "C" {
void **__hipRegisterFatBinary(const void *) {
    static void *h;
    return &h;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *,
                           void *, dim3 *, dim3 *, int *) {
    names()[f] = name;
}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t st) {
    pushed = {g, b, lds, st};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, hipStream_t *st) {
    *g = pushed.grid;
    *b = pushed.block;
    *lds = pushed.lds;
    *st = pushed.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 g, dim3 b, void **, size_t lds, hipStream_t) {
    char s[512];
    snprintf(s, sizeof s, ";%s,%u,%u,%u,%u,%zu", names()[f].c_str(), g.x, g.y, g.z,
             b.x * b.y * b.z, lds);
    launches += s;
    // 2^32 threads in x and 2^16 workgroups in y or z are too many
    if ((unsigned long long)g.x * b.x >= 1ull << 32 || g.y >= 1u << 16 || g.z >= 1u << 16 ||
        !g.x || !g.y || !g.z)
        last = hipErrorInvalidConfiguration;
    return last;
}
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError(void) {
    const hipError_t e = last;
    last = hipSuccess;
    return e;
}
}

// Buffers far apart, none of them there.
static void *at(int i) { return (void *)((uintptr_t)(i + 1) << 52); }
static float *f32(int i) { return (float *)at(i); }
static finc_raster raster(int i, long long rows, long long L) { return {at(i), rows * L, L}; }

#define CALL(name) reinterpret_cast<decltype(&name)>(dlsym(lib, #name))

static int call(void *lib, const std::string &op, int type, int B, int D, int L, int N, int G) {
    if (op == "conv" || op == "conv_back") {
        finc_conv_args a = {type, B, D, L, N, 1, raster(0, D, L), raster(1, D, L), f32(2), f32(3),
                            nullptr, nullptr, nullptr};
        finc_conv_grads g = {raster(4, D, L), raster(5, D, L), f32(6), f32(7), nullptr, nullptr,
                             at(8)};
        return op == "conv" ? CALL(finc_causal_conv_forward)(&a, nullptr)
                            : CALL(finc_causal_conv_backward)(&a, &g, nullptr);
    }
    if (op == "conv_step")
        return CALL(finc_causal_conv_step)(type, at(0), D, at(1), D, f32(2), f32(3), at(4), nullptr,
                                           B, B, D, N, 1, nullptr);
    const long long GN = (long long)G * N;
    if (op == "scan" || op == "scan_back") {
        finc_scan_args a = {type, B, D, L, N, G, 1, raster(0, D, L), raster(1, D, L),
                            raster(2, D, L), raster(3, GN, L), raster(4, GN, L), raster(5, D, L),
                            f32(6), f32(7), f32(8), nullptr, nullptr, f32(9), nullptr};
        finc_scan_grads g = {raster(10, D, L), raster(11, D, L), raster(12, D, L), raster(13, D, L),
                             raster(14, GN, L), raster(15, GN, L), f32(16), f32(17), f32(18),
                             nullptr, nullptr, at(19)};
        return op == "scan" ? CALL(finc_selective_scan_forward)(&a, nullptr)
                            : CALL(finc_selective_scan_backward)(&a, &g, nullptr);
    }
    if (op == "scan_step") {
        finc_scan_step_args a = {type, B, B, D, N, G, 1, at(0), at(1), at(2), at(3), at(4), D, D, D,
                                 GN, GN, D, at(5), f32(6), f32(7), f32(8), f32(9), nullptr};
        return CALL(finc_selective_scan_step)(&a, nullptr);
    }
    if (op == "norm" || op == "norm8") {
        finc_norm_args a = {type, type, B, D, at(0), at(1), at(2), at(3), D, D, D, D, f32(4),
                            op == "norm8" ? f32(5) : nullptr, 1e-5, 0.1, 1, 2};
        return CALL(finc_add_norm_forward)(&a, nullptr);
    }
    if (op == "norm_back") {
        finc_norm_grad_args a = {type, type, B, D, at(0), at(1), at(2), at(3), at(4), D, D, D, D, D,
                                 f32(5), f32(6), 1e-5, 0.1, 1, 2, at(7)};
        return CALL(finc_add_norm_backward)(&a, nullptr);
    }
    if (op == "dropout")
        return CALL(finc_dropout)(type, at(0), D, at(1), D, at(2), D, B, D, 0.1, 1, 2, nullptr);
    return -1000;
}

int main(int argc, char **argv) {
    void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib || names().empty()) {
        fprintf(stderr, "%s\n", argc > 1 ? dlerror() : "no library named");
        return 2;
    }
    char op[32];
    int type, B, D, L, N, G;
    while (scanf("%31s %d %d %d %d %d %d", op, &type, &B, &D, &L, &N, &G) == 7) {
        launches.clear();
        last = hipSuccess;
        const int rc = call(lib, op, type, B, D, L, N, G);
        printf("%d%s\n", rc, launches.c_str());
    }
    return 0;
}
