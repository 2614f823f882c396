// Exercises launches of layers (ms_runtime.cpp) on the CPU, under -fsanitize=thread: the HIP calls are replaced by a bookkeeping of which
// device holds which module, the compiler by an empty code object.  What it checks is which kernel a call launches, with how many
// workgroups, from several threads and on several devices at once.  Exit status 0 = every check held.
#include "../../paper_2205_13603_amd/csrc/ms_internal.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <memory>
#include <mutex>
#include <set>
#include <string>
#include <thread>

#define CHECK(x)                                                               \
    do {                                                                       \
        if (!(x)) {                                                            \
            fprintf(stderr, "%s:%d: CHECK failed: %s (last error: %s)\n", __FILE__, __LINE__, #x, ms_last_error()); \
            exit(1);                                                           \
        }                                                                      \
    } while (0)

static thread_local int t_device;
static thread_local unsigned t_grid[2];
static std::mutex g_mu;
static std::set<std::pair<void *, int>> g_modules; // and the device each is on
static std::atomic<int> g_loaded, g_launched;
static char g_workspace[256];

namespace ms {
int32_t jit_get_code(const KernelSpec &, uint64_t key, std::vector<char> **out)
{
    static std::map<uint64_t, std::unique_ptr<std::vector<char>>> codes;
    std::lock_guard<std::mutex> lk(g_mu);
    auto &c = codes[key];
    if (!c) c.reset(new std::vector<char>(16));
    *out = c.get();
    return MS_OK;
}
} // namespace ms

extern "C" {
hipError_t hipGetDevice(int *d) { return *d = t_device, hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t *p, int d)
{
    memset(p, 0, sizeof *p);
    strcpy(p->gcnArchName, d == 2 ? "gfx942" : "gfx950");
    p->sharedMemPerBlock = 160 << 10;
    p->multiProcessorCount = d ? 64 : 256;
    return hipSuccess;
}
hipError_t hipModuleLoadData(hipModule_t *m, const void *)
{
    *m = (hipModule_t)malloc(1);
    std::lock_guard<std::mutex> lk(g_mu);
    g_modules.insert({*m, t_device});
    ++g_loaded;
    return hipSuccess;
}
hipError_t hipModuleUnload(hipModule_t) { CHECK(!"a layer's kernel stays"); return hipSuccess; }
hipError_t hipModuleGetFunction(hipFunction_t *f, hipModule_t m, const char *) { return *f = (hipFunction_t)m, hipSuccess; }
hipError_t hipModuleLaunchKernel(hipFunction_t f, unsigned x, unsigned y, unsigned z, unsigned, unsigned, unsigned, unsigned, hipStream_t, void **, void **)
{
    std::lock_guard<std::mutex> lk(g_mu);
    CHECK(g_modules.count({(void *)f, t_device}) && z == 1); // a kernel of a module that is loaded on this device
    t_grid[0] = x;
    t_grid[1] = y;
    ++g_launched;
    return hipSuccess;
}
hipError_t hipGetSymbolAddress(void **p, const void *) { return *p = g_workspace, hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *) { return hipErrorUnknown; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipErrorUnknown; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipErrorUnknown; }
hipError_t hipEventElapsedTime(float *, hipEvent_t, hipEvent_t) { return hipErrorUnknown; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipErrorUnknown; }
hipError_t hipGetLastError(void) { return hipErrorUnknown; }
hipError_t hipDeviceGetAttribute(int *, hipDeviceAttribute_t, int) { return hipErrorUnknown; }
const char *hipGetErrorString(hipError_t) { return "stub"; }
}

static ms_variant *build(int32_t kind, int32_t in, int32_t out, std::vector<int32_t> dims, int64_t code)
{
    ms_op_desc d = {};
    d.kind = kind;
    d.in_dtype = in;
    d.out_dtype = out;
    for (size_t i = 0; i < dims.size(); ++i) d.dims[i] = dims[i];
    ms_op *op = nullptr;
    ms_space space;
    ms_trace t;
    ms_variant *v = nullptr;
    CHECK(ms_op_create(&d, &op) == MS_OK && ms_space_describe(op, MS_SPACE_DEFAULT, &space) == MS_OK && ms_trace_default(&space, &t) == MS_OK);
    const ms_slot &s = space.slots[0];
    for (int i = 0; i < s.n_candidates; ++i)
        if (s.candidates[i] == code) t.d[0].v[0] = i;
    CHECK(ms_variant_build(op, &space, &t, &v) == MS_OK);
    ms_op_destroy(op);
    return v;
}

int main()
{
    static char memory[64] __attribute__((aligned(64)));
    const void *in[5] = {memory, memory, memory, memory, memory};
    void *out[3] = {memory, memory, memory};

    // two threads launch one variant on two devices at once: each runs its own device's kernel, loaded once
    ms_variant *v = build(MS_OP_GROUPED_GEMM, MS_BF16, MS_BF16, {4, 1000, 512, 256}, 128128);
    CHECK(ms_variant_launch_static(v, in, out, 1, nullptr) == MS_ERR_BAD_ARG && g_launched == 0); // not loaded yet
    auto run = [&](int device) {
        t_device = device;
        for (int i = 0; i < 3000; ++i) CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_OK);
    };
    std::thread a(run, 0), b(run, 1);
    a.join();
    b.join();
    CHECK(g_loaded == 2 && g_launched == 6000);
    // and one thread in turn, also without what would load
    for (int i = 0; i < 6; ++i) {
        t_device = i % 2;
        CHECK(ms_variant_launch_static(v, in, out, 1, nullptr) == MS_OK);
    }
    CHECK(g_loaded == 2);
    // operators of other sizes on the same kernel load nothing, and outlive its first variant
    ms_variant *w = build(MS_OP_GROUPED_GEMM, MS_BF16, MS_BF16, {4, 1001, 520, 264}, 128128);
    ms_variant_destroy(v);
    t_device = 0;
    CHECK(ms_variant_launch(w, in, out, nullptr, 1, nullptr) == MS_OK && g_loaded == 2);
    t_device = 2;
    CHECK(ms_variant_launch(w, in, out, nullptr, 1, nullptr) == MS_ERR_UNSUPPORTED && ms_variant_prepare(w) == MS_ERR_UNSUPPORTED);
    t_device = 0;
    ms_variant_destroy(w);

    // grids: persistent workgroups, at most one a compute unit of the device and four a tile; instances along y
    ms_variant *p = build(MS_OP_SCALED_GEMM, MS_F8E4M3, MS_BF16, {4096, 4096, 512}, 256256), *one = build(MS_OP_SCALED_GEMM, MS_F8E4M3, MS_BF16, {16, 4096, 512}, 256256);
    CHECK(ms_variant_launch(p, in, out, nullptr, 3, nullptr) == MS_OK && t_grid[0] == 256 && t_grid[1] == 3);
    CHECK(ms_variant_launch(one, in, out, nullptr, 1, nullptr) == MS_OK && t_grid[0] == 64);
    t_device = 1;
    CHECK(ms_variant_launch(p, in, out, nullptr, 1, nullptr) == MS_OK && t_grid[0] == 64);
    t_device = 0;
    CHECK(ms_variant_launch(p, in, out, nullptr, 65536, nullptr) == MS_ERR_BAD_ARG);
    ms_variant *n = build(MS_OP_RMS_NORM, MS_BF16, MS_F8E4M3, {1000, 512, 1}, 1);
    CHECK(ms_variant_launch(n, in, out, nullptr, 1, nullptr) == MS_OK && t_grid[0] == 250 && t_grid[1] == 1);
    CHECK(ms_variant_launch(n, in, out, nullptr, 100000, nullptr) == MS_ERR_BAD_ARG || t_grid[0] == 1 << 20); // workgroups go on to further rows

    // tensors that are not there or lie off their alignment
    const int launched = g_launched;
    for (int i = 0; i < 4; ++i) {
        const void *bad[5] = {memory, memory, memory, memory, memory};
        bad[i] = nullptr;
        CHECK(ms_variant_launch(p, bad, out, nullptr, 1, nullptr) == MS_ERR_BAD_ARG);
        bad[i] = memory + 2;
        CHECK(ms_variant_launch(p, bad, out, nullptr, 1, nullptr) == MS_ERR_BAD_ARG);
    }
    for (int i = 0; i < 2; ++i) {
        void *bad[3] = {memory, memory, nullptr};
        bad[i] = nullptr;
        CHECK(ms_variant_launch(n, in, bad, nullptr, 1, nullptr) == MS_ERR_BAD_ARG);
    }
    CHECK(g_launched == launched);
    ms_variant_destroy(p);
    ms_variant_destroy(one);
    ms_variant_destroy(n);
    printf("layer checks ok\n");
    return 0;
}
