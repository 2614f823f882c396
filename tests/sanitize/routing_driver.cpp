// Exercises launches of routing's operators (ms_runtime.cpp, ms_routing.h) on the CPU: the HIP calls are replaced by a bookkeeping of what was
// launched with which arguments, the compiler by an empty code object.  Exit status 0 = every check held.
#include "../../paper_2205_13603_amd/csrc/ms_internal.h"
#include "../../paper_2205_13603_amd/csrc/ms_routing.h"

#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <memory>
#include <string>

#define CHECK(x)                                                               \
    do {                                                                       \
        if (!(x)) {                                                            \
            fprintf(stderr, "%s:%d: CHECK failed: %s (last error: %s)\n", __FILE__, __LINE__, #x, ms_last_error()); \
            exit(1);                                                           \
        }                                                                      \
    } while (0)

struct launch_t {
    std::string kernel;
    unsigned x, y, threads;
    unsigned char args[160];
};
static std::vector<launch_t> g_launches;
static char g_workspace[256];
static std::vector<char *> g_handles;

namespace ms {
int32_t jit_get_code(const KernelSpec &, uint64_t key, std::vector<char> **out)
{
    static std::map<uint64_t, std::unique_ptr<std::vector<char>>> codes;
    auto &c = codes[key];
    if (!c) c.reset(new std::vector<char>(16));
    *out = c.get();
    return MS_OK;
}
} // namespace ms

extern "C" {
hipError_t hipGetDevice(int *d) { return *d = 0, hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t *p, int)
{
    memset(p, 0, sizeof *p);
    strcpy(p->gcnArchName, "gfx950");
    p->sharedMemPerBlock = 160 << 10;
    p->multiProcessorCount = 256;
    return hipSuccess;
}
hipError_t hipModuleLoadData(hipModule_t *m, const void *) { return *m = (hipModule_t)g_workspace, hipSuccess; }
hipError_t hipModuleUnload(hipModule_t) { return hipSuccess; }
hipError_t hipModuleGetFunction(hipFunction_t *f, hipModule_t, const char *name)
{
    g_handles.push_back(strdup(name));
    return *f = (hipFunction_t)g_handles.back(), hipSuccess;
}
hipError_t hipModuleLaunchKernel(hipFunction_t f, unsigned x, unsigned y, unsigned z, unsigned bx, unsigned by, unsigned bz, unsigned lds, hipStream_t, void **args, void **)
{
    CHECK(z == 1 && by == 1 && bz == 1 && lds == 0);
    launch_t l = {(const char *)f, x, y, bx, {}};
    // the largest of the argument structs is read by its own type below: copy what the smallest has for sure
    memcpy(l.args, args[0], sizeof(ms::OrderArgs));
    g_launches.push_back(l);
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

static ms_variant *build(int32_t kind, int32_t in, int32_t out, std::vector<int64_t> dims, int64_t code = 0, int32_t bias = 0)
{
    ms_op_desc d = {};
    d.kind = kind;
    d.in_dtype = in;
    d.out_dtype = out;
    d.has_bias = bias;
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
    static char a[64] __attribute__((aligned(64))), b[64] __attribute__((aligned(64))), c[64] __attribute__((aligned(64)));
    const void *in[4] = {a, a, a, a};
    void *out[2] = {b, c};

    // a few choices: one kernel of one workgroup, no workspace
    ms_variant *v = build(MS_OP_EXPERT_ORDER, MS_I32, MS_I32, {32, 2, 8});
    CHECK(ms_variant_launch(v, in, out, nullptr, 3, nullptr) == MS_OK && g_launches.size() == 1);
    CHECK(g_launches[0].kernel == "ms_kernel" && g_launches[0].x == 1 && g_launches[0].y == 3 && g_launches[0].threads == 64);
    ms_variant_destroy(v);

    // many: the runs are counted first, by as many workgroups, in the caller's workspace or the built-in one
    g_launches.clear();
    v = build(MS_OP_EXPERT_ORDER, MS_I32, MS_I32, {300, 5000, 8}, 2);
    size_t need = 0;
    ms_variant_params p;
    CHECK(ms_variant_info(v, &p, &need) == MS_OK && p.grid[0] == 20 && need == 20 * 300 * 4);
    CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_ERR_BAD_ARG && ms_variant_launch(v, in, out, a + 8, 1, nullptr) == MS_ERR_BAD_ARG && g_launches.empty());
    CHECK(ms_variant_launch_static(v, in, out, 1, nullptr) == MS_ERR_BAD_ARG && g_launches.empty()); // not prepared
    CHECK(ms_variant_launch(v, in, out, a, 2, nullptr) == MS_OK && g_launches.size() == 2);
    CHECK(g_launches[0].kernel == "ms_count" && g_launches[1].kernel == "ms_kernel");
    for (const launch_t &l : g_launches) {
        ms::OrderArgs g;
        memcpy(&g, l.args, sizeof g);
        CHECK(l.x == 20 && l.y == 2 && l.threads == 1024 && g.counts == a && g.total == 40000 && g.experts == 300 && g.runs == 20);
    }
    CHECK(ms_variant_prepare(v) == MS_OK && ms_variant_launch_static(v, in, out, 1, nullptr) == MS_OK && g_launches.size() == 4);
    ms::OrderArgs g;
    memcpy(&g, g_launches[3].args, sizeof g);
    CHECK(g.counts == g_workspace);
    CHECK(ms_variant_launch_static(v, in, out, 3000, nullptr) == MS_ERR_BAD_ARG); // 72 MB
    ms_variant_destroy(v);

    // a workgroup for so many tokens
    g_launches.clear();
    v = build(MS_OP_ROUTE, MS_F32, MS_F32, {100, 256, 8, 8, 4, 2, 3, 0}, 16, 1);
    CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_OK && g_launches[0].x == 7 && g_launches[0].threads == 256);
    in[1] = nullptr;
    CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_ERR_BAD_ARG);
    ms_variant_destroy(v);
    v = build(MS_OP_ROUTE, MS_F32, MS_F32, {100, 240, 8, 8, 4, 2, 3, 0}, 16); // groups of 30: by way of LDS
    CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_OK && g_launches[1].x == 25 && g_launches[1].threads == 64);
    ms_variant_destroy(v);
    v = build(MS_OP_JOIN_ROWS, MS_BF16, MS_BF16, {100, 4, 4096, 400, 0}, 8);
    in[1] = a;
    in[2] = in[3] = nullptr;
    CHECK(ms_variant_launch(v, in, out, nullptr, 65535, nullptr) == MS_OK && g_launches[2].x == 100 && g_launches[2].y == 65535 && g_launches[2].threads == 512);
    ms_variant_destroy(v);
    v = build(MS_OP_SPREAD_ROWS, MS_BF16, MS_I8, {100, 1, 4096, 100}, 1);
    in[1] = nullptr;
    CHECK(ms_variant_launch(v, in, out, nullptr, 1, nullptr) == MS_OK && g_launches[3].x == 25);
    ms_variant_destroy(v);
    for (char *h : g_handles) free(h);
    printf("routing checks ok\n");
    return 0;
}
