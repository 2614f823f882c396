// Choices sorted by expert, in their own order within each: where each expert's rows begin, and the row of each choice.
//
// A workgroup takes a run of choices, each of its wavefronts ROUNDS times 64 of them.  Lanes with the same expert find each other bit by bit
// (ballots); a lane's place among them is the number of those below it, and one of them adds theirs to the wavefront's count of the expert in LDS.  No
// atomic operation decides an order, so that the result is the same every time.
//
// More choices than one workgroup takes: a first kernel counts each run's experts (counts), and each workgroup adds up what lies ahead of its own.
//
// What bounds it is latency: 16 choices 4.5 us, the launch; 131072 choices of 256 experts 7.2, of which the second launch is 2; 524288 10.3, 2^20 12.4, 2^23 56.
// Beyond that it is the counts, of which each run reads those of all: 2^26 choices 1143 us for 0.5 GB of choices and places, 1024 experts 3458.
#include "common.h"

struct order_args {
    const int *ids;
    int *offsets, *place;
    int *counts; // [runs][experts] of each instance
    int total, experts, runs;
};

constexpr int WAVES = THREADS / 64, RUN = THREADS * ROUNDS, BITS = EXPERTS <= 64 ? 6 : EXPERTS <= 256 ? 8 : 10;
static_assert(EXPERTS <= 1 << BITS, "bits of an expert's index");

// LDS that only this wavefront uses: what its lanes have written is there for all of them.
__device__ __forceinline__ void wave_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// Sums over the lanes up to and including each: within rows of 16, over the rows of a half, over the halves.
__device__ __forceinline__ int sums_of_lanes(int n)
{
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xa, 0xf, false);
    return n + __builtin_amdgcn_update_dpp(0, n, 0x143, 0xc, 0xf, false);
}
// Choice n of the instance's; -1: none, or of no expert.
__device__ __forceinline__ int id_at(const order_args &g, const int *ids, int n)
{
    int id = -1;
    if (n < g.total) id = ids[n];
    return id >= 0 && id < g.experts ? id : -1;
}

#if MANY
extern "C" __global__ void __launch_bounds__(THREADS) ms_count(const order_args g)
{
    __shared__ int count[EXPERTS];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, inst = blockIdx.y;
    const int *ids = g.ids + (long)inst * g.total;
    for (int e = tid; e < EXPERTS; e += THREADS) count[e] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int id = id_at(g, ids, (int)blockIdx.x * RUN + (wave * ROUNDS + r) * 64 + lane);
        if (id >= 0) atomicAdd(&count[id], 1);
    }
    __syncthreads();
    int *to = g.counts + ((long)inst * g.runs + blockIdx.x) * g.experts;
    for (int e = tid; e < g.experts; e += THREADS) to[e] = count[e];
}
#endif

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const order_args g)
{
    __shared__ int count[WAVES][EXPERTS], before[EXPERTS], all[EXPERTS];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, inst = blockIdx.y;
    const int *ids = g.ids + (long)inst * g.total;
    const int first = (int)blockIdx.x * RUN + wave * ROUNDS * 64 + lane;
    int id[ROUNDS], place[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) id[r] = id_at(g, ids, first + r * 64);
    for (int e = tid; e < EXPERTS; e += THREADS) before[e] = all[e] = 0;
    for (int e = lane; e < EXPERTS; e += 64) count[wave][e] = 0;
    __syncthreads();

    // ---- what lies ahead of this run, and in all of them
    if (MANY) {
        const int *from = g.counts + (long)inst * g.runs * g.experts;
        constexpr int PARTS = THREADS / EXPERTS > 0 ? THREADS / EXPERTS : 1;
        static_assert(!MANY || THREADS % EXPERTS == 0, "a thread for each expert, or several");
        const int e = tid % EXPERTS;
        if (e < g.experts) {
            int a = 0, b = 0;
#pragma unroll 8
            for (int run = tid / EXPERTS; run < g.runs; run += PARTS) {
                const int n = from[(long)run * g.experts + e];
                a += n;
                b += run < (int)blockIdx.x ? n : 0;
            }
            atomicAdd(&all[e], a);
            atomicAdd(&before[e], b);
        }
    }

    // ---- places among the wavefront's own
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        unsigned long same = __ballot(id[r] >= 0);
#pragma unroll
        for (int b = 0; b < BITS; ++b) {
            const bool set = id[r] >> b & 1;
            const unsigned long m = __ballot(set);
            same &= set ? m : ~m;
        }
        const int below = __builtin_popcountl(same & ((1ul << lane) - 1));
        int so_far = 0;
        if (id[r] >= 0) so_far = count[wave][id[r]];
        place[r] = so_far + below;
        wave_lds();
        if (id[r] >= 0 && below == 0) count[wave][id[r]] = so_far + __builtin_popcountl(same);
        wave_lds();
    }
    __syncthreads();

    // ---- wavefronts after each other
    for (int e = tid; e < EXPERTS; e += THREADS) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int here = count[w][e];
            count[w][e] = n;
            n += here;
        }
        if (!MANY) all[e] = n;
    }
    __syncthreads();
    if (wave == 0) { // experts after each other
        int n = 0;
#pragma unroll
        for (int e0 = 0; e0 < EXPERTS; e0 += 64) {
            const int own = all[e0 + lane], sum = sums_of_lanes(own) + n;
            before[e0 + lane] += sum - own;
            if (blockIdx.x == 0 && e0 + lane < g.experts) {
                int *offsets = g.offsets + (long)inst * (g.experts + 1);
                if (e0 + lane == 0) offsets[0] = 0;
                offsets[e0 + lane + 1] = sum;
            }
            n = __builtin_amdgcn_readlane(sum, 63);
        }
    }
    __syncthreads();
    int *to = g.place + (long)inst * g.total;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (first + r * 64 < g.total) to[first + r * 64] = id[r] >= 0 ? before[id[r]] + count[wave][id[r]] + place[r] : -1;
}
