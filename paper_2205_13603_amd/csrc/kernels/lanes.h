// Shared by the kernels in which groups of LANES neighbouring lanes take a token each: LANES = 8 to 64, all lanes of a wavefront together.

// From the lane of the other half of the 2 * STEP lanes that this one is among: the one STEP away (1, 2, 16, 32) or the mirrored one (4, 8),
// which is as good where each half holds the same in all of its lanes.
template <int STEP> __device__ __forceinline__ unsigned from_other(unsigned x)
{
    if constexpr (STEP == 1) return __builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true);
    else if constexpr (STEP == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true);
    else if constexpr (STEP == 4) return __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true);
    else if constexpr (STEP == 8) return __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true);
    else return __builtin_amdgcn_ds_bpermute((threadIdx.x % 64 ^ STEP) * 4, x);
}
template <int STEP> __device__ __forceinline__ float from_other(float x) { return __uint_as_float(from_other<STEP>(__float_as_uint(x))); }
template <int STEP> __device__ __forceinline__ double from_other(double x)
{
    const unsigned long b = __builtin_bit_cast(unsigned long, x);
    return __builtin_bit_cast(double, (unsigned long)from_other<STEP>((unsigned)(b >> 32)) << 32 | from_other<STEP>((unsigned)b));
}
// Over a token's lanes, the same in all of them afterwards.
template <class T, class F, int STEP = 1> __device__ __forceinline__ T over_lanes(T x, F f)
{
    if constexpr (STEP < LANES) return over_lanes<T, F, STEP * 2>(f(x, from_other<STEP>(x)), f);
    else return x;
}
template <class T> __device__ __forceinline__ T sum_lanes(T x)
{
    return over_lanes(x, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ float max_lanes(float x)
{
    return over_lanes(x, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ unsigned or_lanes(unsigned x)
{
    return over_lanes(x, [](unsigned a, unsigned b) { return a | b; });
}
// LDS that only this wavefront uses: what its lanes have written is there for all of them.
__device__ __forceinline__ void wave_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A token's logits: chunks of CH neighbouring experts, the chunks of its lanes after each other, so that a load of all lanes takes whole lines.
constexpr int CH = 16 / (int)sizeof(in_t) < VALUES ? 16 / (int)sizeof(in_t) : VALUES;
__device__ __forceinline__ int expert_of(int i, int l) { return (i / CH * LANES + l) * CH + i % CH; }
struct __attribute__((packed, aligned(sizeof(in_t)))) logits_t { in_t v[CH]; };
// The logits of a lane, `none` where there is no expert.  All loads of a chunk are on their way together: none is behind a branch of its own.
__device__ __forceinline__ void load_logits(const in_t *row, int l, int experts, float none, float (&x)[VALUES])
{
#pragma unroll
    for (int c = 0; c < VALUES; c += CH) {
        const int e = expert_of(c, l);
        if (e + CH <= experts) {
            const logits_t q = *reinterpret_cast<const logits_t *>(row + e);
#pragma unroll
            for (int i = 0; i < CH; ++i) x[c + i] = to_acc(q.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i) x[c + i] = to_acc(row[e + i < experts ? e + i : experts - 1]);
#pragma unroll
            for (int i = 0; i < CH; ++i) x[c + i] = e + i < experts ? x[c + i] : none;
        }
    }
}
