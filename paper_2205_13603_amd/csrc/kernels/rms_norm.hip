// Root-mean-square norm of rows, with a residual's addition ahead of it and 8-bit floats with scales behind it.
//
// h = x + r, rounded once to the type of x; y = h * rsqrt(sum(h^2) / N + eps) * w in fp32; per 128 columns s = max |y| / 448 and the
// 8-bit float nearest to y / s.  One pass over memory: a row's values stay in the registers of the WAVES wavefronts that share it, 8
// consecutive columns of a lane in each of up to NV chunks; columns beyond those are read again.  A scale's 128 columns are then 16
// neighbouring lanes, whose maximum needs four cross-lane steps and no memory; the maximum is one of bit patterns without sign, which
// order like the values and put NaN on top.
//
// What bounds it is memory: 16384 x 8192 in bf16 with a residual into 8 bits 174 us, 5.4 TB/s of four streams (a copy reaches 5.2 to 6.4);
// the vector ALUs are busy 60 % of the cycles.  Results leave past the L2s, which otherwise hold lines to be written back when the kernel
// ends (6 us more; 16384 x 1024 28.2 -> 21.8, 8192 x 5120 bf16 without residual 38.8 -> 27).  Loads past the L2s 31 us
// more; weights loaded ahead of the sum 28, for the registers that they take.  One row: 3.9 to 4.9, the launch; 613 x 5000 6.2 to 6.8 back to back.
#include "common.h"

struct rms_args {
    const in_t *x, *w, *r;
    void *y;
    float *s;
    in_t *h;
    long x_row, x_inst;
    int rows, cols, instances;
    float eps;
};

constexpr int NV = 4, THREADS = WAVES < 4 ? 256 : WAVES * 64, GROUPS = THREADS / 64 / WAVES; // rows of a workgroup at a time
constexpr bool F8 = OUT_DT == DT_F8E4M3;
constexpr float LARGEST = 448.f, LEAST = 0x1p-126f; // of the 8-bit floats; of the scales, so that a block of zeros has one

struct raw_t { in_t v[8]; };
typedef unsigned u4a_t __attribute__((ext_vector_type(4), aligned(sizeof(in_t))));
typedef unsigned u2a_t __attribute__((ext_vector_type(2), aligned(1)));

// the hardware loads and stores vectors at any address; n: how many of the 8 columns there are
__device__ __forceinline__ raw_t load8(const in_t *p, int n)
{
    raw_t x;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(raw_t) / 16; ++i) reinterpret_cast<u4a_t *>(&x)[i] = reinterpret_cast<const u4a_t *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = i < n ? p[i] : in_t(0);
    }
    return x;
}
__device__ __forceinline__ void store8(in_t *p, const raw_t &x, int n)
{
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(raw_t) / 16; ++i) __builtin_nontemporal_store(reinterpret_cast<const u4a_t *>(&x)[i], reinterpret_cast<u4a_t *>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = x.v[i];
    }
}
__device__ __forceinline__ in_t round_in(float x)
{
#if IN_DT == DT_BF16
    return float_to_bf16(x);
#else
    return (in_t)x;
#endif
}

template <int CTRL> __device__ __forceinline__ unsigned across(unsigned x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
// over 16 neighbouring lanes: pairs, quads, halves of a row, rows
__device__ __forceinline__ float sum16(float x)
{
    x += __uint_as_float(across<0xb1>(__float_as_uint(x)));
    x += __uint_as_float(across<0x4e>(__float_as_uint(x)));
    x += __uint_as_float(across<0x141>(__float_as_uint(x)));
    return x + __uint_as_float(across<0x140>(__float_as_uint(x)));
}
__device__ __forceinline__ unsigned max16(unsigned x)
{
    unsigned o;
    o = across<0xb1>(x), x = x > o ? x : o;
    o = across<0x4e>(x), x = x > o ? x : o;
    o = across<0x141>(x), x = x > o ? x : o;
    o = across<0x140>(x);
    return x > o ? x : o;
}
// y / s in fp32 as close as the rounding to 8-bit floats can tell from a division's: a reciprocal in two parts is within 3 * 2^-48 of the true one, which
// leaves a quotient on its side of every tie and on the ties themselves.  (Only 518 pairs of significands have quotients so near to where the fp32
// rounding would cross one; all of them come out as the division's.  The rounded reciprocal alone, 1.5 units off, moves one near tie in four.  16384 x 8192 in
// bf16: 171.6 us with the reciprocal, 174.4 this way, 181 with divisions.)
__device__ __forceinline__ void quotients(float (&y)[8], float s)
{
    if (s > 0x1p60f) { // the second part would be subnormal
        s *= 0x1p-60f;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= 0x1p-60f;
    }
    const float to = 1.f / s, rest = s < __builtin_inff() ? __builtin_fmaf(-s, to, 1.f) * to : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(y[i], to, y[i] * rest);
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const rms_args g)
{
    __shared__ float parts[2][THREADS / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, group = wave / WAVES, part = wave % WAVES;
    const int blocks = (g.cols + 127) / 128;
    const long total = (long)g.rows * g.instances;
    const int c0 = (part * 64 + lane) * 8; // this lane's columns in chunk 0
    constexpr int STEP = WAVES * 512;      // columns of a chunk of the row's wavefronts
    int flip = 0;
    for (long base = (long)blockIdx.x * GROUPS; base < total; base += (long)gridDim.x * GROUPS) {
        const long row = base + group;
        const bool live = row < total; // wavefronts of rows behind the last only meet the barrier
        const long inst = live && g.instances > 1 ? row / g.rows : 0, at = live ? row * g.cols : 0;
        const in_t *x = g.x + inst * g.x_inst + (live ? row - inst * g.rows : 0) * g.x_row, *w = g.w + inst * g.cols;
#if RESIDUAL
        const in_t *r = g.r + at;
        in_t *h = g.h + at;
        const in_t *again = h; // what columns beyond the registers are read from
#else
        const in_t *again = x;
#endif
        // columns [c, c + 8) that there are
        auto left = [&](int c) { return live ? g.cols - c : 0; };
        raw_t keep[NV] = {};
        float sum = 0;
        auto take = [&](int c) {
            const int n = left(c);
            raw_t v = load8(x + c, n);
#if RESIDUAL
            const raw_t q = load8(r + c, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) v.v[i] = round_in(to_acc(v.v[i]) + to_acc(q.v[i]));
            store8(h + c, v, n);
#endif
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += to_acc(v.v[i]) * to_acc(v.v[i]);
            return v;
        };
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (left(c0 + k * STEP) > 0) keep[k] = take(c0 + k * STEP);
        for (int c = c0 + NV * STEP; left(c) > 0; c += STEP) take(c);
        sum = sum16(sum);
        sum = lane_of(sum, 0) + lane_of(sum, 16) + lane_of(sum, 32) + lane_of(sum, 48);
        if (WAVES > 1) {
            if (lane == 0) parts[flip][wave] = sum;
            __syncthreads();
            sum = 0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) sum += parts[flip][group * WAVES + i];
            flip ^= 1; // the next row's partial sums go where nobody reads any more
        }
        const float scale = 1.f / sqrtf(sum / (float)g.cols + g.eps);
        auto give = [&](int c, const raw_t &v) {
            const int n = left(c);
            const raw_t q = load8(w + c, n);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = to_acc(v.v[i]) * scale * to_acc(q.v[i]);
            if constexpr (F8) {
                unsigned most = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned m = i < n ? __float_as_uint(y[i]) & 0x7fffffffu : 0;
                    most = most > m ? most : m;
                }
                float s = __uint_as_float(max16(most)) / LARGEST;
                s = s < LEAST ? LEAST : s; // NaN stays
                if (lane % 16 == 0) g.s[row * blocks + c / 128] = s;
                quotients(y, s);
                int lo = 0, hi = 0;
                lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
                lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
                hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
                hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
                char *o = (char *)g.y + at + c;
                if (n >= 8) {
                    __builtin_nontemporal_store(u2a_t{(unsigned)lo, (unsigned)hi}, reinterpret_cast<u2a_t *>(o));
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < n) o[i] = (char)((i < 4 ? lo : hi) >> 8 * (i & 3));
                }
            } else {
                raw_t o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o.v[i] = round_in(y[i]);
                store8((in_t *)g.y + at + c, o, n);
            }
        };
        // the 16 lanes of a scale take part together: lanes behind the row's end with nothing to give but zero
        const int last = live ? (g.cols + 127) / 128 * 128 : 0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (c0 + k * STEP < last) give(c0 + k * STEP, keep[k]);
        for (int c = c0 + NV * STEP; c < last; c += STEP) give(c, load8(again + c, left(c)));
    }
}
