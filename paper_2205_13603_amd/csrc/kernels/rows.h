// Shared by the kernels whose lanes hold eight neighbouring columns of a row each.
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
