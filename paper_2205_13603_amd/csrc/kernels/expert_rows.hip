// Rows of tokens to the rows of their choices, and back.
//
//   OUT    Y[place[t][j]] = X[t], or X[t] in 8 bits: integers with a scale for the row, S = max(max |x| * fl(1 / 127), 2^-126), x / S to the nearest; floats with a
//          scale for each 128 columns, S = max(max |x| / 448, 2^-126).  X in 8 bits already: its scales go along.
//   BACK   Y[t] = R[t] + sum_j W[t][j] X[place[t][j]] in fp32, in the order of j, rounded once
//   GRAD   Y[place[t][j]] = W[t][j] X[t], S[t][j] = sum_c X[t][c] C[place[t][j]][c]: the gradients of BACK's X and W where X here is that of its Y
// Places outside of [0, rows) are of no choice: nothing is read or written for them, S is 0 there.
//
// WAVES wavefronts share a token, 8 neighbouring columns of a lane in each chunk of 512 columns; OUT keeps up to NV chunks in registers and reads what
// lies beyond again.  A token's places and weights lie in the lanes of each of its wavefronts, from where scalar registers take them: a row's
// address is computed once, by the scalar unit.
//
// What bounds it is memory: bf16, 4096 x 2048 to 8 choices into 8-bit integers 14.8 us (5.7 TB/s), into 8-bit floats 15.3 (5.6; from fp32 17.5, 5.9), as they are 26.2 (5.8),
// 8 bits as they are 14.4 (integers) and 15.1 (floats); back 28.4 (5.3, rows of 4 KiB read in any
// order); gradients 57 (5.0, as much written as read; 3000 x 2050 to 6 choices, whose rows are no whole 16 bytes, 30 to 36 by what the card's last level cache
// holds).  Results stay out of the L2s: kept there 4096 x 2048 to 8 choices takes 32 us instead of 26, back 32 instead of 28.  Few tokens: the launch.
#include "common.h"
#include "rows.h"

struct rows_args {
    const char *x;
    const int *place;
    const float *w;
    const char *c; // BACK: R; GRAD: C; OUT: scales of X
    char *y;
    float *s;
    long x_row, x_inst, c_row, c_inst; // in bytes
    int tokens, chosen, cols, rows;
};

constexpr int NV = 4, THREADS = WAVES < 3 ? 256 : WAVES * 64, GROUPS = THREADS / 64 / WAVES, STEP = WAVES * 512;
constexpr int ES = sizeof(in_t), OS = sizeof(out_t);
constexpr bool BYTES = ES == 1, TO_I8 = OUT_DT == DT_I8 && !BYTES, TO_F8 = OUT_DT == DT_F8E4M3 && !BYTES;

struct bytes_t { char v[8]; };
struct results_t { out_t v[8]; };
__device__ __forceinline__ out_t round_out(float x)
{
#if OUT_DT == DT_BF16
    return float_to_bf16(x);
#else
    return (out_t)x;
#endif
}
// n (up to 8) values at `dst`, which need only be aligned to them; past the L2s
template <class T> __device__ __forceinline__ void give8(char *dst, const T &o, int n)
{
    constexpr int SIZE = sizeof(T) / 8;
    typedef unsigned words_t __attribute__((ext_vector_type(SIZE == 1 ? 2 : 4), aligned(SIZE)));
    struct parts_t { words_t v[SIZE == 4 ? 2 : 1]; };
    if (n >= 8) {
        const parts_t p = __builtin_bit_cast(parts_t, o);
#pragma unroll
        for (int i = 0; i < (SIZE == 4 ? 2 : 1); ++i) __builtin_nontemporal_store(p.v[i], reinterpret_cast<words_t *>(dst) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) __builtin_memcpy(dst + i * SIZE, &o.v[i], SIZE);
    }
}
__device__ __forceinline__ float value_of(out_t x)
{
#if OUT_DT == DT_BF16
    return bf16_to_float(x);
#else
    return (float)x;
#endif
}
__device__ __forceinline__ results_t take_results(const char *p, int n)
{
    results_t x;
    if (n >= 8) {
        typedef unsigned words_t __attribute__((ext_vector_type(2), aligned(OS)));
#pragma unroll
        for (int i = 0; i < OS; ++i) reinterpret_cast<words_t *>(&x)[i] = reinterpret_cast<const words_t *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.v[i] = out_t(0);
            if (i < n) x.v[i] = reinterpret_cast<const out_t *>(p)[i];
        }
    }
    return x;
}
__device__ __forceinline__ float sum_wave(float x)
{
    x = sum16(x);
    return lane_of(x, 0) + lane_of(x, 16) + lane_of(x, 32) + lane_of(x, 48);
}
#if !(IN_DT == DT_I8 || IN_DT == DT_F8E4M3)
typedef raw_t chunk_t;
__device__ __forceinline__ chunk_t take8(const char *p, int n) { return load8(reinterpret_cast<const in_t *>(p), n); }
#else
typedef bytes_t chunk_t;
__device__ __forceinline__ chunk_t take8(const char *p, int n)
{
    chunk_t x;
    if (n >= 8) x = __builtin_bit_cast(chunk_t, *reinterpret_cast<const u2a_t *>(p));
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = i < n ? p[i] : 0;
    }
    return x;
}
#endif

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const rows_args g)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), group = wave / WAVES, part = wave % WAVES, inst = blockIdx.y;
    const int token = (int)blockIdx.x * GROUPS + group;
    const bool live = token < g.tokens; // wavefronts of tokens behind the last only meet the barriers
    const int cols = live ? g.cols : 0, chosen = live ? g.chosen : 0, c0 = (part * 64 + lane) * 8;
    const long at = (long)inst * g.tokens + (live ? token : 0);

    // A lane's eight columns.  The last ones of a row begin eight ahead of its end and share some with the lane before, which has the same values:
    // no load or store is one of single columns.  Rows of less than eight columns: one by one.
    const bool wide = g.cols >= 8;
    auto begin = [&](int c) { return wide && c > g.cols - 8 ? g.cols - 8 : c; };
    auto left = [&](int c) { return wide ? 8 : g.cols - c; }; // of them that there are

    // ---- the token's choices: place j in lane j, -1 where it is none
    int place = -1;
    float weight = 1;
    if (lane < chosen) {
        place = g.place ? g.place[at * g.chosen + lane] : token;
        if (place >= g.rows) place = -1;
        if (g.w) weight = g.w[at * g.chosen + lane];
    }
    const unsigned long real = __ballot(place >= 0);
    auto take = [&](const char *row, int c) { return take8(row + (long)begin(c) * ES, left(c)); };
    auto place_of = [&](int j) { return (long)__builtin_amdgcn_readlane(place, j); };
    auto weight_of = [&](int j) { return lane_of(weight, j); };

#if MODE == 0 // OUT
    const char *x = g.x + inst * g.x_inst + (live ? token : 0) * g.x_row;
    char *y = g.y + (long)inst * g.rows * g.cols * OS;
    chunk_t keep[NV] = {};
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (c0 + k * STEP < cols) keep[k] = TO_F8 ? take8(x + (long)(c0 + k * STEP) * ES, cols - c0 - k * STEP) : take(x, c0 + k * STEP);
    auto each = [&](auto f) { // of the lane's chunks
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (c0 + k * STEP < cols) f(c0 + k * STEP, keep[k]);
        for (int c = c0 + NV * STEP; c < cols; c += STEP) f(c, take(x, c));
    };
    auto to_all = [&](int c, const auto &o) {
        for (unsigned long m = real; m; m &= m - 1) give8(y + (place_of(__builtin_ctzl(m)) * g.cols + begin(c)) * OS, o, left(c));
    };
    if constexpr (TO_I8) {
        __shared__ unsigned parts[THREADS / 64];
        unsigned most = 0; // of bit patterns without sign, which order like the values and put NaN on top
        each([&](int, const chunk_t &v) {
#if !(IN_DT == DT_I8 || IN_DT == DT_F8E4M3)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned b = __float_as_uint(to_acc(v.v[i])) & 0x7fffffffu;
                most = most > b ? most : b;
            }
#endif
        });
        most = max16(most);
#pragma unroll
        for (int i = 0; i < 64; i += 16) {
            const unsigned b = __builtin_amdgcn_readlane(most, i);
            most = most > b ? most : b;
        }
        most = __builtin_amdgcn_readfirstlane(most);
        if (WAVES > 1) {
            if (lane == 0) parts[wave] = most;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                const unsigned b = parts[group * WAVES + i];
                most = most > b ? most : b;
            }
        }
        float s = __uint_as_float(most) * (1.f / 127.f);
        s = s < LEAST ? LEAST : s; // NaN stays
        if (part == 0 && place >= 0) g.s[(long)inst * g.rows + place] = s;
        each([&](int c, const chunk_t &v) {
#if !(IN_DT == DT_I8 || IN_DT == DT_F8E4M3)
            bytes_t o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float q = __builtin_rintf(to_acc(v.v[i]) / s); // ties to even; of NaN and of infinity over infinity 0
                o.v[i] = (char)(int)(q == q ? q : 0.f);
            }
            to_all(c, o);
#endif
        });
    } else if constexpr (TO_F8) {
        const int blocks = (g.cols + 127) / 128;
        auto one = [&](int c, const chunk_t &v) { // the 16 lanes of a scale together
#if !(IN_DT == DT_I8 || IN_DT == DT_F8E4M3)
            float f[8];
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = to_acc(v.v[i]);
                const unsigned b = c + i < cols ? __float_as_uint(f[i]) & 0x7fffffffu : 0;
                most = most > b ? most : b;
            }
            float s = __uint_as_float(max16(most)) / LARGEST;
            s = s < LEAST ? LEAST : s;
            quotients(f, s);
            int lo = 0, hi = 0;
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], hi, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], hi, true);
            bytes_t o = __builtin_bit_cast(bytes_t, (unsigned long)(unsigned)hi << 32 | (unsigned)lo);
            for (unsigned long m = real; m; m &= m - 1) {
                const long to = (long)inst * g.rows + place_of(__builtin_ctzl(m));
                if (c < cols) give8(g.y + to * g.cols + c, o, cols - c);
                if (lane % 16 == 0) g.s[to * blocks + c / 128] = s;
            }
#endif
        };
        const int last = (cols + 127) / 128 * 128;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (c0 + k * STEP < last) one(c0 + k * STEP, keep[k]);
        for (int c = c0 + NV * STEP; c < last; c += STEP) one(c, take8(x + (long)c * ES, cols - c));
    } else {
        each([&](int c, const chunk_t &v) { to_all(c, v); });
        if (BYTES) { // scales go along
            const int blocks = OUT_DT == DT_I8 ? 1 : (g.cols + 127) / 128;
            const float *from = reinterpret_cast<const float *>(g.c) + at * blocks;
            for (int b = part * 64 + lane; live && b < blocks; b += WAVES * 64) {
                const float s = from[b];
                for (unsigned long m = real; m; m &= m - 1) g.s[((long)inst * g.rows + place_of(__builtin_ctzl(m))) * blocks + b] = s;
            }
        }
    }
#else
    // the token's choices AT_ONCE at a time, their rows in flight together
    constexpr int AT_ONCE = 4;
    auto batches = [&](auto f) { // f(places, numbers, how many)
        for (unsigned long m = real; m;) {
            long p[AT_ONCE];
            int j[AT_ONCE], n = 0;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                j[u] = m ? __builtin_ctzl(m) : 0;
                p[u] = place_of(j[u]);
                n += m != 0;
                m &= m - 1;
            }
            f(p, j, n);
        }
    };
#if MODE == 1 // BACK
    const char *x = g.x + inst * g.x_inst, *r = g.c + at * g.cols * OS;
    char *y = g.y + at * g.cols * OS;
    for (int c = c0; c < cols; c += STEP) {
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (RESIDUAL) {
            const results_t o = take_results(r + (long)begin(c) * OS, left(c));
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = value_of(o.v[i]);
        }
        batches([&](const long (&p)[AT_ONCE], const int (&j)[AT_ONCE], int count) {
            chunk_t v[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (u < count) v[u] = take(x + p[u] * g.x_row, c);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (u < count) {
                    const float w = weight_of(j[u]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(w, to_acc(v[u].v[i]), sum[i]);
                }
        });
        results_t o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = round_out(sum[i]);
        if (RESIDUAL && c > cols - 8) { // R may be Y: what the lane before shares with this one is its to write
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (begin(c) + i >= c && i < left(c)) reinterpret_cast<out_t *>(y)[begin(c) + i] = o.v[i];
        } else {
            give8(y + (long)begin(c) * OS, o, left(c));
        }
    }
#else
    const char *x = g.x + inst * g.x_inst + (live ? token : 0) * g.x_row, *other = g.c + inst * g.c_inst;
    char *y = g.y + (long)inst * g.rows * g.cols * OS;
    __shared__ float parts[THREADS / 64][64];
    float dots = 0; // of choice j in lane j
    for (int c1 = part * 512; c1 < cols; c1 += STEP) { // all lanes together: their sums are added up
        const int c = c1 + lane * 8, from = begin(c), n = left(c);
        const bool there = c < cols;
        chunk_t v = {};
        if (wide || there) v = take(x, c);
        const bool tail = c1 + 512 > cols; // some lanes have columns that are not to be counted: none, or the lane before's
        batches([&](const long (&p)[AT_ONCE], const int (&j)[AT_ONCE], int count) {
            chunk_t q[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (u < count && (wide || there)) q[u] = take(other + p[u] * g.c_row, c);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (u < count) {
                    const float w = weight_of(j[u]);
                    if (tail) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!there || from + i < c) q[u].v[i] = in_t(0);
                    }
                    float dot = 0;
                    results_t o;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dot = __builtin_fmaf(tail && (!there || from + i < c) ? 0.f : to_acc(v.v[i]), to_acc(q[u].v[i]), dot);
                        o.v[i] = round_out(w * to_acc(v.v[i]));
                    }
                    if (there) give8(y + (p[u] * g.cols + from) * OS, o, n);
                    dot = sum_wave(dot);
                    dots += lane == j[u] ? dot : 0.f;
                }
        });
    }
    if (WAVES > 1) {
        parts[wave][lane] = dots;
        __syncthreads();
        dots = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) dots += parts[group * WAVES + i][lane];
    }
    if (part == 0 && lane < chosen) g.s[at * g.chosen + lane] = dots;
#endif
#endif
}
