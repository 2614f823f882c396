// Which experts a token goes to, and with which weights.
//
// Scores s = softmax(x) or sigmoid(x) over a token's logits; choice c = s + bias; the best `kept` groups of experts by the sum of their best one or
// two c, of the experts in them the best `chosen` by c; weights s of the chosen, over their sum (RENORM), times a scale.
//
// Whom a token goes to must not hang on how an exponential rounds: c is formed in 64 bits.  Its lowest 10 bits of significand make room for the expert's
// index (the others tell 2^-42 apart), in the order that puts the lower index first among equals, and choosing is then sorting of doubles that
// differ.  Without a bias, and with one expert to speak for a group, the logits choose, whose order is that of their scores; they are exact in what is left.
// Experts that cannot be chosen (logit -infinity or NaN) are less than all others.
//
// LANES lanes take a token, VALUES experts each: a lane sorts its own (Batcher's exchanges, blocks of TOP, the best TOP of two blocks are the
// larger of one block's ascending and the other's descending list), then the lanes' lists meet in log2(LANES) steps the same way, after which all
// lanes have the token's.  Groups of a power of two experts find their best in the lanes that hold them, others by way of LDS.
//
// What bounds it are the vector ALUs: 16384 x 256 in fp32, sigmoid, bias, 8 groups, 12.3 us, of which each SIMD issues 5270 instructions for some 9 us
// (a third forms scores, a third sorts, a sixth finds groups); the logits take 2.7 from memory.  Choices by logits alone, 16384 x 128: 4.4 us, the launch.
// Wavefronts that go on to further tokens with the next logits under way take 13.2: what is hoisted out of their loop costs half the wavefronts.
// One token 4.5 us, the launch.
#include "common.h"
#include "lanes.h"

struct route_args {
    const in_t *x;
    const float *bias;
    int *ids;
    float *w;
    long x_row, x_inst; // in elements
    int tokens, experts, chosen, groups, kept;
    float scale;
};

constexpr int TOKENS = 64 / LANES, WAVES = THREADS / 64;
constexpr bool BY_LOGIT = !BIAS && BEST == 1;     // what chooses; else scores
constexpr bool SUM = !SIGMOID && !(BY_LOGIT && RENORM); // of the exponentials of all logits
static_assert(TOP <= LANES * VALUES, "a list of them all at most");

__device__ __forceinline__ double larger(double a, double b) { return __builtin_fmax(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return __builtin_fmin(a, b); }
__device__ __forceinline__ void exchange(double &a, double &b) // a the larger
{
    const double x = larger(a, b);
    b = smaller(a, b);
    a = x;
}
// Batcher's odd-even merge sort, the largest first.
template <int N, int P, int K> __device__ __forceinline__ void sort_step(double *k)
{
#pragma unroll
    for (int j = K % P; j <= N - 1 - K; j += 2 * K)
#pragma unroll
        for (int i = 0; i < (K < N - j - K ? K : N - j - K); ++i)
            if ((i + j) / (2 * P) == (i + j + K) / (2 * P)) exchange(k[i + j], k[i + j + K]);
    if constexpr (K > 1) sort_step<N, P, K / 2>(k);
    else if constexpr (2 * P < N) sort_step<N, 2 * P, 2 * P>(k);
}
// Of a list that rises and falls (or falls and rises), the largest first.
template <int N> __device__ __forceinline__ void merge(double *k)
{
    if constexpr (N > 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) exchange(k[i], k[i + N / 2]);
        merge<N / 2>(k);
        merge<N / 2>(k + N / 2);
    }
}
// The lists of N of two halves of 2 * STEP lanes become one of up to TOP.
template <int N, int STEP> __device__ __forceinline__ void meet(double (&k)[TOP])
{
    if constexpr (STEP < LANES) {
        double o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = from_other<STEP>(k[i]);
        if constexpr (N < TOP) {
#pragma unroll
            for (int i = 0; i < N; ++i) k[2 * N - 1 - i] = o[i];
            merge<2 * N>(k);
            meet<2 * N, STEP * 2>(k);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) k[i] = larger(k[i], o[N - 1 - i]);
            merge<N>(k);
            meet<N, STEP * 2>(k);
        }
    }
}

constexpr float LEAST = -__builtin_inff(), LARGEST = 0x1.fffffep127f;
constexpr double NONE = -0x1.fffffffffffffp1023, ANY = -0x1p1000; // what cannot be chosen; what all that can is larger than
constexpr unsigned INDEX = 1023;
__device__ __forceinline__ unsigned high_of(double x) { return __builtin_bit_cast(unsigned long, x) >> 32; }
__device__ __forceinline__ unsigned low_of(double x) { return (unsigned)__builtin_bit_cast(unsigned long, x); }
__device__ __forceinline__ double of_halves(unsigned high, unsigned low) { return __builtin_bit_cast(double, (unsigned long)high << 32 | low); }
__device__ __forceinline__ unsigned sign_of(unsigned high) { return __builtin_amdgcn_sbfe(high, 31, 1); } // all bits the sign
// A finite number (no negative zero) with the index `e` in its lowest bits, the lower index the larger; SIGNED: it may be negative.
template <bool SIGNED> __device__ __forceinline__ double with_index(double c, unsigned e)
{
    unsigned x = e ^ INDEX;
    if (SIGNED) x ^= sign_of(high_of(c)) & INDEX;
    return of_halves(high_of(c), (low_of(c) & ~INDEX) | x);
}
__device__ __forceinline__ int index_of(double k) { return (int)((low_of(k) ^ ~sign_of(high_of(k))) & INDEX); }
__device__ __forceinline__ double without_index(double k) { return of_halves(high_of(k), low_of(k) & ~INDEX); }
// k, or something like NONE
__device__ __forceinline__ double only_if(bool there, double k) { return of_halves(there ? high_of(k) : high_of(NONE), low_of(k)); }

// e^x, |x| <= 710, within 2^-44.4 of it (up to 100, where ln(2) as one number costs nothing yet, 2^-45.3): 2^n times a polynomial of degree 9 in the rest r, |r| <= ln(2) / 2, that meets e^r in the ten Chebyshev points of a
// little more than that (2^-45.6).  The coefficients lie in scalar registers: as literals each would cost two moves.
struct series_t { double c[10], per_ln2, ln2, round; };
__device__ __forceinline__ series_t series()
{
    series_t s = {{0x1.72e14a22d5652p-19, 0x1.a17e4c1ffac89p-16, 0x1.a019949078924p-13, 0x1.6c162b6b117dcp-10, 0x1.11111123cd74bp-7, 0x1.55555588dfcb2p-5, 0x1.5555555550d3ep-3,
                   0x1.ffffffffe735cp-2, 0x1.0000000000006p+0, 0x1.000000000003dp+0},
                  0x1.71547652b82fep0, 0x1.62e42fefa39efp-1, 0x1.8p52};
#pragma unroll
    for (int i = 0; i < 10; ++i) asm("" : "+s"(s.c[i]));
    asm("" : "+s"(s.per_ln2), "+s"(s.ln2), "+s"(s.round));
    return s;
}
__device__ __forceinline__ double power_of_e(const series_t &s, double x)
{
    const double t = __builtin_fma(x, s.per_ln2, s.round); // n in its lowest bits
    const double r = __builtin_fma(t - s.round, -s.ln2, x);
    double p = s.c[0];
#pragma unroll
    for (int i = 1; i < 10; ++i) p = __builtin_fma(p, r, s.c[i]);
    return __builtin_ldexp(p, (int)low_of(t));
}
// 1 / x of normal numbers up to 10^306: the hardware's 2^-23, cubed; NaN for zero
__device__ __forceinline__ double reciprocal_of(double x)
{
    const double y = __builtin_amdgcn_rcp(x), e = __builtin_fma(-x, y, 1.);
    return __builtin_fma(y, __builtin_fma(e, e, e), y);
}

#if GROUPED
// The two largest (BEST 1: the one) of the ACROSS lanes that hold a group.
template <int STEP, int ACROSS> __device__ __forceinline__ void best_of_lanes(double &a, double &b)
{
    if constexpr (STEP < ACROSS) {
        const double c = from_other<STEP>(a);
        if constexpr (BEST == 2) b = larger(smaller(a, c), larger(b, from_other<STEP>(b)));
        a = larger(a, c);
        best_of_lanes<STEP * 2, ACROSS>(a, b);
    }
}
// The N values of each lane's part, of all parts.
template <int N, int STEP, int ALL> __device__ __forceinline__ void gather(double (&v)[ALL])
{
    if constexpr (N < ALL) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[N + i] = from_other<STEP>(v[i]);
        gather<N * 2, STEP * 2>(v);
    }
}
__device__ __forceinline__ double of_group(double a, double b, int n) // what chooses group n
{
    double c = without_index(a);
    if (BEST == 2) c += b > ANY ? without_index(b) : 0.;
    return only_if(a > ANY, with_index<true>(c, n));
}
#endif

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const route_args g)
{
    const int lane = threadIdx.x % 64, l = lane % LANES, wave = threadIdx.x / 64, inst = blockIdx.y;
    const int token = ((int)blockIdx.x * WAVES + wave) * TOKENS + lane / LANES;
    const bool live = token < g.tokens; // lanes behind the last token do as if they were its, but give nothing
    const int experts = g.experts;
    const in_t *row = g.x + inst * g.x_inst + (live ? token : g.tokens - 1) * g.x_row;
    float x[VALUES];
    load_logits(row, l, experts, LEAST, x);
#if BIAS
    float bias[VALUES];
    const float *biases = g.bias + (long)inst * experts;
#pragma unroll
    for (int c = 0; c < VALUES; c += CH) {
        const int e = expert_of(c, l);
        struct __attribute__((packed, aligned(4))) biases_t { float v[CH]; };
        if (e + CH <= experts) {
            const biases_t q = *reinterpret_cast<const biases_t *>(biases + e);
#pragma unroll
            for (int i = 0; i < CH; ++i) bias[c + i] = q.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i) bias[c + i] = biases[e + i < experts ? e + i : experts - 1];
        }
    }
#endif

    // ---- the largest logit, the sum of exponentials; NaN, and infinity under a softmax, make the row's weights NaN
    bool bad = false;
    float most = LEAST;
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        bad |= x[i] != x[i];
        most = __builtin_fmaxf(most, x[i]);
    }
    float top = 0;
    double sum = 0, inverse = 0;
    const series_t terms = series();
    double key[VALUES];
    if constexpr (!SIGMOID) {
        most = max_lanes(most);
        bad |= most == -LEAST;
        top = most > LEAST ? most : 0.f; // a row without experts
    }
    bad = or_lanes(bad);
    if constexpr (SUM) {
        if constexpr (BY_LOGIT) { // the sum is that of the weights only
            float s = 0;
#pragma unroll
            for (int i = 0; i < VALUES; ++i) s += expf(x[i] - top);
            sum = sum_lanes(s);
        } else {
#pragma unroll
            for (int i = 0; i < VALUES; ++i) {
                key[i] = power_of_e(terms, larger((double)x[i] - top, -700.)); // 10^-304 for what cannot be chosen
                sum += key[i];
            }
            sum = sum_lanes(sum);
            inverse = reciprocal_of(sum);
        }
    }

    // ---- what chooses
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        const int e = expert_of(i, l);
        bool there = x[i] > LEAST; // and no NaN
        double c;
        if constexpr (BY_LOGIT) {
            c = __builtin_fminf(x[i], LARGEST) + 0.f; // an infinity would become NaN; the two zeros are one
        } else {
            if constexpr (SIGMOID) c = reciprocal_of(1 + power_of_e(terms, -(double)__builtin_amdgcn_fmed3f(x[i], -700.f, 700.f)));
            else c = key[i] * inverse;
            if constexpr (!SIGMOID) there = there && !bad; // no score is a number then
#if BIAS
            there = there && bias[i] > LEAST;
            c += (double)__builtin_fminf(bias[i], LARGEST);
#endif
        }
        key[i] = only_if(there, with_index<BY_LOGIT || BIAS>(c, e));
    }

    // ---- groups
#if GROUPED && GROUP_SIZE
    // of a power of two experts: whole rows of the lanes' chunks, or the chunks of neighbouring lanes
    constexpr int ROW = LANES * CH, PER = GROUP_SIZE > ROW ? GROUP_SIZE / ROW : 1, SLOTS = VALUES / CH / PER, ACROSS = GROUP_SIZE < ROW ? GROUP_SIZE / CH : LANES, IN_ROW = LANES / ACROSS;
    double all[SLOTS * IN_ROW];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        double a = key[s * PER * CH], b = NONE;
#pragma unroll
        for (int i = s * PER * CH + 1; i < (s + 1) * PER * CH; ++i) {
            if constexpr (BEST == 2) b = larger(b, smaller(a, key[i]));
            a = larger(a, key[i]);
        }
        best_of_lanes<1, ACROSS>(a, b);
        all[s] = of_group(a, b, s * IN_ROW + l / ACROSS);
    }
    gather<SLOTS, ACROSS>(all);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        int ahead = 0;
#pragma unroll
        for (int i = 0; i < SLOTS * IN_ROW; ++i)
            if (i != s) ahead += all[i] > all[s];
        const bool keep = ahead < g.kept;
#pragma unroll
        for (int i = s * PER * CH; i < (s + 1) * PER * CH; ++i) key[i] = only_if(keep, key[i]);
    }
#elif GROUPED
    // of any size: by way of LDS, where groups of 32 lie in banks of their own
    constexpr int KEYS = LANES * VALUES + LANES * VALUES / 32 + 4;
    __shared__ double keys[WAVES * TOKENS][KEYS], best[WAVES * TOKENS][GROUPS + 1];
    double *const mine = keys[wave * TOKENS + lane / LANES], *const groups = best[wave * TOKENS + lane / LANES];
    auto at = [](int e) { return e + e / 32; };
#pragma unroll
    for (int i = 0; i < VALUES; ++i) mine[at(expert_of(i, l))] = key[i];
    wave_lds();
    const int size = experts / g.groups;
    for (int n = l; n < g.groups; n += LANES) {
        double a = NONE, b = NONE;
#pragma unroll 8
        for (int i = 0; i < size; ++i) {
            const double k = mine[at(n * size + i)];
            if constexpr (BEST == 2) b = larger(b, smaller(a, k));
            a = larger(a, k);
        }
        groups[n] = of_group(a, b, n);
    }
    wave_lds();
    unsigned keep[2] = {0, 0}; // groups by their number
    for (int n = l; n < g.groups; n += LANES) {
        const double k = groups[n];
        int ahead = 0;
#pragma unroll 8
        for (int i = 0; i < g.groups; ++i) ahead += groups[i] > k;
        if (ahead < g.kept) keep[n / 32] |= 1u << n % 32;
    }
    keep[0] = or_lanes(keep[0]);
    keep[1] = or_lanes(keep[1]);
    const unsigned long kept = (unsigned long)keep[1] << 32 | keep[0];
    const unsigned reciprocal = ((1u << 21) + size - 1) / size; // e * size < 2^20: the quotient below is e / size
#pragma unroll
    for (int i = 0; i < VALUES; ++i) key[i] = only_if(kept >> ((unsigned)expert_of(i, l) * reciprocal >> 21) % 64 & 1, key[i]);
#endif

    // ---- the best of them
    constexpr int BLOCK = VALUES < TOP ? VALUES : TOP;
    double list[TOP];
#pragma unroll
    for (int b = 0; b < VALUES; b += BLOCK)
        if constexpr (BLOCK > 1) sort_step<BLOCK, 1, 1>(key + b);
#pragma unroll
    for (int i = 0; i < BLOCK; ++i) list[i] = key[i];
#pragma unroll
    for (int b = BLOCK; b < VALUES; b += BLOCK) {
#pragma unroll
        for (int i = 0; i < BLOCK; ++i) list[i] = larger(list[i], key[b + BLOCK - 1 - i]);
        merge<BLOCK>(list);
    }
    meet<BLOCK, 1>(list);

    // ---- weights: choice j in lane j % LANES
    constexpr int ROUNDS = (TOP + LANES - 1) / LANES;
    float logit[ROUNDS];
    int id[ROUNDS];
    float high = LEAST;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        double k = NONE;
#pragma unroll
        for (int j = r * LANES; j < TOP && j < r * LANES + LANES; ++j) k = l == j - r * LANES ? list[j] : k;
        const int j = r * LANES + l;
        id[r] = k > ANY && j < g.chosen ? index_of(k) : -1;
        if constexpr (BY_LOGIT) logit[r] = (float)without_index(k); // exactly
        else logit[r] = to_acc(row[id[r] >= 0 ? id[r] : 0]);
        if (id[r] < 0) logit[r] = LEAST;
        high = __builtin_fmaxf(high, logit[r]);
    }
    if constexpr (!SIGMOID && RENORM) { // relative to the largest chosen: their sum is no less than one
        high = max_lanes(high);
        top = high > LEAST ? high : 0.f;
        sum = 0;
    }
    double w[ROUNDS], total = 0;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const double d = SIGMOID ? (double)logit[r] : (double)logit[r] - top;
        const double e = power_of_e(terms, smaller(larger(SIGMOID ? -d : d, -700.), 700.));
        w[r] = id[r] >= 0 && d >= -700. ? SIGMOID ? reciprocal_of(1 + e) : e : 0.; // e^-700 is none: fp32 ends at e^-103
        total += w[r];
    }
    if constexpr (RENORM) sum = sum_lanes(total);
    const double factor = RENORM || !SIGMOID ? g.scale * reciprocal_of(sum) : (double)g.scale;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int j = r * LANES + l;
        if (live && j < g.chosen) {
            const long to = ((long)inst * g.tokens + token) * g.chosen + j;
            const float y = id[r] >= 0 ? (float)(w[r] * factor) : 0.f;
            g.ids[to] = id[r];
            g.w[to] = bad ? __builtin_nanf("") : y;
        }
    }
}
