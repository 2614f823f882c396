// Which experts a token goes to, and with which weights.
//
// Scores s = softmax(x) or sigmoid(x) over a token's logits; choice c = s + bias; the best `kept` groups of experts by the sum of their best one or
// two c, of the experts in them the best `chosen` by c; weights s of the chosen, over their sum (RENORM), times a scale.
//
// Whom a token goes to must not hang on how an exponential rounds: c is formed in 64 bits.  Its lowest 10 bits of significand make room for the expert's
// index (the others tell 2^-42 apart), in the order that puts the lower index first among equals, and choosing is then sorting of doubles that
// differ.  Without a bias, and with one expert to speak for a group, the logits choose, whose order is that of their scores; they are exact in what is left.
// Experts that cannot be chosen (logit -infinity or NaN) are -infinity.
//
// LANES lanes take a token, VALUES experts each: a lane sorts its own (Batcher's exchanges, blocks of TOP, the best TOP of two blocks are the
// larger of one block's ascending and the other's descending list), then the lanes' lists meet in log2(LANES) steps the same way, after which all
// lanes have the token's.
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
constexpr int MOST_GROUPS = 64, KEYS = LANES * VALUES + LANES * VALUES / 32 + 4; // of a token in LDS, groups of 32 in banks of their own
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

constexpr double NONE = -__builtin_inf(), MOST = 0x1.fffffffffffffp1023;
constexpr unsigned long INDEX = 1023;
// a number with the index `e` in its lowest bits, the lower index the larger
__device__ __forceinline__ double with_index(double c, int e)
{
    c = smaller(c, MOST) + 0.0; // infinity would become NaN; the two zeros are one
    const unsigned long b = __builtin_bit_cast(unsigned long, c);
    return __builtin_bit_cast(double, (b & ~INDEX) | ((long)b < 0 ? (unsigned long)e : INDEX - e));
}
__device__ __forceinline__ int index_of(double k)
{
    const unsigned long b = __builtin_bit_cast(unsigned long, k);
    return (int)((long)b < 0 ? b & INDEX : INDEX - (b & INDEX));
}
__device__ __forceinline__ double without_index(double k) { return __builtin_bit_cast(double, __builtin_bit_cast(unsigned long, k) & ~INDEX); }

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const route_args g)
{
    const int lane = threadIdx.x % 64, l = lane % LANES, wave = threadIdx.x / 64, inst = blockIdx.y;
    const int token = ((int)blockIdx.x * WAVES + wave) * TOKENS + lane / LANES;
    const bool live = token < g.tokens;
    const int experts = live ? g.experts : 0;
    const in_t *row = g.x + inst * g.x_inst + (live ? token : 0) * g.x_row;
    float x[VALUES];
    load_logits(row, l, experts, NONE, x);

    // ---- the largest logit, the sum of exponentials; NaN, and infinity under a softmax, make the row's weights NaN
    bool bad = false;
    float most = NONE;
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        bad |= x[i] != x[i];
        most = __builtin_fmaxf(most, x[i]);
    }
    float top = 0;
    double sum = 0, inverse = 0;
    double key[VALUES];
    if constexpr (!SIGMOID) {
        most = max_lanes(most);
        bad |= most == (float)__builtin_inf();
        top = most > (float)NONE ? most : 0.f; // a row without experts
    }
    if constexpr (SUM) {
        if constexpr (BY_LOGIT) { // the sum is that of the weights only
            float s = 0;
#pragma unroll
            for (int i = 0; i < VALUES; ++i) s += expf(x[i] - top);
            sum = sum_lanes(s);
        } else {
#pragma unroll
            for (int i = 0; i < VALUES; ++i) {
                key[i] = exp((double)x[i] - top);
                sum += key[i];
            }
            sum = sum_lanes(sum);
            inverse = 1 / sum;
        }
    }
    bad = or_lanes(bad);

    // ---- what chooses
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        const int e = expert_of(i, l);
        const bool there = x[i] > (float)NONE; // and no NaN
        double c = x[i];
        if constexpr (!BY_LOGIT) {
            if constexpr (SIGMOID) c = 1 / (1 + exp(-(double)x[i]));
            else c = key[i] * inverse;
            if constexpr (BIAS) {
                float b = 0;
                if (e < experts) b = g.bias[(long)inst * g.experts + e];
                c += (double)b;
            }
        }
        key[i] = there && c > NONE ? with_index(c, e) : NONE;
    }

    // ---- groups
#if GROUPED
    __shared__ double keys[WAVES * TOKENS][KEYS], best[WAVES * TOKENS][MOST_GROUPS + 1];
    double *const mine = keys[wave * TOKENS + lane / LANES], *const groups = best[wave * TOKENS + lane / LANES];
    auto at = [](int e) { return e + e / 32; };
#pragma unroll
    for (int i = 0; i < VALUES; ++i) mine[at(expert_of(i, l))] = key[i];
    wave_lds();
    const int size = g.experts / g.groups;
    for (int n = l; n < g.groups; n += LANES) {
        double a = NONE, b = NONE;
        for (int i = 0; i < size; ++i) {
            const double k = mine[at(n * size + i)];
            if constexpr (BEST == 2) b = larger(b, smaller(a, k));
            a = larger(a, k);
        }
        double c = without_index(a);
        if (BEST == 2 && b > NONE) c += without_index(b);
        groups[n] = a > NONE ? with_index(c, n) : NONE;
    }
    wave_lds();
    unsigned keep[2] = {0, 0}; // groups by their number
    for (int n = l; n < g.groups; n += LANES) {
        const double k = groups[n];
        int ahead = 0;
        for (int i = 0; i < g.groups; ++i) ahead += groups[i] > k;
        if (ahead < g.kept) keep[n / 32] |= 1u << n % 32;
    }
    keep[0] = or_lanes(keep[0]);
    keep[1] = or_lanes(keep[1]);
    const unsigned long kept = (unsigned long)keep[1] << 32 | keep[0];
    const unsigned reciprocal = ((1u << 21) + size - 1) / size; // e * size < 2^20: the quotient below is e / size
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        const unsigned e = expert_of(i, l);
        if (!(kept >> (e * reciprocal >> 21) % 64 & 1)) key[i] = NONE;
    }
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
    float high = NONE;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        double k = NONE;
#pragma unroll
        for (int j = r * LANES; j < TOP && j < r * LANES + LANES; ++j) k = l == j - r * LANES ? list[j] : k;
        const int j = r * LANES + l;
        id[r] = k > NONE && j < g.chosen ? index_of(k) : -1;
        logit[r] = id[r] >= 0 ? to_acc(row[id[r]]) : (float)NONE;
        high = __builtin_fmaxf(high, logit[r]);
    }
    if constexpr (!SIGMOID && RENORM) { // relative to the largest chosen: their sum is no less than one
        high = max_lanes(high);
        top = high > (float)NONE ? high : 0.f;
        sum = 0;
    }
    double w[ROUNDS], total = 0;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if constexpr (SIGMOID) w[r] = id[r] >= 0 ? 1 / (1 + exp(-(double)logit[r])) : 0;
        else w[r] = id[r] >= 0 ? exp((double)logit[r] - top) : 0;
        total += w[r];
    }
    if constexpr (RENORM) sum = sum_lanes(total);
    const double factor = RENORM || !SIGMOID ? (double)g.scale / sum : (double)g.scale;
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
