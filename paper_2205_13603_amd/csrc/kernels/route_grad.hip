// The gradient of a token's logits from that of its weights (route.hip): with g_j = scale * dw_j, p = softmax(x) or s = sigmoid(x), q the chosen ones over
// their sum,
//   softmax                 dx_e = p_e (sum_{j: id_j = e} g_j - sum_j g_j p_{id_j})
//   softmax, over the sum   dx_{id_j} = q_j (g_j - sum_i g_i q_i)
//   sigmoid                 dx_{id_j} = g_j s_j (1 - s_j)
//   sigmoid, over the sum   dx_{id_j} = (g_j - sum_i g_i q_i) q_j (1 - s_j)
// and zero elsewhere.  Ids outside of the experts are no choices.  A choice that occurs twice adds up, in the order of the choices.  Over the sum, p and s are taken
// relative to the largest chosen one's exponential: s e^-h = e^(min(x, 0) - h) / (1 + e^-|x|), h the largest min(x, 0).
//
// LANES lanes take a token, VALUES experts each: the chosen ones' parts go into the token's row in LDS, from where all lanes take theirs.
//
// What bounds it is memory, up to some 8 MB the launch: bf16, 16384 x 128, all experts of a row involved, 4.6 us; fp32, 16384 x 512 8.3 (34 MB written, 4.0 TB/s).
#include "common.h"
#include "lanes.h"

struct route_grad_args {
    const in_t *x;
    const int *ids;
    const float *dw;
    in_t *dx;
    long x_row, x_inst; // in elements
    int tokens, experts, chosen;
    float scale;
};

constexpr int TOKENS = 64 / LANES, WAVES = THREADS / 64, ROUNDS = (TOP + LANES - 1) / LANES, ROW = LANES * VALUES + 4;
constexpr bool DENSE = !SIGMOID && !RENORM; // all experts of a row take part

__device__ __forceinline__ in_t round_in(float x)
{
#if IN_DT == DT_BF16
    return float_to_bf16(x);
#else
    return (in_t)x;
#endif
}

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const route_grad_args g)
{
    __shared__ __attribute__((aligned(16))) float parts[WAVES * TOKENS][ROW];
    const int lane = threadIdx.x % 64, l = lane % LANES, wave = threadIdx.x / 64, inst = blockIdx.y;
    const int token = ((int)blockIdx.x * WAVES + wave) * TOKENS + lane / LANES;
    const bool live = token < g.tokens;
    const int experts = g.experts;
    const in_t *row = g.x + inst * g.x_inst + (live ? token : g.tokens - 1) * g.x_row;
    const long at = (long)inst * g.tokens + (live ? token : 0);
    float *const mine = parts[wave * TOKENS + lane / LANES];

    // ---- the choices, choice j in lane j % LANES
    int id[ROUNDS];
    float grad[ROUNDS], logit[ROUNDS], high = -__builtin_inff();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int j = r * LANES + l;
        id[r] = -1;
        grad[r] = 0;
        logit[r] = -__builtin_inff();
        if (live && j < g.chosen) {
            const int e = g.ids[at * g.chosen + j];
            if (e >= 0 && e < experts) {
                id[r] = e;
                grad[r] = g.dw[at * g.chosen + j] * g.scale;
                logit[r] = to_acc(row[e]);
            }
        }
        high = __builtin_fmaxf(high, logit[r]);
    }
    float x[VALUES];
    float inverse = 0;
    if constexpr (DENSE) {
        load_logits(row, l, experts, -__builtin_inff(), x);
#pragma unroll
        for (int i = 0; i < VALUES; ++i) high = __builtin_fmaxf(high, x[i]);
    }
    if constexpr (!SIGMOID) {
        high = max_lanes(high);
        high = high > -__builtin_inff() ? high : 0.f; // a row without experts
    } else if constexpr (RENORM) {
        high = __builtin_fminf(max_lanes(high), 0.f);
        high = high > -__builtin_inff() ? high : 0.f;
    }
    if constexpr (DENSE) {
        float sum = 0;
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
            x[i] = expf(x[i] - high);
            sum += x[i];
        }
        sum = sum_lanes(sum);
        inverse = sum == 0 ? 0.f : 1 / sum;
    }
    float part[ROUNDS], dot = 0;
    {
        float s[ROUNDS], sum = 0, slope[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if constexpr (SIGMOID) {
                const float t = expf(-__builtin_fabsf(logit[r])), a = 1 / (1 + t), b = t / (1 + t); // of |x| and -|x|
                // over their sum: times e^-high, so that the largest is one half at least, however small the scores are (fp32 has bits of them down to logits of -103 only)
                if constexpr (RENORM) s[r] = expf(__builtin_fminf(logit[r], 0.f) - high) * a;
                else s[r] = logit[r] < 0 ? b : a;
                slope[r] = logit[r] < 0 ? a : b; // 1 - s
            } else {
                s[r] = expf(logit[r] - high);
                slope[r] = 1;
            }
            if (id[r] < 0) s[r] = 0;
            sum += s[r];
        }
        float over = inverse;
        if constexpr (RENORM) {
            sum = sum_lanes(sum);
            over = sum;
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if constexpr (RENORM) s[r] = id[r] < 0 ? 0.f : s[r] / over;
            else if constexpr (DENSE) s[r] *= over;
            dot += id[r] < 0 ? 0.f : grad[r] * s[r];
        }
        dot = sum_lanes(dot);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if constexpr (DENSE) part[r] = grad[r];
            else if constexpr (RENORM) part[r] = (grad[r] - dot) * s[r] * slope[r];
            else part[r] = grad[r] * s[r] * slope[r];
        }
    }

    // ---- the row's parts: the first of equal choices takes them all
#pragma unroll
    for (int i = 0; i < VALUES; ++i) mine[expert_of(i, l)] = 0;
    float all[ROUNDS];
    bool first[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        all[r] = 0;
        first[r] = id[r] >= 0;
    }
#pragma unroll
    for (int q = 0; q < ROUNDS; ++q)
        for (int i = 0; i < LANES && q * LANES + i < g.chosen; ++i) {
            const int from = (lane / LANES * LANES + i) * 4, other = __builtin_amdgcn_ds_bpermute(from, id[q]);
            const float p = __uint_as_float(__builtin_amdgcn_ds_bpermute(from, __float_as_uint(part[q])));
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                if (other == id[r]) all[r] += p;
                if (other == id[r] && q * LANES + i < r * LANES + l) first[r] = false;
            }
        }
    wave_lds();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (first[r]) mine[id[r]] = all[r];
    wave_lds();

    // ---- results
    in_t *to = g.dx + at * g.experts;
#pragma unroll
    for (int c = 0; c < VALUES; c += CH) {
        const int e = expert_of(c, l);
        logits_t o;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float y = mine[e + i];
            if constexpr (DENSE) y = x[c + i] * inverse * (y - dot);
            o.v[i] = round_in(y);
        }
        if (live && e + CH <= experts) {
            *reinterpret_cast<logits_t *>(to + e) = o;
        } else if (live) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (e + i < experts) to[e + i] = o.v[i];
        }
    }
}
