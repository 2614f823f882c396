// Routing to experts: the operators around the products by expert (which experts a token goes to, the choices sorted by expert, rows to their
// choices and back), on the host.  Their kernels take sizes as arguments: sizes select code by their power of two only.
#pragma once
#include "ms_internal.h"

#include <algorithm>
#include <cstring>

namespace ms {

inline bool is_route(int32_t kind) { return kind == MS_OP_ROUTE || kind == MS_OP_ROUTE_GRAD; }
inline bool moves_rows(int32_t kind) { return kind == MS_OP_SPREAD_ROWS || kind == MS_OP_JOIN_ROWS || kind == MS_OP_JOIN_GRAD; }
inline const char *routing_body_name(int32_t body) { return body == MS_BODY_ROUTE ? "route" : body == MS_BODY_ORDER ? "order" : "expert-rows"; }

// What a launch hands to the kernels; the same structs stand in route.hip, route_grad.hip, order.hip and expert_rows.hip.
struct RouteArgs {
    const void *x, *bias;
    void *ids, *w;
    int64_t x_row, x_inst; // in elements
    int32_t tokens, experts, chosen, groups, kept;
    float scale;
};
struct RouteGradArgs {
    const void *x, *ids, *dw;
    void *dx;
    int64_t x_row, x_inst; // in elements
    int32_t tokens, experts, chosen;
    float scale;
};
struct OrderArgs {
    const void *ids;
    void *offsets, *place, *counts;
    int32_t total, experts, runs;
};
struct RowsArgs {
    const void *x, *place, *w, *c;
    void *y, *s;
    int64_t x_row, x_inst, c_row, c_inst; // in bytes
    int32_t tokens, chosen, cols, rows;
};

inline int64_t power_of_two(int64_t n) // the next, n >= 1
{
    int64_t p = 1;
    while (p < n) p *= 2;
    return p;
}
// dims of ROUTE and ROUTE_GRAD by what they are
inline int64_t route_flags(const ms_op_desc &d) { return d.dims[d.kind == MS_OP_ROUTE ? 6 : 3]; }
inline float route_scale(const ms_op_desc &d)
{
    const uint32_t bits = (uint32_t)d.dims[d.kind == MS_OP_ROUTE ? 7 : 4];
    float f = 1;
    if (bits) memcpy(&f, &bits, sizeof f);
    return f;
}
inline int64_t moved_rows(const ms_op *op) { return op->d.dims[3]; } // of the choices' side
// scales that go with a row in 8 bits
inline int64_t row_scales(const ms_op *op) { return op->d.out_dtype == MS_I8 ? 1 : op->d.out_dtype == MS_F8E4M3 ? scale_blocks(op->N) : 0; }

// The operator in *op, its dims and types checked.
inline int32_t create_routing(const ms_op_desc &d, ms_op *op)
{
    const char *name = op_kind_name(d.kind);
    const int ndims = d.kind == MS_OP_ROUTE ? 8 : d.kind == MS_OP_ROUTE_GRAD || d.kind == MS_OP_JOIN_ROWS ? 5 : d.kind == MS_OP_EXPERT_ORDER ? 3 : 4;
    for (int i = 0; i < 8; ++i) {
        const bool free_form = is_route(d.kind) ? i >= (d.kind == MS_OP_ROUTE ? 6 : 3) : d.kind == MS_OP_JOIN_ROWS && i == 4;
        if (i >= ndims ? d.dims[i] != 0 : !free_form && (d.dims[i] < 1 || d.dims[i] > int64_t(1) << 30))
            return fail(MS_ERR_BAD_ARG, "ms_op_create: dims[%d] of %s = %lld", i, name, (long long)d.dims[i]);
    }
    if (d.stride || d.pad || d.relu || d.dilation || (d.has_bias && d.kind != MS_OP_ROUTE && d.kind != MS_OP_JOIN_ROWS))
        return fail(MS_ERR_BAD_ARG, "ms_op_create: stride/pad/bias/relu/dilation do not apply to %s", name);
    if (d.has_bias != 0 && d.has_bias != 1) return fail(MS_ERR_BAD_ARG, "ms_op_create: has_bias = %d", d.has_bias);
    if (!dtype_size(d.in_dtype) || !dtype_size(d.out_dtype)) return fail(MS_ERR_BAD_ARG, "ms_op_create: bad dtype %d or %d", d.in_dtype, d.out_dtype);
    const bool real = d.in_dtype == MS_F32 || d.in_dtype == MS_F16 || d.in_dtype == MS_BF16, same = d.out_dtype == d.in_dtype;
    bool ok = false;
    switch (d.kind) {
    case MS_OP_ROUTE: ok = real && d.out_dtype == MS_F32; break;
    case MS_OP_ROUTE_GRAD:
    case MS_OP_JOIN_GRAD: ok = real && same; break;
    case MS_OP_EXPERT_ORDER: ok = d.in_dtype == MS_I32 && same; break;
    case MS_OP_SPREAD_ROWS: ok = real ? same || d.out_dtype == MS_I8 || d.out_dtype == MS_F8E4M3 : same && (d.in_dtype == MS_I8 || d.in_dtype == MS_F8E4M3); break;
    case MS_OP_JOIN_ROWS: ok = real && (same || d.out_dtype == MS_F32); break;
    }
    if (!ok) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %s with in %s -> out %s is not supported", name, dtype_name(d.in_dtype), dtype_name(d.out_dtype));
    op->d = d;
    op->nb = 1;
    op->in_size = dtype_size(d.in_dtype);
    op->out_size = dtype_size(d.out_dtype);
    int64_t *a = op->d.a_strides, *b = op->d.b_strides;
    for (int i = 0; i < 3; ++i)
        if (a[i] < 0 || b[i] < 0) return fail(MS_ERR_BAD_ARG, "ms_op_create: negative stride");
    const bool a_zero = !a[0] && !a[1] && !a[2], b_zero = !b[0] && !b[1] && !b[2];
    int64_t cols = 0; // of the tensor that a_strides are those of
    if (is_route(d.kind)) {
        op->M = d.dims[0];
        op->K = cols = d.dims[1];
        op->N = d.dims[2];
        const int64_t flags = route_flags(d), scale = d.dims[d.kind == MS_OP_ROUTE ? 7 : 4];
        if (op->K > MS_MAX_EXPERTS || op->N > MS_MAX_CHOSEN) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %lld of %lld experts, at most %d of %d", (long long)op->N, (long long)op->K, MS_MAX_CHOSEN, MS_MAX_EXPERTS);
        if (op->N > op->K) return fail(MS_ERR_BAD_ARG, "ms_op_create: %lld of %lld experts", (long long)op->N, (long long)op->K);
        if (flags & ~int64_t(MS_ROUTE_SIGMOID | MS_ROUTE_RENORMALISE)) return fail(MS_ERR_BAD_ARG, "ms_op_create: flags %lld of %s", (long long)flags, name);
        const float f = route_scale(d);
        if (scale < 0 || scale > 0x7f7fffff || !(f >= 0x1p-126f)) return fail(MS_ERR_BAD_ARG, "ms_op_create: the scale of %s is no positive finite fp32 number", name);
        if (d.kind == MS_OP_ROUTE) {
            if (d.dims[3] > MS_MAX_GROUPS) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %lld groups of experts, at most %d", (long long)d.dims[3], MS_MAX_GROUPS);
            if (op->K % d.dims[3] || d.dims[4] > d.dims[3] || d.dims[5] > 2)
                return fail(MS_ERR_BAD_ARG, "ms_op_create: %lld groups of %lld experts, %lld kept by the best %lld", (long long)d.dims[3], (long long)op->K, (long long)d.dims[4], (long long)d.dims[5]);
        }
    } else if (d.kind == MS_OP_EXPERT_ORDER) {
        op->K = d.dims[0];
        op->M = d.dims[1];
        op->N = d.dims[2];
        if (op->K > MS_MAX_EXPERTS) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %lld experts, at most %d", (long long)op->K, MS_MAX_EXPERTS);
        if (op->M * op->N > MS_MAX_CHOICES) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %lld choices, at most %d", (long long)(op->M * op->N), MS_MAX_CHOICES);
        cols = op->N;
    } else {
        op->M = d.dims[0];
        op->K = d.dims[1];
        op->N = cols = d.dims[2];
        if (op->K > MS_MAX_ROW_CHOICES) return fail(MS_ERR_UNSUPPORTED, "ms_op_create: %lld choices of a token, at most %d", (long long)op->K, MS_MAX_ROW_CHOICES);
        if (d.kind == MS_OP_JOIN_ROWS && d.dims[4] != 0 && d.dims[4] != 1) return fail(MS_ERR_BAD_ARG, "ms_op_create: dims[4] of %s = %lld", name, (long long)d.dims[4]);
    }
    if (a_zero) a[1] = cols, a[2] = 1;
    if (a[0] || a[2] != 1 || a[1] < cols || a[1] > int64_t(1) << 30 || (d.kind == MS_OP_EXPERT_ORDER && a[1] != cols))
        return fail(MS_ERR_BAD_ARG, "ms_op_create: %s takes a_strides {0, at least %lld, 1}", name, (long long)cols);
    if (d.kind == MS_OP_JOIN_GRAD) {
        if (b_zero) b[1] = cols, b[2] = 1;
        if (b[0] || b[2] != 1 || b[1] < cols || b[1] > int64_t(1) << 30) return fail(MS_ERR_BAD_ARG, "ms_op_create: %s takes b_strides {0, at least %lld, 1}", name, (long long)cols);
    } else if (!b_zero) {
        return fail(MS_ERR_BAD_ARG, "ms_op_create: %s takes no b_strides", name);
    }
    const double rows = moves_rows(d.kind) ? (double)std::max(op->M, moved_rows(op)) : (double)op->M;
    if (rows * (double)std::max(a[1], b[1]) > 1099511627776.0) return fail(MS_ERR_BAD_ARG, "ms_op_create: tensor too large");
    return MS_OK;
}

// Bytes of tensor idx of one instance (-1, -2: outputs); -1: there is none.
inline int64_t routing_tensor_bytes(const ms_op *op, int32_t idx)
{
    const ms_op_desc &d = op->d;
    const int64_t T = op->M, choices = 4 * T * (moves_rows(d.kind) ? op->K : op->N), es = op->in_size, os = op->out_size;
    auto strided = [&](int64_t rows, int64_t stride, int64_t cols) { return ((rows - 1) * stride + cols) * es; };
    switch (d.kind) {
    case MS_OP_ROUTE:
        if (idx == -1 || idx == -2) return choices;
        if (idx == 0) return strided(T, d.a_strides[1], op->K);
        return idx == 1 && d.has_bias ? 4 * op->K : -1;
    case MS_OP_ROUTE_GRAD:
        if (idx == -1) return T * op->K * os;
        if (idx == 0) return strided(T, d.a_strides[1], op->K);
        return idx == 1 || idx == 2 ? choices : -1;
    case MS_OP_EXPERT_ORDER:
        if (idx == -1) return 4 * (op->K + 1);
        return idx == -2 || idx == 0 ? choices : -1;
    case MS_OP_SPREAD_ROWS:
        if (idx == -1) return moved_rows(op) * op->N * os;
        if (idx == -2) return 4 * moved_rows(op) * row_scales(op);
        if (idx == 0) return strided(T, d.a_strides[1], op->N);
        if (idx == 1) return choices;
        return idx == 2 && es == 1 ? 4 * T * row_scales(op) : -1;
    case MS_OP_JOIN_ROWS:
        if (idx == -1) return T * op->N * os;
        if (idx == 0) return strided(moved_rows(op), d.a_strides[1], op->N);
        if (idx == 1 || (idx == 2 && d.dims[4])) return choices;
        return idx == 3 && d.has_bias ? T * op->N * os : -1;
    default:
        if (idx == -1) return moved_rows(op) * op->N * os;
        if (idx == 0) return strided(T, d.a_strides[1], op->N);
        if (idx == -2 || idx == 1 || idx == 2) return choices;
        return idx == 3 ? strided(moved_rows(op), d.b_strides[1], op->N) : -1;
    }
}
// tensors of a launch, some of which an operator may not have
inline int routing_inputs(int32_t kind) { return kind == MS_OP_EXPERT_ORDER ? 1 : kind == MS_OP_ROUTE ? 2 : kind == MS_OP_JOIN_ROWS || kind == MS_OP_JOIN_GRAD ? 4 : 3; }
inline int routing_outputs(int32_t kind) { return kind == MS_OP_ROUTE_GRAD || kind == MS_OP_JOIN_ROWS ? 1 : 2; }

// As if every choice were one of an expert, and had a row.
inline void routing_work(const ms_op *op, double *flop, double *bytes)
{
    const ms_op_desc &d = op->d;
    const double T = (double)op->M, K = (double)op->K, N = (double)op->N, es = op->in_size, os = op->out_size;
    const bool dense = !(route_flags(d) & (MS_ROUTE_SIGMOID | MS_ROUTE_RENORMALISE));
    switch (d.kind) {
    case MS_OP_ROUTE: // exponential, sum, quotient, bias, a comparison
        *flop = 5 * T * K;
        *bytes = T * K * es + 8 * T * N + (d.has_bias ? 4 * K : 0);
        break;
    case MS_OP_ROUTE_GRAD:
        *flop = dense ? 8 * T * K : 8 * T * N;
        *bytes = T * (dense ? K : N) * es + T * K * os + 8 * T * N;
        break;
    case MS_OP_EXPERT_ORDER:
        *flop = 0;
        *bytes = 8 * T * N + 4 * (K + 1);
        break;
    case MS_OP_SPREAD_ROWS: // maximum, quotient, rounding
        *flop = es == os ? 0 : 3 * T * N;
        *bytes = T * N * es + T * K * (N * os + 4 + 4.0 * (double)row_scales(op)) + (es == 1 ? 4 * T * (double)row_scales(op) : 0);
        break;
    case MS_OP_JOIN_ROWS:
        *flop = 2 * T * K * N;
        *bytes = T * K * (N * es + 4 + (d.dims[4] ? 4 : 0)) + T * N * os * (d.has_bias ? 2 : 1);
        break;
    default:
        *flop = 3 * T * K * N;
        *bytes = T * N * es + T * K * (2 * N * es + 12);
    }
}

// ---- variants

inline bool routing_block_fits(const ms_op *op, int64_t code)
{
    if (moves_rows(op->d.kind)) return code >= 1 && code <= 16;
    if (code < 1 || (code & (code - 1))) return false;
    if (is_route(op->d.kind)) return code >= 8 && code <= 64 && power_of_two(op->K) <= 32 * code; // 32 experts of a lane
    return code <= 16;
}

// lanes that share a token (ROUTE, ROUTE_GRAD), choices of a lane (EXPERT_ORDER), wavefronts that share a token (the others)
inline int64_t routing_rule(const ms_op *op)
{
    const int64_t T = op->M;
    if (is_route(op->d.kind)) {
        // Fewer lanes have less to exchange, more of them finish sooner: a wavefront for each SIMD, four where a lane would get 32 experts.  256 experts by groups,
        // choices of 8, by lanes: 1 token 64: 4.5 us, 8: 7.3; 2048 tokens 64: 4.8, 32: 4.4, 8: 7.7; 8192 32: 8.0, 16: 6.9, 8: 7.4; 16384 32: 14.2, 16: 12.3, 8: 13.0.
        // 512 experts, choices of 16, 16384 tokens: 32: 24.1, 16: 21.3.  128 experts, 16384 tokens: 16: 5.1, 8: 4.4.
        int64_t lanes = 64;
        while (lanes > 8 && T * lanes > 64 * (power_of_two(op->K) > 8 * lanes ? 4096 : 1024) && routing_block_fits(op, lanes / 2)) lanes /= 2;
        return lanes;
    }
    if (op->d.kind == MS_OP_EXPERT_ORDER) {
        // One workgroup up to 4096 choices (256 experts, 2400 choices: 4.9 us, in three runs 6.9; 8192: 8.1 and 6.8).  Beyond, the least of what a workgroup takes for
        // its choices, 0.75 us for each of a lane, and for the counts of all runs, 120 bytes a nanosecond, in as many turns as 256 compute units need (256 experts,
        // 131072 choices by 1, 2, 4: 7.1, 7.2, 8.5; 1024 experts: 13.4, 11.2, 11.8; 524288 choices, 256 experts: 18.0, 10.0, 9.8).
        const int64_t n = T * op->N;
        int64_t rounds = 1;
        if (n <= 4096) {
            while (1024 * rounds < n) rounds *= 2;
            return rounds;
        }
        double least = 0;
        for (int64_t r = 1; r <= 16; r *= 2) {
            const int64_t runs = (n + 1024 * r - 1) / (1024 * r);
            const double time = (double)((runs + 255) / 256) * (0.75 * (double)r + (double)(runs * op->K) / 30000);
            if (r == 1 || time < least) least = time, rounds = r;
        }
        return rounds;
    }
    // A chunk of 512 columns for each wavefront, or as many for all of them.  bf16, by wavefronts to a token: 4096 x 2048 into 8-bit integers for 8 choices 4: 14.8 us, 1:
    // 16.6, 16: 22; 8 rows of 4096 x 2048 back 4: 28.4, 1: 35.8; 7 tokens of 4096 columns back 8: 4.5, 1: 16; gradients of 512 x 8192 for 4 choices 16: 12.6, 4: 14.9.
    // fp32, 15276 x 4827 into 8-bit integers for 5 choices 10: 135, 16: 144, 4: 171.
    const int64_t chunks = (op->N + 511) / 512, passes = (chunks + 15) / 16, waves = (chunks + passes - 1) / passes;
    for (int64_t w : {1, 2, 3, 4, 5, 6, 8, 10, 12, 14})
        if (w >= waves) return w;
    return 16;
}

inline int order_threads(const ms_op *op) { return op->M * op->N <= 64 ? 64 : op->M * op->N <= 256 ? 256 : 1024; }
inline int64_t order_runs(const ms_op *op, int64_t rounds)
{
    const int64_t run = order_threads(op) * rounds;
    return (op->M * op->N + run - 1) / run;
}
inline int order_experts(const ms_op *op) { return op->K <= 64 ? 64 : op->K <= 256 ? 256 : 1024; } // that its tables have room for
inline size_t routing_workspace(const ms_op *op, const ms_variant_params *p) // of one instance
{
    if (op->d.kind != MS_OP_EXPERT_ORDER) return 0;
    const int64_t runs = order_runs(op, p->body_tile);
    return runs > 1 ? (size_t)runs * (size_t)op->K * 4u : 0;
}
inline int route_values(const ms_op *op, int64_t lanes) { return (int)std::max<int64_t>(1, power_of_two(op->K) / lanes); }
inline bool route_grouped(const ms_op *op) { return op->d.kind == MS_OP_ROUTE && op->d.dims[3] > 1; }
inline int route_chunk(const ms_op *op, int64_t lanes) { return std::min(16 / op->in_size, route_values(op, lanes)); } // neighbouring experts of a lane
// Experts of a group where its best are found in the registers of lanes: a power of two, whole chunks, up to 16 groups; else 0, by way of LDS.
inline int64_t route_group_size(const ms_op *op, int64_t lanes)
{
    if (!route_grouped(op)) return 0;
    const int64_t size = op->K / op->d.dims[3];
    return power_of_two(size) == size && size >= route_chunk(op, lanes) && lanes * route_values(op, lanes) <= 16 * size ? size : 0;
}
// one expert that speaks for a group, where there are no groups
inline int route_best(const ms_op *op) { return route_grouped(op) ? (int)op->d.dims[5] : 1; }

inline void resolve_routing(const ms_op *op, int64_t code, ms_variant_params *p, int64_t *grid)
{
    p->block_n = p->block_k = 1;
    p->acc_per_thread = 0;
    if (is_route(op->d.kind)) {
        const int values = route_values(op, code), room = (int)code * values;
        p->body = MS_BODY_ROUTE;
        const bool in_lds = route_grouped(op) && !route_group_size(op, code);
        p->waves = in_lds ? 1 : 4;
        p->threads = 64 * p->waves;
        p->block_m = p->threads / (int)code;
        p->block_k = room;
        p->vec = route_chunk(op, code);
        p->acc_per_thread = 2 * values + 2 * (int)power_of_two(op->N);
        p->lds_bytes = op->d.kind == MS_OP_ROUTE_GRAD ? p->block_m * (room + 4) * 4 : in_lds ? p->block_m * (room + room / 32 + 4 + (int)power_of_two(op->d.dims[3]) + 1) * 8 : 0;
        *grid = (op->M + p->block_m - 1) / p->block_m;
    } else if (op->d.kind == MS_OP_EXPERT_ORDER) {
        const int experts = order_experts(op);
        p->body = MS_BODY_ORDER;
        p->threads = order_threads(op);
        p->waves = p->threads / 64;
        p->block_m = p->threads * (int)code;
        p->vec = 1;
        p->acc_per_thread = 2 * (int)code;
        p->lds_bytes = (p->waves + 2) * experts * 4;
        *grid = order_runs(op, code);
    } else {
        p->body = MS_BODY_EXPERT_ROWS;
        p->waves = code < 3 ? 4 : (int)code;
        p->threads = p->waves * 64;
        p->block_m = p->waves / (int)code;
        p->block_k = (int)code * 512;
        p->vec = 8;
        p->acc_per_thread = 32;
        p->lds_bytes = op->d.kind == MS_OP_JOIN_GRAD ? p->waves * 256 : op->d.kind == MS_OP_SPREAD_ROWS ? p->waves * 4 : 0;
        *grid = (op->M + p->block_m - 1) / p->block_m;
    }
}

// the -D options of a variant's kernel, and its file; sizes only by their power of two
template <class Def> std::string routing_spec(const ms_op *op, const ms_variant_params *p, std::vector<std::string> &D, Def def)
{
    const ms_op_desc &d = op->d;
    D.push_back(def("THREADS", p->threads));
    if (is_route(d.kind)) {
        D.push_back(def("LANES", p->body_tile));
        D.push_back(def("VALUES", route_values(op, p->body_tile)));
        D.push_back(def("TOP", power_of_two(op->N)));
        D.push_back(def("SIGMOID", (route_flags(d) & MS_ROUTE_SIGMOID) != 0));
        D.push_back(def("RENORM", (route_flags(d) & MS_ROUTE_RENORMALISE) != 0));
        if (d.kind == MS_OP_ROUTE_GRAD) return "route_grad.hip";
        D.push_back(def("BIAS", d.has_bias));
        D.push_back(def("GROUPED", route_grouped(op)));
        D.push_back(def("BEST", route_best(op)));
        D.push_back(def("GROUP_SIZE", route_group_size(op, p->body_tile)));
        if (route_grouped(op) && !route_group_size(op, p->body_tile)) D.push_back(def("GROUPS", power_of_two(op->d.dims[3])));
        return "route.hip";
    }
    if (d.kind == MS_OP_EXPERT_ORDER) {
        D.push_back(def("ROUNDS", p->body_tile));
        D.push_back(def("EXPERTS", order_experts(op)));
        D.push_back(def("MANY", order_runs(op, p->body_tile) > 1));
        return "order.hip";
    }
    D.pop_back(); // THREADS follow from WAVES
    D.push_back(def("WAVES", p->body_tile));
    D.push_back(def("MODE", d.kind == MS_OP_SPREAD_ROWS ? 0 : d.kind == MS_OP_JOIN_ROWS ? 1 : 2));
    D.push_back(def("RESIDUAL", d.kind == MS_OP_JOIN_ROWS && d.has_bias));
    return "expert_rows.hip";
}

// ---- walks of the kernels: their workgroups, wavefronts and lanes

// How often each position of the reduction of one result is read: experts of a token, choices, columns.
inline int64_t routing_reduction(const ms_op *op) { return op->d.kind == MS_OP_EXPERT_ORDER ? op->M * op->N : op->d.kind == MS_OP_JOIN_GRAD || op->d.kind == MS_OP_SPREAD_ROWS ? op->N : op->K; }
template <class F> void routing_columns(const ms_op *op, const ms_variant_params *p, F column) // of the chunks of 8 that the lanes of a token's wavefronts take
{
    const int64_t step = (int64_t)p->body_tile * 512;
    for (int64_t c0 = 0; c0 < step; c0 += 8)
        for (int64_t c = c0; c < op->N; c += step)
            for (int64_t i = c; i < std::min(op->N, c + 8); ++i) column(i);
}
template <class F> void route_experts(const ms_op *op, const ms_variant_params *p, F expert) // of a token's lanes
{
    const int lanes = p->body_tile, values = route_values(op, lanes), chunk = p->vec;
    for (int l = 0; l < lanes; ++l)
        for (int i = 0; i < values; ++i) {
            const int64_t e = ((int64_t)(i / chunk) * lanes + l) * chunk + i % chunk;
            if (e < op->K) expert(e);
        }
}
// Outputs: ids of ROUTE; of EXPERT_ORDER the offsets, which the first workgroup writes; of SPREAD_ROWS and JOIN_GRAD the rows of a place that
// keeps the order of the choices.
inline void routing_coverage(const ms_op *op, const ms_variant_params *p, int32_t *counts)
{
    const int64_t T = op->M;
    if (op->d.kind == MS_OP_EXPERT_ORDER) {
        if (p->grid[0] > 0)
            for (int64_t e = 0; e <= op->K; ++e) ++counts[e];
        return;
    }
    for (int64_t wg = 0; wg < p->grid[0]; ++wg)
        for (int64_t t = wg * p->block_m; t < std::min(T, (wg + 1) * p->block_m); ++t) {
            if (op->d.kind == MS_OP_ROUTE) {
                for (int l = 0; l < p->body_tile; ++l)
                    for (int64_t j = l; j < op->N; j += p->body_tile) ++counts[t * op->N + j];
            } else if (op->d.kind == MS_OP_ROUTE_GRAD) {
                route_experts(op, p, [&](int64_t e) { ++counts[t * op->K + e]; });
            } else if (op->d.kind == MS_OP_JOIN_ROWS) {
                routing_columns(op, p, [&](int64_t c) { ++counts[t * op->N + c]; });
            } else {
                for (int64_t j = 0; j < op->K && t * op->K + j < moved_rows(op); ++j) routing_columns(op, p, [&](int64_t c) { ++counts[(t * op->K + j) * op->N + c]; });
            }
        }
}
inline void routing_reduction_coverage(const ms_op *op, const ms_variant_params *p, int32_t *counts)
{
    if (is_route(op->d.kind)) {
        route_experts(op, p, [&](int64_t e) { ++counts[e]; });
    } else if (op->d.kind == MS_OP_EXPERT_ORDER) {
        for (int64_t wg = 0; wg < p->grid[0]; ++wg)
            for (int w = 0; w < p->waves; ++w)
                for (int r = 0; r < p->body_tile; ++r)
                    for (int lane = 0; lane < 64; ++lane) {
                        const int64_t n = wg * p->block_m + (w * p->body_tile + r) * 64 + lane;
                        if (n < op->M * op->N) ++counts[n];
                    }
    } else if (op->d.kind == MS_OP_JOIN_ROWS) {
        for (int64_t j = 0; j < op->K; ++j) ++counts[j];
    } else {
        routing_columns(op, p, [&](int64_t c) { ++counts[c]; });
    }
}

} // namespace ms
