// The products of gemm_ragged.hip in tiles of 256 x 256, for launches of so many tiles that they fill the chip.
//
// Persistent workgroups of eight wavefronts in two groups, one of each on every SIMD.  A k step n of 128 bytes is four phases of a group:
//   R0  read the fragments of B and of the first four row tiles A0; request the other four, A1, of step n + 1
//   M0  multiply
//   R1  read the fragments of A1; request three of the six loads of A0 and B of step n + 2
//   M1  multiply; request the other three
// The second group runs the same program one phase behind, so that one wavefront of a SIMD multiplies while the other reads.  Two
// stages of 64 KiB lie in LDS, and each request goes to places that all wavefronts have read: A0 and B of step n in its R0 (the second
// group's is the first one's M0), A1 in its R1.  Requests run on over the end of a tile, into the next one's operands, while results leave.
//
// Whole tiles of a last round that would leave most workgroups without one, and the rests of experts' rows of up to 128, are made in
// quarters at the end, by all eight wavefronts of a workgroup each.
//
// What bounds it: the clock under load (1.8 to 2.0 GHz) at 53 to 57 % of the matrix cores' cycles in long products of 8- and 16-bit floats, and what a tile's end leaves
// uncovered, 9 us of stores and first reads for each round of tiles.  8192^3 in 8 bits 450 to 490 us by card and by what ran before (2.2 to 2.4
// PFLOP/s; loads alone 338, products alone 215 at this clock); bf16, 8 experts, 8192 x 4096 x 4096 230 to 246 (1.1 to 1.2); 8 bits, 32 experts, 16384 x
// 2048 x 4096 168 to 179 (1.6); gradient of 8 experts, 4096 x 2048 into fp32 147 to 174 by the experts' rows (0.8 to 0.9, and 2.1 to 2.5 TB/s).
// 8-bit integers: 8192^3 380 to 430 by card (2.6 to 2.9 Pop/s, the matrix cores busy 71 % of the cycles), 32 experts, 16384 x 2048 x 4096 139 to 157 (1.8 to 2.0).
// Their scales meet the sums once, at the end; they come in by way of LDS with a tile's first step (read there instead, each tile waited 4 us for them).
//
// 8-bit floats: the products of a block of 128 k values are one instruction, whose four results per lane are added to the sums
// with their scales, SA of the lane's row times SB of the wavefront's columns, while the matrix core works on the next.  Scales are
// requested in R1, two steps ahead, in runs that share two places by turns (ragged_schedule.h).
#include "common.h"
#include "ragged.h"
#define ALIGNED 1
#include "ragged_tile.h"

constexpr int BM = 256, BN = 256, WJ = 4, NW = 8, THREADS = NW * 64, TM = 8, TN = 4, BK = 128 / ES;
constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
constexpr bool SCALED = IN_DT == DT_F8E4M3, LINE_SCALED = IN_DT == DT_I8; // scales of blocks of k; of rows and columns
constexpr int KB = SCALE_RUN, LS = KB * BM / 64 / NW; // k blocks whose scales are in LDS at a time, twice; loads of a wavefront for them
constexpr int SC_BYTES = SCALED ? KB * BM * 4 : 0, LINE_BYTES = LINE_SCALED ? (BM + BN) * 4 : 0, SB_BYTES = SCALED ? 256 : 0, OS = sizeof(out_t);
constexpr int SC_AT = 2 * STAGE, SB_AT = SC_AT + 2 * SC_BYTES, LINES_AT = SB_AT + 2 * SB_BYTES, TABLE_AT = LINES_AT + 3 * LINE_BYTES;
constexpr int LDS_BYTES = TABLE_AT + (WGRAD ? 2048 : GROUPED ? 4096 + 2048 : 0);
typedef ragged_tile<128, 128, 2, 2, 2> quarter;
static_assert(quarter::LDS_BYTES <= TABLE_AT, "quarters lie where whole tiles did");
static_assert(LDS_BYTES == LDS_HOST, "the host's count of LDS");

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const ragged_args g)
{
    __shared__ __attribute__((aligned(1024))) char lds[LDS_BYTES];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wi = wave / WJ, wj = wave % WJ, lrow = lane % 16, lgrp = lane / 16;
    const bool late = wi == 1; // the group one phase behind
    const int inst = blockIdx.y;
    const int *offsets = GROUPED ? g.offsets + (long)inst * (g.experts + 1) : nullptr;
    int *table = reinterpret_cast<int *>(lds + TABLE_AT);
    unsigned short *halves = reinterpret_cast<unsigned short *>(table + 1024), *order = reinterpret_cast<unsigned short *>(table);

    // ---- the tiles.  Products: whole ones, of up to 256 rows but more than 128, then quarters of 128 x 128: the rest of each expert's rows,
    // and the whole tiles of a last round that would leave most workgroups without one.
    const unsigned nt = (unsigned)(g.cols + BN - 1) / BN;
    unsigned total, half_rows = 0;
    rounds_t rounds = {0, 0};
    if constexpr (WGRAD) {
        // experts by their rows, most first, and every other round backwards: the workgroups' sums of rows are then nearly the same
        int *rows = reinterpret_cast<int *>(lds);
        for (int e = tid; e < g.experts; e += THREADS) {
            const range_t r = rows_of(offsets, e, g.depth);
            rows[e] = r.last - r.first;
        }
        barrier();
        for (int e = tid; e < g.experts; e += THREADS) {
            int place = 0;
            for (int j = 0; j < g.experts; ++j) place += rows[j] > rows[e] || (rows[j] == rows[e] && j < e);
            order[place] = (unsigned short)e;
        }
        barrier();
        total = tiles_of<BM, BN>(g, table);
    } else {
        int full_rows;
        if (GROUPED) {
            if (wave == 0) count_wide_tiles(offsets, g.experts, g.rows, lane, table, halves);
            barrier();
            full_rows = table[g.experts - 1];
            half_rows = uniform((unsigned)halves[g.experts - 1]);
        } else {
            full_rows = whole_tiles(g.rows);
            half_rows = half_left(g.rows);
        }
        rounds = split_rounds(uniform((unsigned)full_rows) * nt, half_rows * nt, gridDim.x);
        total = rounds.whole;
    }
    // the tile of a workgroup's f-th turn, f counted in steps of the grid; false: there is nothing to do
    auto tile_of = [&](unsigned f, tile_t &t) {
        if (WGRAD) {
            f = back_and_forth(f, gridDim.x);
            return f < total && decode<BM, BN>(g, offsets, table, f, lane, t, order);
        }
        return decode<BM, BN, true>(g, offsets, table, run_of_xcd(f, total), lane, t);
    };
    const unsigned turns = WGRAD ? (total + gridDim.x - 1) / gridDim.x * gridDim.x : total;
    auto make_quarters = [&]() {
        if constexpr (!WGRAD) {
            for (unsigned f = blockIdx.x; f < rounds.quarters; f += gridDim.x) {
                const quarter_t q = quarter_of(run_of_xcd(f, rounds.quarters), rounds, half_rows * nt, nt);
                tile_t t;
                bool any;
                if (!q.half) {
                    any = decode<BM, BN, true>(g, offsets, table, q.tile, lane, t);
                    t.row += q.row;
                    t.rows -= q.row;
                    t.col += q.col;
                } else {
                    tile_at where = {0, 0, 1};
                    int first = 0, end = g.rows;
                    if (GROUPED) {
                        where = find_tile(halves, g.experts, (int)q.tile, lane);
                        const range_t r = rows_of(offsets, where.expert, g.rows);
                        first = __builtin_amdgcn_readfirstlane(r.first);
                        end = __builtin_amdgcn_readfirstlane(r.last);
                    }
                    const int whole = whole_tiles(end - first) * 256;
                    t = {where.expert, first + whole, end - first - whole, (int)q.col, 0, g.depth};
                    any = true;
                }
                t.rows = t.rows < 128 ? t.rows : 128;
                if (!any || t.rows <= 0 || t.col >= g.cols) continue;
                barrier(); // the LDS of the tile before is free
                quarter::make(g, inst, t, lds);
            }
        }
    };
    const char *const a_ = g.a + inst * g.a_inst, *const b_ = g.b + inst * g.b_inst;
    const unsigned lds0 = lds_address(lds);

    // ---- the cursor of the loads: step lk of tile lt, the lf-th of the launch, into stage wr; a tile's steps are counted from `first` up to lsteps
    tile_t lt;
    unsigned lf = blockIdx.x;
    int lk = 0, lsteps = 0, wr = 0, lchunk = 0; // lchunk: which of the two places its run of scales goes to
    int llines = 0; // which of the three places its tile's scales of rows and columns go to: the cursor may be two tiles ahead of the products
    bool more = true;                           // false: past the last tile, the last step is requested again (never read)
    const char *la, *lb;                        // first row of the step's operands
    unsigned va[4], vb[4]; // of A's parts and B's halves two loads each, from la and lb
    const int chunk = lane % 8 ^ lane / 8;
    const int a_k = wave * 4 + lane / 16, b_k = wave * 2 + lane / 32; // k row of a transposed operand's load 0
#if IN_DT == DT_F8E4M3
    const int blocks = (g.depth + 127) / 128, col_blocks = (g.cols + 127) / 128, first = first_step(blocks);
    unsigned vsa, vsb; // of the scales: row wave / 2 * 64 + lane; lane = 8 * (block of columns) + block of k
    static_assert(KB == 8 && LS == 4, "two wavefronts share 64 rows");
#else
    constexpr int first = 0; // no scales
#endif
    // What is computed once for a tile stays there: hoisted out of the loops its parts would take the registers of the products.
    auto opaque = [](int x) {
        asm volatile("" : "+v"(x));
        return x;
    };
    auto scalar = [](const char *p) { return (const char *)uniform(p); };
    // the next tile with something to multiply, from the lf-th on; false: there is none
    auto place = [&]() {
        const int lane = opaque(tid % 64), chunk = lane % 8 ^ lane / 8, a_k = wave * 4 + lane / 16, b_k = wave * 2 + lane / 32;
        for (;; lf += gridDim.x) {
            if (lf >= turns) return false;
            tile_t t; // lt stays as it is where there is none: the loads past the end are its last step's
            if (tile_of(lf, t) && t.depth > 0) {
                lt = t;
                break;
            }
        }
        lk = first;
        lsteps = first + (lt.depth + BK - 1) / BK;
        la = scalar(a_ + (A_KC ? (long)lt.row * g.a_row : (long)lt.k0 * g.a_row + (long)lt.row * ES));
        lb = scalar(b_ + lt.expert * g.b_expert + (B_KC ? (long)lt.col * g.b_row : (long)lt.k0 * g.b_row + (long)lt.col * ES));
        const int cols = g.cols - lt.col;
#pragma unroll
        for (int l = 0; l < 4; ++l) {
            if (A_KC) {
                const int r = l % 2 * 128 + l / 2 * 64 + wave * 8 + lane / 8;
                va[l] = r < lt.rows ? (unsigned)(r * (int)g.a_row + chunk * 16) : OUTSIDE;
            } else {
                // a part is 64 rows of k by the 128 columns of its row tiles
                const int k = a_k + l % 2 * 32, c0 = (((lane % 16 >> 1) ^ (k % 4 | k / 2 & 4)) << 4) + lane % 2 * 8, c = c0 + c0 / 64 * 64 + l / 2 * 64;
                va[l] = c < lt.rows ? (unsigned)(k * (int)g.a_row + c * ES) : OUTSIDE;
            }
            if (B_KC) {
                const int r = l * 64 + wave * 8 + lane / 8;
                vb[l] = r < cols ? (unsigned)(r * (int)g.b_row + chunk * 16) : OUTSIDE;
            } else {
                const int k = b_k + l * 16, c = (((lane % 32 >> 1) ^ (k % 4 | k / 2 & 4)) << 4) + lane % 2 * 8;
                vb[l] = c < cols ? (unsigned)(k * (int)g.b_row + c * ES) : OUTSIDE;
            }
        }
#if IN_DT == DT_F8E4M3
        vsa = wave / 2 * 64 + lane < lt.rows ? (unsigned)((wave / 2 * 64 + lane) * blocks) * 4 : OUTSIDE;
        vsb = (lane < 16) & (lt.col / 128 + lane / KB < col_blocks) ? (unsigned)(lane / KB * blocks + lane % KB) * 4 : OUTSIDE;
#endif
        return true;
    };
    // load l of step lk: 0, 1 of A0, 2 to 5 of B, 6, 7 of A1
    auto load = [&](int l, bool inner = false) { // inner: a step that the tile's reduction fills
        const int here = lt.depth - (lk - first) * BK;
        const bool of_a = l < 2 || l >= 6;
        const int n = l < 2 ? l : l >= 6 ? l - 4 : l - 2;
        unsigned v = of_a ? va[n] : vb[n];
        if (!inner && here < BK) { // behind the last k
            const int k = of_a ? (A_KC ? chunk * (16 / ES) : a_k + n % 2 * 32) : (B_KC ? chunk * (16 / ES) : b_k + n * 16);
            if (k >= here) v = OUTSIDE;
        }
        unsigned at = lds0 + wr * STAGE + wave * 1024;
        if (of_a) at += A_KC ? n % 2 * 16384 + n / 2 * 8192 : n / 2 * 16384 + n % 2 * 8192;
        else at += A_BYTES + n * 8192;
        gather_lds16_at(buffer_at(of_a ? la : lb), v, at);
    };
    auto load_scales = [&](bool inner = false) { // inner: not a tile's first step
#if IN_DT == DT_F8E4M3
        if (inner ? lk % KB == 0 : starts_run(lk, first)) {
            const int start = (inner ? lk : head_of_run(lk)) - first; // block at the head of the place: none ahead of block 0
            const char *const lsa = scalar((const char *)g.sa + inst * g.sa_inst + (long)lt.row * blocks * 4);
            const char *const lsb = scalar((const char *)g.sb + inst * g.sb_inst + ((long)lt.expert * col_blocks + lt.col / 128) * blocks * 4);
            // 64 rows of a wavefront, the blocks of one line after each other
            const int k0 = wave % 2 * LS;
            const unsigned at = lds0 + SC_AT + lchunk * SC_BYTES + (k0 * BM + wave / 2 * 64) * 4;
#pragma unroll
            for (int l = 0; l < LS; ++l) gather_lds4(buffer_at(lsa + (start + k0 + l) * 4), (unsigned)(start + k0 + l) < (unsigned)blocks ? vsa : OUTSIDE, at + l * BM * 4);
            if (wave == 0) gather_lds4(buffer_at(lsb + start * 4), (unsigned)(start + lane % KB) < (unsigned)blocks ? vsb : OUTSIDE, lds0 + SB_AT + lchunk * SB_BYTES);
        }
#elif IN_DT == DT_I8
        if (!inner && lk == first) { // 64 rows of four wavefronts, 64 columns of the others, ahead of the tile's first step
            const bool of_rows = wave < 4;
            const char *const from = scalar(of_rows ? (const char *)g.sa + inst * g.sa_inst + (long)lt.row * 4 : (const char *)g.sb + inst * g.sb_inst + ((long)lt.expert * g.cols + lt.col) * 4);
            const int n = wave % 4 * 64 + lane;
            gather_lds4(buffer_at(from), n < (of_rows ? lt.rows : g.cols - lt.col) ? (unsigned)n * 4 : OUTSIDE, lds0 + LINES_AT + llines * LINE_BYTES + wave * 256);
        }
#endif
    };
    auto next_step = [&]() { // inside the tile
        wr ^= 1;
        ++lk;
        la += A_KC ? 128 : BK * g.a_row;
        lb += B_KC ? 128 : BK * g.b_row;
        if (SCALED && lk % KB == 0) lchunk ^= 1;
    };
    auto advance = [&]() {
        if (more && lk + 1 < lsteps) {
            next_step();
            return;
        }
        wr ^= 1;
        if (more) {
            lf += gridDim.x;
            more = place();
            if (more) {
                lchunk ^= 1;
                llines = llines == 2 ? 0 : llines + 1;
            }
        }
    };
    const tile_t none = {0, 0, 0, 0, 0, 0};
    lt = none;

    // ---- fragments
    sum4_t acc[TM][TN];
    frag_t fa[KQ][TM / 2], fb[KQ][TN];
    float fs[TM / 2];
    auto frag_kc = [&](const char *p, int q) {
        frag_t f;
        if (KQ == 2) {
            f.v[0] = *reinterpret_cast<const u4_t *>(p + ((q * 4 + lgrp) ^ lrow % 8) * 16);
        } else {
#pragma unroll
            for (int h = 0; h < (int)(sizeof(frag_t) / 16); ++h) f.v[h] = *reinterpret_cast<const u4_t *>(p + ((h * 4 + lgrp) ^ lrow % 8) * 16);
        }
        return f;
    };
    auto frag_tr = [&](const char *p, int width, int granule, int q) {
        frag_t f;
#if IN_DT != DT_F8E4M3
        typedef short tr4_t __attribute__((ext_vector_type(4)));
        struct { tr4_t v[2]; } x;
        const int r = lrow / 4, swz = r | (lgrp & 1) << 2;
        const char *at = p + (q * 32 + lgrp * 8 + r) * width * 2 + (granule ^ swz) * 32 + lrow % 4 * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) x.v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) tr4_t *)(at + h * 4 * width * 2));
        f.v[0] = __builtin_bit_cast(u4_t, x);
#endif
        return f;
    };
    auto read_a = [&](int stage, int half) {
        const char *p = lds + stage * STAGE;
#pragma unroll
        for (int q = 0; q < KQ; ++q)
#pragma unroll
            for (int i = 0; i < TM / 2; ++i)
                fa[q][i] = A_KC ? frag_kc(p + (wi * 128 + half * 64 + i * 16 + lrow) * 128, q) : frag_tr(p + half * 16384, 128, wi * 4 + i, q);
    };
    auto read_b = [&](int stage) {
        const char *p = lds + stage * STAGE + A_BYTES;
#pragma unroll
        for (int q = 0; q < KQ; ++q)
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[q][j] = B_KC ? frag_kc(p + (wj * 64 + j * 16 + lrow) * 128, q) : frag_tr(p, 256, wj * 4 + j, q);
    };
    auto read_scales = [&](int half, int k, int place) {
#if IN_DT == DT_F8E4M3
        const float *sc = reinterpret_cast<const float *>(lds + SC_AT + place * SC_BYTES) + k % KB * BM + wi * 128 + half * 64 + lrow;
        const float sj = reinterpret_cast<const float *>(lds + SB_AT + place * SB_BYTES)[wj / 2 * KB + k % KB];
#pragma unroll
        for (int i = 0; i < TM / 2; ++i) fs[i] = sc[i * 16] * sj;
#endif
    };
    // the products of four row tiles, in M1 with three loads between them
    auto multiply = [&](int half, bool inner) {
        __builtin_amdgcn_s_setprio(1);
#if IN_DT == DT_F8E4M3
        constexpr int N = TM / 2 * TN, LAG = 3; // results wait for the matrix core while it works on LAG further products
        f4_t d[LAG + 1];
#pragma unroll
        for (int m = 0; m < N + LAG; ++m) {
            if (m < N) d[m % (LAG + 1)] = mfma(fb[0][m % TN], fa[0][m / TN], f4_t{0, 0, 0, 0});
            __builtin_amdgcn_sched_barrier(0); // the product first
            if (half == 1 && m % 5 == 3 && m < 15) load(3 + m / 5, inner);
            if (m >= LAG) {
                const int o = m - LAG;
                f4_t &sum = acc[half * 4 + o / TN][o % TN];
                sum = __builtin_elementwise_fma(d[o % (LAG + 1)], f4_t{fs[o / TN], fs[o / TN], fs[o / TN], fs[o / TN]}, sum);
                asm volatile("" : "+v"(sum)); // here, not where the sum is read next: 16 products in registers would be 64
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#else
#pragma unroll
        for (int q = 0; q < KQ; ++q)
#pragma unroll
            for (int i = 0; i < TM / 2; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    acc[half * 4 + i][j] = mfma(fb[q][j], fa[q][i], acc[half * 4 + i][j]);
                    if (half == 1 && j == 1 && (q * 4 + i) % 3 == 0) load(3 + (q * 4 + i) / 3, inner);
                }
#endif
        __builtin_amdgcn_s_setprio(0);
    };
    auto zero = [&]() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = sum4_t{0, 0, 0, 0};
    };
    auto store = [&](const tile_t &t, int place) {
        const int lane = opaque(tid % 64), lrow = lane % 16, lgrp = lane / 16;
        char *c = g.c + inst * g.c_inst + (WGRAD ? (long)t.expert * g.rows * g.cols * OS : 0);
        const int cols = g.cols - t.col < BN ? g.cols - t.col : BN;
        const float *const lines = reinterpret_cast<const float *>(lds + LINES_AT + place * LINE_BYTES);
        f4_t sj[TN];
        float si[TM];
#pragma unroll
        for (int j = 0; j < TN; ++j) sj[j] = LINE_SCALED ? *reinterpret_cast<const f4_t *>(lines + BM + wj * 64 + j * 16 + lgrp * 4) : f4_t{1.f, 1.f, 1.f, 1.f};
#pragma unroll
        for (int i = 0; i < TM; ++i) si[i] = LINE_SCALED ? lines[wi * 128 + i * 16 + lrow] : 1.f;
#if OUT_DT == DT_F32
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            f4_t x[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) x[j] = results(acc[i][j], si[i], sj[j]);
            rows_together(x);
            const int col = wj * 64 + lrow / 4 * 16 + lgrp * 4;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int r = wi * 128 + i * 16 + s * 4 + lrow % 4;
                if (r < t.rows && col < cols) store4<true>(c + ((long)(t.row + r) * g.cols + t.col + col) * OS, x[s], cols - col);
            }
        }
#else
        // A row's 64 columns leave as one line, put together between lanes (by way of LDS: 8-bit integers, 32 experts 148 us instead of 145).  Neighbouring column tiles swap their quads with neighbouring quads of
        // lanes, so that a lane has eight columns of a row; then the upper eight rows' left halves with the lower ones' right halves.  Where rows begin off 16
        // bytes stores of neighbouring lanes have to be neighbours too: there lanes change places once more (bf16, 8192 x 8191 x 512 97 -> 78 us).
        typedef unsigned u2_t __attribute__((ext_vector_type(2)));
        struct oct_t { unsigned w[4]; };
        const bool off = g.cols % 8 != 0;
        const int col = wj * 64 + (off ? lane % 8 * 8 : lrow / 8 * 32 + lgrp % 2 * 16 + lgrp / 2 * 8);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            unsigned of[2][4];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                u2_t w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    struct { out_t v[4]; } o;
                    const f4_t x = results(acc[i][p * 2 + e], si[i], sj[p * 2 + e]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o.v[v] = round_out(x[v]);
                    w[e] = __builtin_bit_cast(u2_t, o);
                }
                const u2_t lo = __builtin_amdgcn_permlane16_swap(w[0][0], w[1][0], false, false), hi = __builtin_amdgcn_permlane16_swap(w[0][1], w[1][1], false, false);
                of[p][0] = lo[0], of[p][1] = hi[0], of[p][2] = lo[1], of[p][3] = hi[1];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                oct_t o;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    o.w[w] = h ? __builtin_amdgcn_update_dpp(of[1][w], of[0][w], 0x128, 0xf, 0x3, false)  // the other half is that of the lane eight on
                               : __builtin_amdgcn_update_dpp(of[0][w], of[1][w], 0x128, 0xf, 0xc, false);
                if (off) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) o.w[w] = __builtin_amdgcn_ds_bpermute((lane / 8 + lane % 8 / 4 * 8 + lane % 4 / 2 * 16 + lane % 2 * 32) * 4, o.w[w]);
                }
                const int row = wi * 128 + i * 16 + h * 8 + (off ? lane / 8 : lrow % 8);
                if (row < t.rows && col < cols) {
                    char *dst = c + ((long)(t.row + row) * g.cols + t.col + col) * OS;
                    if (col + 8 <= cols) {
                        stream_out(dst, o);
                    } else {
                        struct { out_t v[8]; } each = __builtin_bit_cast(decltype(each), o);
#pragma unroll
                        for (int v = 0; v < 8; ++v)
                            if (col + v < cols) reinterpret_cast<out_t *>(dst)[v] = each.v[v];
                    }
                }
            }
        }
#endif
    };

    // What has to have landed at the end of a phase, and how many younger loads may still be in flight (those of scales and stores, not
    // counted, make a wait longer): at the end of R0 A1 of this step, behind it A0 and B (6) and A1 (2) of the next; at the end of R1 A0 and B of the
    // next step, behind them its A1 and the three of this phase.
    constexpr int KEEP_R0 = 8, KEEP_R1 = 5;
    if (!place()) more = false;
    tile_t ct = lt; // the tile whose products are made
    // tiles without a reduction (an expert without rows) hold zeros
    auto empty_tiles = [&]() {
        if (!WGRAD) return;
        zero();
        tile_t t;
        for (unsigned f = blockIdx.x; f < turns; f += gridDim.x)
            if (tile_of(f, t) && t.depth <= 0) store(t, 0);
    };
    if (!more) {
        empty_tiles();
        make_quarters();
        return;
    }
    unsigned cf = lf; // the tile of the products, by its number
    load_scales();
#pragma unroll
    for (int l = 0; l < 8; ++l) load(l);
    advance();
    load_scales();
#pragma unroll
    for (int l = 0; l < 6; ++l) load(l);
    DL_WAIT_VM(8); // A0 and B of the first step
    barrier();
    if (late) barrier();
    int rd = 0, cchunk = 0, clines = 0;
    zero();
    for (;;) {
        const int steps = first + (ct.depth + BK - 1) / BK;
        int k = first;
        auto step = [&](auto moves_on, bool inner) {
            if (SCALED && k && k % KB == 0) cchunk ^= 1;
            read_b(rd);
            read_a(rd, 0);
            read_scales(0, k, cchunk);
            load(6, inner);
            load(7, inner);
            DL_WAIT_VM(KEEP_R0);
            barrier();
            multiply(0, inner);
            moves_on();
            barrier();
            read_a(rd, 1);
            read_scales(1, k, cchunk);
            load_scales(inner);
            load(0, inner);
            load(1, inner);
            load(2, inner);
            DL_WAIT_VM(KEEP_R1);
            barrier();
            multiply(1, inner);
            barrier();
            rd ^= 1;
            ++k;
        };
        // the cursor of a tile of one step is in the next tile from the start, which is as deep (products) or need not be (gradients)
        const bool reaches = !WGRAD || steps > 1;
        // the last steps, in which the cursor goes on to the next tile, in a loop of their own: its registers are not the others'
#pragma unroll 1
        while (reaches && more && lk + 2 < lsteps) step(next_step, true); // requests of steps lk and lk + 1, neither the tile's last
#pragma unroll 1
        while (k < steps) step(advance, false);
        store(ct, clines);
        zero();
        // the next tile of the products: the one that the cursor found
        bool any = false;
        for (cf += gridDim.x; cf < turns; cf += gridDim.x)
            if (tile_of(cf, ct) && ct.depth > 0) {
                any = true;
                break;
            }
        if (!any) break;
        cchunk ^= 1;
        clines = clines == 2 ? 0 : clines + 1;
    }
    if (!late) barrier(); // the other group's last phase
    DL_WAIT_VM(0);        // loads past the end land before the workgroup's LDS is released
    empty_tiles();
    barrier();
    make_quarters();
}
