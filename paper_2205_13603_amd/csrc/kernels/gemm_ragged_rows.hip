// Products of few rows (of each expert) with matrices whose rows run along k: a decoding step.
//
//   C[t][j] = sum_k A[t][k] B[e(t)][j][k]           8-bit floats: sum over blocks of 128 k of SA[t][b] SB[e][j/128][b] (block's sum)
//
// What bounds it is reading B once.  The wavefronts of a workgroup split the reduction of its BM x BN tile, blocks of 128 bytes in
// turn, and add their sums up in LDS at the end, in the order of their numbers.  Each has a ring of LDS stages of its own, which
// loads fill directly and only it reads: no barrier ahead of the end, no registers for data in flight, and eight lanes of a load take a
// whole line (fragments loaded as the matrix cores take them touch 16 rows with 64 lanes and cost four times the address lookups).
// Measured: bf16, 16 rows of 12 experts, 1024 x 2048 by 16 x 16 9.4 us, 5.4 TB/s; 8 bits, 4 x 4096 x 4096 5.0, of which the launch is 4;
// 16 x 8192 x 8192 11.9, 5.6 TB/s.
#include "common.h"
#include "ragged.h"

constexpr int NW = WI, THREADS = NW * 64, MT = BM / 16, NC = BN / 16, LA = BM / 8, LB = BN / 8;
constexpr bool SCALED = IN_DT == DT_F8E4M3;
constexpr int LOADS = LA + LB + (SCALED ? 2 : 0), SLOT = (BM + BN) * 128 + (SCALED ? 512 : 0);
constexpr int RING = NW * STAGES * SLOT, SUMS = NW * BM * BN * 4, TABLE_AT = RING > SUMS ? RING : SUMS;
constexpr int LDS_BYTES = TABLE_AT + (GROUPED ? 4096 : 0);
static_assert(LDS_BYTES == LDS_HOST, "the host's count of LDS");
static_assert(STAGES <= 2 && (STAGES - 1) * LOADS < 64 && BM <= 64 && 128 % BN == 0, "see ragged_tile()");

extern "C" __global__ void __launch_bounds__(THREADS) ms_kernel(const ragged_args g)
{
    __shared__ __attribute__((aligned(1024))) char lds[LDS_BYTES];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), lrow = lane % 16, lgrp = lane / 16;
    const int inst = blockIdx.y, nt = (g.cols + BN - 1) / BN;

    // ---- which tile: an expert's row tiles of one run of columns follow each other on an XCD
    int expert = 0, row, rows, col;
    {
        tile_at where = {0, 0, (g.rows + BM - 1) / BM};
        unsigned of;
        range_t r = {0, g.rows};
        if (GROUPED) {
            int *table = reinterpret_cast<int *>(lds + TABLE_AT);
            if (!find_row_tile(g.offsets + (long)inst * (g.experts + 1), g.experts, g.rows, BM, nt, blockIdx.x, lane, wave, table, where, of, r)) return;
            expert = where.expert;
        } else {
            of = run_of_xcd(blockIdx.x, (unsigned)where.tiles * nt);
        }
        row = r.first + of % (unsigned)where.tiles * BM;
        col = of / (unsigned)where.tiles * BN;
        rows = r.last - row < BM ? r.last - row : BM;
        if (rows <= 0) return; // offsets that decrease
    }
    const int cols = g.cols - col < BN ? g.cols - col : BN;
    const char *a = g.a + inst * g.a_inst + (long)row * g.a_row, *b = g.b + inst * g.b_inst + expert * g.b_expert + (long)col * g.b_row;

    // ---- 8 rows of 128 bytes per load instruction, 16-byte chunks swizzled by the row so that a fragment read meets each bank once
    unsigned avoff[LA], bvoff[LB];
    const int chunk = lane % 8 ^ lane / 8;
#pragma unroll
    for (int l = 0; l < LA; ++l) avoff[l] = l * 8 + lane / 8 < rows ? (unsigned)((l * 8 + lane / 8) * (int)g.a_row + chunk * 16) : OUTSIDE;
#pragma unroll
    for (int l = 0; l < LB; ++l) bvoff[l] = l * 8 + lane / 8 < cols ? (unsigned)((l * 8 + lane / 8) * (int)g.b_row + chunk * 16) : OUTSIDE;
    const int bytes = g.depth * ES, blocks = (bytes + 127) / 128;
    const int mine = blocks > wave ? (blocks - wave + NW - 1) / NW : 0; // blocks of this wavefront
    const unsigned ring = lds_address(lds) + wave * STAGES * SLOT;
    const char *const ring_p = lds + wave * STAGES * SLOT;
#if IN_DT == DT_F8E4M3
    const rsrc_t sa = buffer_at((const char *)g.sa + inst * g.sa_inst + (long)row * blocks * 4);
    const rsrc_t sb = buffer_at((const char *)g.sb + inst * g.sb_inst + ((long)expert * ((g.cols + 127) / 128) + col / 128) * blocks * 4);
#endif
    auto load = [&](int i, int stage) {
        const int k = wave + i * NW, here = bytes - k * 128;
        const rsrc_t ra = buffer_at(a + (long)k * 128), rb = buffer_at(b + (long)k * 128);
        const unsigned at = ring + stage * SLOT;
        const bool tail = here < 128;
#pragma unroll
        for (int l = 0; l < LB; ++l) gather_lds16_at(rb, tail && chunk * 16 >= here ? OUTSIDE : bvoff[l], at + BM * 128 + l * 1024);
#pragma unroll
        for (int l = 0; l < LA; ++l) gather_lds16_at(ra, tail && chunk * 16 >= here ? OUTSIDE : avoff[l], at + l * 1024);
#if IN_DT == DT_F8E4M3
        gather_lds4(sa, lane < rows ? (unsigned)(lane * blocks + k) * 4 : OUTSIDE, at + (BM + BN) * 128);
        gather_lds4(sb, lane == 0 ? (unsigned)k * 4 : OUTSIDE, at + (BM + BN) * 128 + 256);
#endif
    };
    f4_t acc[MT][NC];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NC; ++j) acc[i][j] = f4_t{0, 0, 0, 0};

#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < mine) load(s, s);
    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const int behind = mine - 1 - i; // blocks whose loads may still be in flight
        if (behind >= STAGES - 1) DL_WAIT_VM((STAGES - 1) * LOADS);
        else DL_WAIT_VM(0);
        asm volatile("" ::: "memory");
        const char *p = ring_p + stage * SLOT;
        frag_t fa[KQ][MT], fb[KQ][NC];
        auto frag = [&](const char *r, int q) {
            frag_t f;
            if (ES == 2) {
                f.v[0] = *reinterpret_cast<const u4_t *>(r + ((q * 4 + lgrp) ^ lrow % 8) * 16);
            } else {
#pragma unroll
                for (int h = 0; h < (int)(sizeof(frag_t) / 16); ++h) f.v[h] = *reinterpret_cast<const u4_t *>(r + ((h * 4 + lgrp) ^ lrow % 8) * 16);
            }
            return f;
        };
#pragma unroll
        for (int q = 0; q < KQ; ++q) {
#pragma unroll
            for (int j = 0; j < NC; ++j) fb[q][j] = frag(p + (BM + j * 16 + lrow) * 128, q);
#pragma unroll
            for (int m = 0; m < MT; ++m) fa[q][m] = frag(p + (m * 16 + lrow) * 128, q);
        }
#if IN_DT == DT_F8E4M3
        const float *sc = reinterpret_cast<const float *>(p + (BM + BN) * 128);
        float f[MT];
        const float sj = sc[64];
#pragma unroll
        for (int m = 0; m < MT; ++m) f[m] = sc[m * 16 + lrow];
#endif
        lds_done(); // the stage may be filled again
        if (i + STAGES < mine) load(i + STAGES, stage);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NC; ++j) {
#if IN_DT == DT_F8E4M3
                const f4_t d = mfma(fb[0][j], fa[0][m], f4_t{0, 0, 0, 0});
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[m][j][v] = __builtin_fmaf(d[v], f[m] * sj, acc[m][j][v]);
#else
#pragma unroll
                for (int q = 0; q < KQ; ++q) acc[m][j] = mfma(fb[q][j], fa[q][m], acc[m][j]);
#endif
            }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }

    // ---- the wavefronts' sums, in the order of their numbers
    barrier();
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NC; ++j) *reinterpret_cast<f4_t *>(lds + ((wave * MT + m) * NC + j) * 1024 + lane * 16) = acc[m][j];
    barrier();
    char *c = g.c + inst * g.c_inst;
#pragma unroll
    for (int i = 0; i < (MT * NC + NW - 1) / NW; ++i) {
        const int tile = i * NW + wave;
        if (tile >= MT * NC) break;
        f4_t sum = f4_t{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const f4_t x = *reinterpret_cast<const f4_t *>(lds + (w * MT * NC + tile) * 1024 + lane * 16);
#pragma unroll
            for (int v = 0; v < 4; ++v) sum[v] += x[v];
        }
        const int r = tile / NC * 16 + lrow, j = tile % NC * 16 + lgrp * 4;
        if (r < rows && j < cols) store4<false>(c + ((long)(row + r) * g.cols + col + j) * (long)sizeof(out_t), sum, cols - j);
    }
}
