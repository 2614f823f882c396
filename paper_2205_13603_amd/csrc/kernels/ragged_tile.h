// One tile of a product over rows by expert, or of the gradient of the experts' matrices, by all wavefronts of a workgroup: TR rows by TC columns,
// WR by WC wavefronts of a group, two stages of LDS.
//
// k steps of 128 bytes of each row of the operands go straight into a ring of LDS stages; operands contiguous along k (A_KC, B_KC)
// lie there as rows of eight 16-byte chunks, swizzled by the row so that a fragment read meets each bank once; the others as rows of
// k, in 32-byte granules swizzled by k, read with the transposing LDS loads.  What lies behind an expert's rows, the last column or the last
// k is read as zeros and not stored.
//
// Where a tile has its compute unit to itself GROUPS = 2: two groups of wavefronts take the k steps in turn, each with a ring of its own and
// half a step behind the other, so that one reads fragments while the other multiplies; in the end each adds up half of the sums.
// (128 x 128 alone on its compute unit, a step: 8 bits 0.75 us with one group, 0.60 with two, 0.40 without products or without loads; 16 bits
// 0.70, 0.54, 0.40 and 0.35.)
template <int TR, int TC, int WR, int WC, int GROUPS = 1> struct ragged_tile {
    static constexpr int BM = TR, BN = TC, WI = WR, WJ = WC, STAGES = 2, NW = WI * WJ, TM = BM / WI / 16, TN = BN / WJ / 16, BK = 128 / ES;
    static constexpr int THREADS = NW * GROUPS * 64;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LOADS = LA + LB; // load instructions of a wavefront and step
    static constexpr bool SCALED = IN_DT == DT_F8E4M3;
    static constexpr int KB = 8;                                              // k blocks whose scales are in LDS at a time, twice
    static constexpr int SC_BYTES = SCALED ? KB * BM * 4 : 0, SB_BYTES = SCALED ? 256 : 0;
    static constexpr int SC_AT = GROUPS * STAGES * STAGE, SB_AT = SC_AT + 2 * SC_BYTES, LDS_BYTES = SB_AT + 2 * SB_BYTES;
    static constexpr int LS = SCALED ? KB * BM / 64 / (NW * GROUPS) : 0;                 // load instructions of a wavefront for the scales of KB blocks
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "every wavefront issues the same loads");
    static_assert(GROUPS == 1 || TM % 2 == 0, "two groups: half the sums each");
    static_assert(BM >= 64 && 128 % (TN * 16) == 0, "a wavefront's columns share a scale");

    // `lds`: LDS_BYTES that no wavefront uses any more
    static __device__ __forceinline__ void make(const ragged_args &g, int inst, const tile_t &t, char *lds)
    {
        const int tid = threadIdx.x, lane = tid % 64, every = __builtin_amdgcn_readfirstlane(tid / 64), group = GROUPS > 1 ? every / NW : 0, wave = GROUPS > 1 ? every % NW : every;
        const int wi = wave / WJ, wj = wave % WJ, lrow = lane % 16, lgrp = lane / 16;
        const int cols = g.cols - t.col < BN ? g.cols - t.col : BN;
        const int steps = (t.depth + BK - 1) / BK;

        // ---- operands: of each load instruction the lane's place from the tile's first element, OUTSIDE where there is nothing
        const char *a = g.a + inst * g.a_inst + (A_KC ? (long)t.row * g.a_row : (long)t.k0 * g.a_row + (long)t.row * ES);
        const char *b = g.b + inst * g.b_inst + t.expert * g.b_expert + (B_KC ? (long)t.col * g.b_row : (long)t.k0 * g.b_row + (long)t.col * ES);
        // chunk of 16 bytes of a k-contiguous row, the same in all of a wavefront's instructions
        const int chunk = lane % 8 ^ lane / 8;
        // k row and first column of a transposed operand
        auto tr_k = [&](int width, int l) { return (wave + l * NW) * (512 / width) + lane * 8 / width; };
        auto tr_col = [&](int width, int l) {
            const int k = tr_k(width, l), slot = lane * 8 % width / 8, swz = (k & 3 | k >> 1 & 4) & (width / 16 - 1);
            return ((slot >> 1 ^ swz) << 4) + (slot & 1) * 8;
        };
        unsigned avoff[LA], bvoff[LB];
#pragma unroll
        for (int l = 0; l < LA; ++l) {
            if (A_KC) {
                const int r = (wave + l * NW) * 8 + lane / 8;
                avoff[l] = r < t.rows ? (unsigned)(r * (int)g.a_row + chunk * 16) : OUTSIDE;
            } else {
                const int c = tr_col(BM, l);
                avoff[l] = c < t.rows ? (unsigned)(tr_k(BM, l) * (int)g.a_row + c * ES) : OUTSIDE;
            }
        }
#pragma unroll
        for (int l = 0; l < LB; ++l) {
            if (B_KC) {
                const int r = (wave + l * NW) * 8 + lane / 8;
                bvoff[l] = r < cols ? (unsigned)(r * (int)g.b_row + chunk * 16) : OUTSIDE;
            } else {
                const int c = tr_col(BN, l);
                bvoff[l] = c < cols ? (unsigned)(tr_k(BN, l) * (int)g.b_row + c * ES) : OUTSIDE;
            }
        }
        const unsigned lds0 = lds_address(lds);
#if ALIGNED
        auto load = [&](int step, int stage) {
            const bool tail = step * BK + BK > t.depth; // elements of k that there are not
            const int here = t.depth - step * BK;
            const rsrc_t ra = buffer_at(a + (A_KC ? (long)step * 128 : (long)step * BK * g.a_row)), rb = buffer_at(b + (B_KC ? (long)step * 128 : (long)step * BK * g.b_row));
            const unsigned at = lds0 + (group * STAGES + stage) * STAGE + wave * 1024;
#pragma unroll
            for (int l = 0; l < LA; ++l) {
                unsigned v = avoff[l];
                if (tail) v = (A_KC ? chunk * (16 / ES) : tr_k(BM, l)) < here ? v : OUTSIDE;
                gather_lds16_at(ra, v, at + l * NW * 1024);
            }
#pragma unroll
            for (int l = 0; l < LB; ++l) {
                unsigned v = bvoff[l];
                if (tail) v = (B_KC ? chunk * (16 / ES) : tr_k(BN, l)) < here ? v : OUTSIDE;
                gather_lds16_at(rb, v, at + A_BYTES + l * NW * 1024);
            }
        };
#else
        // Rows that start anywhere, extents that are no whole 16 bytes: element by element through registers, which takes 7 to 18 times as long
        // (8 bits, 1111 x 2056 by 1360 12.4 us, by 1361 92; 4096 x 4096 by 4096 67, by 4097 1200; bf16, 4096 rows of 8 experts, 2048 by 1024 20, by
        // 1025 273; read the other way 22, with 2049 columns 215; gradients of 1024 x 2048 27, of 1025 213).
        auto load = [&](int step, int stage) {
            auto one = [&](const char *p, bool kc, unsigned voff, int k, int c, int high, int at) {
                union { in_t e[16 / ES]; u4_t v; } x;
#pragma unroll
                for (int i = 0; i < 16 / ES; ++i) {
                    const bool there = voff != OUTSIDE && (kc ? k + i < t.depth : k < t.depth && c + i < high);
                    x.e[i] = in_t(0);
                    if (there) x.e[i] = reinterpret_cast<const in_t *>(p + voff)[i];
                }
                *reinterpret_cast<u4_t *>(lds + at + lane * 16) = x.v;
            };
            const char *pa = a + (A_KC ? (long)step * 128 : (long)step * BK * g.a_row), *pb = b + (B_KC ? (long)step * 128 : (long)step * BK * g.b_row);
#pragma unroll 1
            for (int l = 0; l < LA; ++l) {
                const int r = (wave + l * NW) * 8 + lane / 8, c = tr_col(BM, l);
                const unsigned v = A_KC ? (r < t.rows ? (unsigned)(r * (int)g.a_row + chunk * 16) : OUTSIDE) : (c < t.rows ? (unsigned)(tr_k(BM, l) * (int)g.a_row + c * ES) : OUTSIDE);
                one(pa, A_KC, v, step * BK + (A_KC ? chunk * (16 / ES) : tr_k(BM, l)), c, t.rows, stage * STAGE + (wave + l * NW) * 1024);
            }
#pragma unroll 1
            for (int l = 0; l < LB; ++l) {
                const int r = (wave + l * NW) * 8 + lane / 8, c = tr_col(BN, l);
                const unsigned v = B_KC ? (r < cols ? (unsigned)(r * (int)g.b_row + chunk * 16) : OUTSIDE) : (c < cols ? (unsigned)(tr_k(BN, l) * (int)g.b_row + c * ES) : OUTSIDE);
                one(pb, B_KC, v, step * BK + (B_KC ? chunk * (16 / ES) : tr_k(BN, l)), c, cols, stage * STAGE + A_BYTES + (wave + l * NW) * 1024);
            }
        };
#endif

        // ---- scales of KB blocks: [block][row], gathered from rows of blocks; those of the columns beside them
#if IN_DT == DT_F8E4M3
        const int blocks = (g.depth + 127) / 128, col_blocks = (g.cols + 127) / 128;
        const char *sa = (const char *)g.sa + inst * g.sa_inst + (long)t.row * blocks * 4;
        const char *sb = (const char *)g.sb + inst * g.sb_inst + ((long)t.expert * col_blocks + t.col / 128) * blocks * 4;
        auto load_scales = [&](int first) {
            const rsrc_t r = buffer_at(sa + first * 4);
            const unsigned at = lds0 + SC_AT + first / KB % 2 * SC_BYTES;
#pragma unroll
            for (int l = 0; l < LS; ++l) {
                const int i = every * LS + l, row = i / KB * 64 + lane, k = i % KB; // the blocks of one line follow each other
                gather_lds4(r, row < t.rows && first + k < blocks ? (unsigned)(row * blocks + k) * 4 : OUTSIDE, at + (k * BM + i / KB * 64) * 4);
            }
            if (every == 0) { // columns: lane = 8 * (block of columns) + block of k
                const int n = lane / KB;
                gather_lds4(buffer_at(sb + first * 4), n < (BN + 127) / 128 && t.col / 128 + n < col_blocks && first + lane % KB < blocks ? (unsigned)(n * blocks + lane % KB) * 4 : OUTSIDE,
                            lds0 + SB_AT + first / KB % 2 * SB_BYTES);
            }
        };
#endif

        sum4_t acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = sum4_t{0, 0, 0, 0};

        // ---- fragments
        // of 16 rows from `row0` of a k-contiguous operand at `p`, matrix-core step q
        auto frag_kc = [&](const char *p, int row0, int q) {
            frag_t f;
            const char *r = p + row0 * 128 + lrow * 128;
            if (KQ == 2) {
                f.v[0] = *reinterpret_cast<const u4_t *>(r + ((q * 4 + lgrp) ^ lrow % 8) * 16);
            } else {
#pragma unroll
                for (int h = 0; h < (int)(sizeof(frag_t) / 16); ++h) f.v[h] = *reinterpret_cast<const u4_t *>(r + ((h * 4 + lgrp) ^ lrow % 8) * 16);
            }
            return f;
        };
        // of 16 columns from `col0` of a transposed operand of `width` columns
        auto frag_tr = [&](const char *p, int width, int col0, int q) {
            frag_t f;
#if IN_DT != DT_F8E4M3
            typedef short tr4_t __attribute__((ext_vector_type(4)));
            struct { tr4_t v[2]; } x;
            const int r = lrow / 4, swz = (r | (lgrp & 1) << 2) & (width / 16 - 1);
            const char *at = p + (q * 32 + lgrp * 8 + r) * width * 2 + ((col0 / 16) ^ swz) * 32 + lrow % 4 * 8;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                x.v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) tr4_t *)(at + h * 4 * width * 2));
            f.v[0] = __builtin_bit_cast(u4_t, x);
#endif
            return f;
        };
        auto frag_a = [&](int stage, int tm, int q) {
            const char *p = lds + (group * STAGES + stage) * STAGE;
            return A_KC ? frag_kc(p, (wi * TM + tm) * 16, q) : frag_tr(p, BM, (wi * TM + tm) * 16, q);
        };
        auto frag_b = [&](int stage, int tn, int q) {
            const char *p = lds + (group * STAGES + stage) * STAGE + A_BYTES;
            return B_KC ? frag_kc(p, (wj * TN + tn) * 16, q) : frag_tr(p, BN, (wj * TN + tn) * 16, q);
        };

        // ---- the ring
        frag_t fa[KQ][TM], fb[KQ][TN];
        float fs[TM]; // scales of step s
        auto read = [&](int s, int stage) {
#pragma unroll
            for (int q = 0; q < KQ; ++q) {
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[q][j] = frag_b(stage, j, q);
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[q][i] = frag_a(stage, i, q);
            }
#if IN_DT == DT_F8E4M3
            const float *sc = reinterpret_cast<const float *>(lds + SC_AT + s / KB % 2 * SC_BYTES) + s % KB * BM + wi * TM * 16 + lrow;
            const float sj = reinterpret_cast<const float *>(lds + SB_AT + s / KB % 2 * SB_BYTES)[(t.col % 128 + wj * TN * 16) / 128 * KB + s % KB];
#pragma unroll
            for (int i = 0; i < TM; ++i) fs[i] = sc[i * 16] * sj;
#endif
        };
        auto multiply = [&]() {
#if IN_DT == DT_F8E4M3
            constexpr int N = TM * TN, LAG = N > 3 ? 3 : N - 1; // results wait for the matrix core while it works on LAG further products
            f4_t d[LAG + 1];
#pragma unroll
            for (int m = 0; m < N + LAG; ++m) {
                if (m < N) {
                    d[m % (LAG + 1)] = mfma(fb[0][m % TN], fa[0][m / TN], f4_t{0, 0, 0, 0});
                    __builtin_amdgcn_sched_barrier(0); // the product first
                }
                if (m >= LAG) {
                    const int o = m - LAG;
                    f4_t &sum = acc[o / TN][o % TN];
                    sum = __builtin_elementwise_fma(d[o % (LAG + 1)], f4_t{fs[o / TN], fs[o / TN], fs[o / TN], fs[o / TN]}, sum);
                    asm volatile("" : "+v"(sum));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#else
#pragma unroll
            for (int q = 0; q < KQ; ++q)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma(fb[q][j], fa[q][i], acc[i][j]);
#endif
        };
        constexpr int OS = sizeof(out_t), HALF = TM / GROUPS; // row tiles that this wavefront stores
        const int row0 = (wi * TM + group * HALF) * 16;
        // scales of the results' rows and columns (8-bit integers), on their way from here: behind the products they would be waited for
        const float *const of_rows = (const float *)((const char *)g.sa + inst * g.sa_inst) + t.row;
        const float *const of_cols = (const float *)((const char *)g.sb + inst * g.sb_inst) + (long)t.expert * g.cols + t.col;
        f4_t sj[TN];
        float si[HALF];
#pragma unroll
        for (int j = 0; j < TN; ++j) sj[j] = col_scales(of_cols, (wj * TN + j) * 16 + lgrp * 4, cols);
#pragma unroll
        for (int i = 0; i < HALF; ++i) si[i] = row_scale(of_rows, row0 + i * 16 + lrow, t.rows);
#if IN_DT == DT_F8E4M3
        if (steps) load_scales(0);
#endif
        if constexpr (GROUPS == 1) {
            if (steps) load(0, 0);
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                DL_WAIT_VM(0); // this step's loads have landed; the barrier: everyone's, and the other stage has been read
                barrier();
#if IN_DT == DT_F8E4M3
                if (s % KB == 0) load_scales(s + KB); // beyond the last block: zeros
#endif
                if (s + 1 < steps) load(s + 1, (s + 1) % 2);
                read(s, s % 2);
                multiply();
            }
        } else {
            // Group 0 reads step 2 i in phase 2 i and multiplies in the next, group 1 step 2 i + 1 a phase later.  A step's stage is filled again
            // while its products are made: all wavefronts of the group have read it.
            const int turns = (steps + 1) / 2, mine = (steps - group + 1) / 2;
#if ALIGNED
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i < mine) load(group + 2 * i, i);
            if (mine > 1) DL_WAIT_VM(LOADS);
            else DL_WAIT_VM(0);
            barrier();
            if (group) barrier();
#pragma unroll 1
            for (int i = 0; i < turns; ++i) {
                const int s = group + 2 * i;
                if (i < mine) read(s, i % 2);
                barrier();
                if (i < mine) {
#if IN_DT == DT_F8E4M3
                    if (i % (KB / 2) == 0) load_scales(2 * i + KB); // over those of the steps before, which both groups have read
#endif
                    const bool further = i + 2 < mine;
                    if (further) load(s + 4, i % 2);
                    multiply();
                    if (further) DL_WAIT_VM(LOADS);
                    else DL_WAIT_VM(0);
                }
                barrier();
            }
            if (!group) barrier();
            // each group's half of the sums: its own and the other's
            auto of = [&](sum4_t one, sum4_t zero) { // values, not places: chosen by address the sums would lie in memory
                sum4_t x;
#pragma unroll
                for (int v = 0; v < 4; ++v) x[v] = group ? one[v] : zero[v];
                return x;
            };
            char *const other = lds + (1 - group) * (NW * TM / 2 * TN * 1024) + wave * (TM / 2 * TN * 1024) + lane * 16;
            const char *const here = lds + group * (NW * TM / 2 * TN * 1024) + wave * (TM / 2 * TN * 1024) + lane * 16;
            static_assert(NW * TM * TN * 1024 + NW * GROUPS * TN * 512 <= GROUPS * STAGES * STAGE, "sums and results fit where the operands were");
#pragma unroll
            for (int i = 0; i < TM / 2; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) *reinterpret_cast<sum4_t *>(other + (i * TN + j) * 1024) = of(acc[i][j], acc[TM / 2 + i][j]);
            barrier();
#pragma unroll
            for (int i = 0; i < TM / 2; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const sum4_t x = *reinterpret_cast<const sum4_t *>(here + (i * TN + j) * 1024), y = of(acc[TM / 2 + i][j], acc[i][j]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][j][v] = y[v] + x[v];
                }
#endif
        }

        // ---- results
        char *c = g.c + inst * g.c_inst + (WGRAD ? (long)t.expert * g.rows * g.cols * OS : 0);
        if constexpr (OS == 4) {
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                static_assert(TN == 4, "64 columns of a wavefront");
                f4_t x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = results(acc[i][j], si[i], sj[j]);
                rows_together(x);
                const int col = wj * 64 + lrow / 4 * 16 + lgrp * 4;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int r = row0 + i * 16 + s * 4 + lrow % 4;
                    if (r < t.rows && col < cols) store4<true>(c + ((long)(t.row + r) * g.cols + t.col + col) * OS, x[s], cols - col);
                }
            }
        } else {
            // 16 rows at a time by way of LDS, so that a row's columns leave as whole lines
            constexpr int CH = TN * 2; // 16-byte chunks of a wavefront's row
            if (GROUPS == 1) barrier(); // the last step's operands have been read
            char *const mine = lds + (GROUPS > 1 ? NW * TM * TN * 1024 : 0) + every * (16 * CH * 16); // two groups: behind the sums
            static_assert(16 * CH % 64 == 0, "whole rows to a store");
            static_assert(NW * 16 * CH * 16 <= STAGES * STAGE, "results fit where the operands were");
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    struct { out_t v[4]; } o;
                    const f4_t x = results(acc[i][j], si[i], sj[j]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o.v[v] = round_out(x[v]);
                    *reinterpret_cast<decltype(o) *>(mine + (lrow * CH + ((j * 2 + lgrp / 2) ^ (lrow % CH))) * 16 + lgrp % 2 * 8) = o;
                }
                lds_done();
#pragma unroll
                for (int l = 0; l < 16 * CH / 64; ++l) {
                    const int r = (l * 64 + lane) / CH, ch = lane % CH;
                    struct __attribute__((aligned(16))) { out_t v[8]; } o = *reinterpret_cast<const decltype(o) *>(mine + (r * CH + (ch ^ r % CH)) * 16);
                    const int row = row0 + i * 16 + r, col = wj * TN * 16 + ch * 8;
                    if (row < t.rows && col < cols) {
                        char *dst = c + ((long)(t.row + row) * g.cols + t.col + col) * OS;
                        if (col + 8 <= cols) {
                            stream_out(dst, o);
                        } else {
#pragma unroll
                            for (int v = 0; v < 8; ++v)
                                if (col + v < cols) reinterpret_cast<out_t *>(dst)[v] = o.v[v];
                        }
                    }
                }
                lds_done();
            }
        }
    }
};
