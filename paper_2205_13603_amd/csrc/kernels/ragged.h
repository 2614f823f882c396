// Shared by the kernels of products over rows that lie sorted by expert.
#include "ragged_schedule.h"

// As RaggedArgs in ms_internal.h: distances in bytes.  depth, cols and rows of a gradient of weights are T, J and I.
struct ragged_args {
    const char *a, *b;
    const int *offsets;
    const float *sa, *sb;
    char *c;
    long a_row, b_row, b_expert;
    long a_inst, b_inst, sa_inst, sb_inst, c_inst;
    int rows, cols, depth, experts;
};

typedef unsigned u4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef int i8v_t __attribute__((ext_vector_type(8)));
typedef int i4_t __attribute__((ext_vector_type(4)));
#if IN_DT == DT_I8
typedef i4_t sum4_t; // 8-bit integers are summed exactly
#else
typedef f4_t sum4_t;
#endif

// One matrix-core step.  The operands are swapped, so that a lane holds four consecutive columns of one row: rows lane % 16, columns
// 4 * (lane / 16) and on.
#if IN_DT == DT_F8E4M3
struct frag_t { u4_t v[2]; }; // 32 k values: chunks lane / 16 and 4 + lane / 16 of a row's 128 bytes, for both operands alike (chunks 2 lane / 16
                              // and on would meet the banks of other rows: 42 % of the LDS cycles of 8192^3)
__device__ __forceinline__ f4_t mfma(const frag_t &b, const frag_t &a, f4_t c)
{
    // format selectors 0 = this 8-bit float for both operands; zero scale operands select the unscaled form
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i8v_t, b), __builtin_bit_cast(i8v_t, a), c, 0, 0, 0, 0, 0, 0);
}
#else
struct frag_t { u4_t v[1]; }; // 8 k values, of 8-bit integers 16
__device__ __forceinline__ sum4_t mfma(const frag_t &b, const frag_t &a, sum4_t c)
{
#if IN_DT == DT_I8
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4_t, b.v[0]), __builtin_bit_cast(i4_t, a.v[0]), c, 0, 0, 0);
#elif IN_DT == DT_F16
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, b.v[0]), __builtin_bit_cast(h8_t, a.v[0]), c, 0, 0, 0);
#else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, b.v[0]), __builtin_bit_cast(b8_t, a.v[0]), c, 0, 0, 0);
#endif
}
#endif
constexpr int ES = sizeof(in_t), KQ = 8 / (sizeof(frag_t) / 4); // matrix-core steps of a k step of 128 bytes
static_assert(KQ == (IN_DT == DT_F8E4M3 ? 1 : 2), "16 bytes of a row for each lane, or 32");

// The one rounding to the output type.
__device__ __forceinline__ out_t round_out(float x)
{
#if OUT_DT == DT_BF16
    return float_to_bf16(x);
#else
    return (out_t)x;
#endif
}

// Sums as results.  8-bit integers: times the scale of their row, then those of their columns (in this order no product of two small scales
// is formed); the sum is rounded to fp32 first, each product once: 3 * 2^-24 in all.
__device__ __forceinline__ f4_t results(const sum4_t &x, float of_row, const f4_t &of_cols)
{
#if IN_DT == DT_I8
    f4_t y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (float)x[i] * of_row * of_cols[i];
    return y;
#else
    return x;
#endif
}
// Scales of 8-bit integers: of row r of `rows` from `sa`, of four columns from `sb` (1 for what is not there).
__device__ __forceinline__ float row_scale(const float *sa, int r, int rows)
{
#if IN_DT == DT_I8
    return r < rows ? sa[r] : 1.f;
#else
    return 1.f;
#endif
}
__device__ __forceinline__ f4_t col_scales(const float *sb, int col, int cols)
{
    f4_t s = {1.f, 1.f, 1.f, 1.f};
#if IN_DT == DT_I8
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < cols) s[i] = sb[col + i];
#endif
    return s;
}

// A barrier of the workgroup that the compiler moves no memory access across; this wavefront's LDS accesses are through before it.
__device__ __forceinline__ void barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ int clamp_to(int x, int high) { return x < 0 ? 0 : x > high ? high : x; }

// The rows of expert e: offsets outside [0, total] count as the nearer end, and an end ahead of its start as no rows.
struct range_t { int first, last; };
__device__ __forceinline__ range_t rows_of(const int *offsets, int e, int total)
{
    const int first = clamp_to(offsets[e], total), last = clamp_to(offsets[e + 1], total);
    return {first, last < first ? first : last};
}

// Sums over the lanes up to and including each: within rows of 16, over the rows of a half, over the halves.
__device__ __forceinline__ int sums_of_lanes(int n)
{
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xf, 0xf, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xa, 0xf, false);
    return n + __builtin_amdgcn_update_dpp(0, n, 0x143, 0xc, 0xf, false);
}

// Tiles of `bm` rows of the experts up to and including e, for all of them, into `table` (LDS): by the first wavefront, before a barrier.
// Offsets that decrease make ranges overlap: the callers check what they find.
__device__ __forceinline__ void count_tiles(const int *offsets, int experts, int total, int bm, int lane, int *table)
{
    int before = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        int n = 0;
        if (e < experts) {
            const range_t r = rows_of(offsets, e, total);
            n = (r.last - r.first + bm - 1) / bm;
        }
        n = sums_of_lanes(n) + before;
        if (e < experts) table[e] = n;
        before = __builtin_amdgcn_readlane(n, 63);
    }
}

// The same of tiles of 256 rows, with the rest of an expert's rows a tile only where it is more than half of one; `halves`: experts up
// to and including e whose rest is less.
__device__ __forceinline__ void count_wide_tiles(const int *offsets, int experts, int total, int lane, int *table, unsigned short *halves)
{
    int before = 0, before_h = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        int n = 0, h = 0;
        if (e < experts) {
            const range_t r = rows_of(offsets, e, total);
            n = whole_tiles(r.last - r.first);
            h = half_left(r.last - r.first);
        }
        const unsigned long m = __ballot(h); // halves of the lanes up to this one
        h = before_h + __builtin_popcountl(m & (~0ul >> (63 - lane)));
        n = sums_of_lanes(n) + before;
        if (e < experts) {
            table[e] = n;
            halves[e] = (unsigned short)h;
        }
        before = __builtin_amdgcn_readlane(n, 63);
        before_h += __builtin_popcountl(m);
    }
}

// Expert of row tile `t`, and which of the expert's tiles it is; all lanes of a wavefront together.
struct tile_at { int expert, tile, tiles; };
template <class T> __device__ __forceinline__ tile_at find_tile(const T *table, int experts, int t, int lane)
{
    int e0 = 0;
    for (;; e0 += 64) {
        const int e = e0 + lane;
        const bool behind = e < experts ? (int)table[e] > t : true;
        const unsigned long m = __ballot(behind);
        if (m) {
            int e1 = e0 + __builtin_ctzl(m);
            e1 = e1 < experts ? e1 : experts - 1;
            const int from = e1 ? table[e1 - 1] : 0, to = table[e1];
            return {__builtin_amdgcn_readfirstlane(e1), __builtin_amdgcn_readfirstlane(t - from), __builtin_amdgcn_readfirstlane(to - from)};
        }
    }
}

// For workgroups that make one tile: the expert and row tile of workgroup `block` in launches of `nt` tiles of columns, its place among the
// expert's tiles (`of`) and the expert's rows; false: past the last tile.  Up to 64 experts fit in the lanes of each wavefront: one load of
// the offsets and no barrier (8 bits, 43 experts, 647 x 1576 x 768 by 16 x 16: 22.4 us through a table in LDS, 18.1 this way).
__device__ __forceinline__ bool find_row_tile(const int *offsets, int experts, int total, int bm, unsigned nt, unsigned block, int lane, int wave, int *table, tile_at &where, unsigned &of, range_t &rows)
{
    if (experts <= 64) {
        range_t r = {0, 0};
        if (lane < experts) r = rows_of(offsets, lane, total);
        const int n = sums_of_lanes((r.last - r.first + bm - 1) / bm), all = __builtin_amdgcn_readlane(n, 63);
        if (block >= (unsigned)all * nt) return false;
        const unsigned f = run_of_xcd(block, (unsigned)all * nt);
        const int t = uniform(f / nt), e = __builtin_ctzl(__ballot(n > t));
        const int from = e ? __builtin_amdgcn_readlane(n, e - 1) : 0, to = __builtin_amdgcn_readlane(n, e);
        where = {e, t - from, to - from};
        of = f - (unsigned)from * nt;
        rows = {__builtin_amdgcn_readlane(r.first, e), __builtin_amdgcn_readlane(r.last, e)};
        return true;
    }
    if (wave == 0) count_tiles(offsets, experts, total, bm, lane, table);
    barrier();
    const unsigned all = uniform((unsigned)table[experts - 1]) * nt;
    if (block >= all) return false;
    const unsigned f = run_of_xcd(block, all);
    where = find_tile(table, experts, (int)(f / nt), lane);
    if ((unsigned)where.tile >= (unsigned)where.tiles) return false; // offsets that decrease: nothing outside the tensors is touched
    of = f - (unsigned)(f / nt - where.tile) * nt;
    rows = rows_of(offsets, where.expert, total);
    rows = {__builtin_amdgcn_readfirstlane(rows.first), __builtin_amdgcn_readfirstlane(rows.last)};
    return true;
}

#ifdef WGRAD // tiles of rows and columns
struct tile_t {
    int expert, row, rows, col; // first row (of A and C; WGRAD: of D[e]) and how many rows the tile has, first column
    int k0, depth;              // first row and number of rows of the reduction
};

// The launch's tiles; `table` as count_tiles filled it.
template <int TR, int TC> __device__ __forceinline__ unsigned tiles_of(const ragged_args &g, const int *table)
{
    const unsigned nt = (unsigned)(g.cols + TC - 1) / TC;
    if (GROUPED && !WGRAD) return uniform((unsigned)table[g.experts - 1]) * nt;
    return (unsigned)((g.rows + TR - 1) / TR) * nt * (WGRAD ? (unsigned)g.experts : 1u);
}

// The `of`-th tile of an expert (or of the one matrix) with row tiles `where` and rows `r`.  false: it has no rows.
template <int TR, int TC> __device__ __forceinline__ bool tile_from(const ragged_args &g, const tile_at &where, unsigned of, unsigned nt, const range_t &r, tile_t &t)
{
    const tile_in_bands at = in_bands(of, (unsigned)where.tiles, nt);
    t.expert = where.expert;
    t.col = (int)at.col * TC;
    t.row = (int)at.row * TR;
    t.k0 = 0;
    t.depth = g.depth;
    int end = g.rows;
    if (GROUPED) {
        const int first = __builtin_amdgcn_readfirstlane(r.first), last = __builtin_amdgcn_readfirstlane(r.last);
        if (WGRAD) {
            t.k0 = first;
            t.depth = last - first;
        } else {
            t.row += first;
            end = last;
        }
    }
    t.rows = end - t.row < TR ? end - t.row : TR;
    // divisions are made on the vector unit; the tile is the same in all lanes, and its fields belong in scalar registers
    t = {__builtin_amdgcn_readfirstlane(t.expert), __builtin_amdgcn_readfirstlane(t.row), __builtin_amdgcn_readfirstlane(t.rows), __builtin_amdgcn_readfirstlane(t.col), t.k0, t.depth};
    return t.rows > 0;
}

// Tile `f`; false: there is nothing to do (offsets that decrease: nothing outside the tensors is touched).  WIDE: row tiles as count_wide_tiles counts them.  `order` (WGRAD): the experts in the order in which their
// tiles are made.
template <int TR, int TC, bool WIDE = false> __device__ __forceinline__ bool decode(const ragged_args &g, const int *offsets, const int *table, unsigned f, int lane, tile_t &t, const unsigned short *order = nullptr)
{
    const unsigned nt = (unsigned)(g.cols + TC - 1) / TC;
    tile_at where;
    unsigned of;
    if (WGRAD || !GROUPED) {
        const int mt = WIDE ? whole_tiles(g.rows) : (g.rows + TR - 1) / TR;
        const unsigned each = (unsigned)mt * nt;
        where = {(int)(f / each), 0, mt};
        of = f % each;
        if (WGRAD && each % 8 == 0) of = run_of_xcd(of, each); // an expert's tiles over all XCDs: experts differ in their rows
        if (order) where.expert = order[where.expert];
    } else {
        where = find_tile(table, g.experts, (int)(f / nt), lane);
        if ((unsigned)where.tile >= (unsigned)where.tiles) return false;
        of = f - (f / nt - (unsigned)where.tile) * nt;
    }
    range_t r = {0, 0};
    if (GROUPED) r = rows_of(offsets, where.expert, WGRAD ? g.depth : g.rows);
    return tile_from<TR, TC>(g, where, of, nt, r, t);
}
#endif

// 4 bytes per lane from a buffer to `dst` (wave-uniform) + 4 * lane; as gather_lds16 in common.h
__device__ __forceinline__ void gather_lds4(const rsrc_t &buffer, unsigned voff, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(uniform(dst)), "v"(voff), "s"(buffer) : "memory", "m0");
}
__device__ __forceinline__ void gather_lds16_at(const rsrc_t &buffer, unsigned voff, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(uniform(dst)), "v"(voff), "s"(buffer) : "memory", "m0");
}
// this wavefront's LDS accesses are through, and none behind is moved ahead
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Results at `dst` that no L2 keeps: lines that stay there are written back when the kernel ends, which it waits for (f16, gradient of 24 experts
// 1032 x 520: 16.2 us, so 12.9; 1111 x 2056 x 1360 in 8 bits 13.5 and 12.5; 8192 x 4096 x 4096 in bf16 245 and 236).
template <class T> __device__ __forceinline__ void stream_out(char *dst, const T &x)
{
    typedef unsigned words_t __attribute__((ext_vector_type(sizeof(T) / 4), aligned(sizeof(out_t))));
    __builtin_nontemporal_store(__builtin_bit_cast(words_t, x), reinterpret_cast<words_t *>(dst));
}

// Four column tiles of fp32 results, of which lane 16 g + r has columns 4 g to 4 g + 3 of row r, put together between lanes: x[s] is then of row 4 s + r % 4,
// column tile r / 4, so that four rows leave at a time, each as 256 bytes.  (8-bit integers into fp32, 8192 x 8192 x 512 by 256 x 256: 132 us as 64 bytes of 16
// rows, 84 this way; 8192 x 8191 x 512 by 64 x 128 233 and 95; gradient of 8 experts, 4096 x 2048, bf16 154 and 147.)
__device__ __forceinline__ void rows_together(f4_t (&x)[4])
{
    auto both = [](float &a, float &b, auto swap) {
        const int p = __builtin_bit_cast(int, a), q = __builtin_bit_cast(int, b);
        a = __builtin_bit_cast(float, swap(p, q, true));
        b = __builtin_bit_cast(float, swap(q, p, false));
    };
#pragma unroll
    for (int v = 0; v < 4; ++v) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float a = x[j][v], b = x[j + 2][v];
            both(a, b, [](int own, int other, bool first) { // lanes 8 to 15 of a row, and 0 to 7
                return first ? __builtin_amdgcn_update_dpp(own, other, 0x128, 0xf, 0xc, false) : __builtin_amdgcn_update_dpp(own, other, 0x128, 0xf, 0x3, false);
            });
            x[j][v] = a, x[j + 2][v] = b;
        }
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            float a = x[j][v], b = x[j + 1][v];
            both(a, b, [](int own, int other, bool first) { // every other four lanes, and the ones before them
                return first ? __builtin_amdgcn_update_dpp(own, other, 0x114, 0xf, 0xa, false) : __builtin_amdgcn_update_dpp(own, other, 0x104, 0xf, 0x5, false);
            });
            x[j][v] = a, x[j + 1][v] = b;
        }
    }
}

// up to four results of a row at `dst`, the first `n` of them; STREAM: as above (parts of lines are slower that way)
template <bool STREAM> __device__ __forceinline__ void store4(char *dst, f4_t x, int n)
{
    struct __attribute__((packed, aligned(sizeof(out_t)))) quad { out_t v[4]; };
    quad q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = round_out(x[i]);
    if (n >= 4) {
        if (STREAM) stream_out(dst, q);
        else *reinterpret_cast<quad *>(dst) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) reinterpret_cast<out_t *>(dst)[i] = q.v[i];
    }
}
