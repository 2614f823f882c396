// Products over rows that lie sorted by expert (or of one matrix), and the gradient of the experts' matrices, on the matrix cores.
//
//   C[t][j]    = sum_k A[t][k] B[e(t)][k][j]        8-bit floats: sum over blocks of 128 k of SA[t][b] SB[e][j/128][b] (block's sum)
//                                                   8-bit integers: the sum, exact in 32 bits, times SA[t] SB[e][j]
//   D[e][i][j] = sum over the rows t of e of P[t][i] Q[t][j]                                                     (WGRAD)
//
// A workgroup makes one tile of rows of one expert (ragged_tile.h).  Two or three lie on a compute unit and overlap each other's loads, products
// and stores; launches that leave each one alone take the steps in two groups instead.  What bounds it is the way from the L2 into LDS,
// 31 to 46 bytes a clock and compute unit, on top of which come the reads of fragments that no products cover.  Measured: 1111 x 2056 x 1360
// in 8 bits by 128 x 128 12.5 us (153 workgroups, 0.50 PFLOP/s); f16, 4062 rows of 13 experts, 1032 x 2048, transposed 32.6 (0.53); gradient
// of 19 experts, 1489 rows, 1032 x 520 by 64 x 128 12.9, of which it writes 26 MB.
#include "common.h"
#include "ragged.h"
#include "ragged_tile.h"

typedef ragged_tile<TILE_M, TILE_N, TILE_WI, TILE_WJ, TILE_GROUPS> tile;
constexpr int TABLE_AT = tile::LDS_BYTES, LDS_BYTES = TABLE_AT + (GROUPED && !WGRAD ? 4096 : 0);
static_assert(LDS_BYTES == LDS_HOST, "the host's count of LDS");

extern "C" __global__ void __launch_bounds__(tile::THREADS) ms_kernel(const ragged_args g)
{
    __shared__ __attribute__((aligned(1024))) char lds[LDS_BYTES];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), inst = blockIdx.y;
    const int *offsets = GROUPED ? g.offsets + (long)inst * (g.experts + 1) : nullptr;
    int *table = reinterpret_cast<int *>(lds + TABLE_AT);
    tile_t t;
    if (GROUPED && !WGRAD) {
        tile_at where;
        unsigned of;
        range_t r;
        const unsigned nt = (unsigned)(g.cols + tile::BN - 1) / tile::BN;
        if (!find_row_tile(offsets, g.experts, g.rows, tile::BM, nt, blockIdx.x, lane, wave, table, where, of, r)) return;
        if (!tile_from<tile::BM, tile::BN>(g, where, of, nt, r, t)) return;
    } else {
        // products deal runs of tiles to the XCDs, so that the workgroups that run together on one XCD share rows and columns in its L2
        const unsigned total = tiles_of<tile::BM, tile::BN>(g, table);
        if (blockIdx.x >= total || !decode<tile::BM, tile::BN>(g, offsets, table, WGRAD ? blockIdx.x : run_of_xcd(blockIdx.x, total), lane, t)) return;
    }
    tile::make(g, inst, t, lds);
}
