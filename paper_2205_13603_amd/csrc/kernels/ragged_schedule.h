// Index arithmetic of the products over rows by expert that the host walks too: no vector types, no memory.

// Place of workgroup f of `total` in an order in which each XCD, the hardware dealing workgroups to the 8 in turn, has a run of neighbours.
constexpr unsigned run_of_xcd(unsigned f, unsigned total)
{
    const unsigned xcd = f % 8, left = total % 8;
    return xcd * (total / 8) + (xcd < left ? xcd : left) + f / 8;
}

// The `of`-th of `tiles` rows of tiles by `nt` columns of them: 8 rows by all columns at a time, rows first.
struct tile_in_bands {
    unsigned row, col;
};
constexpr tile_in_bands in_bands(unsigned of, unsigned tiles, unsigned nt)
{
    constexpr unsigned GM = 8;
    const unsigned band = of / (GM * nt), in = of - band * GM * nt, rest = tiles - band * GM, high = rest < GM ? rest : GM;
    return {band * GM + in % high, in / high};
}

// ---- tiles of 256 x 256 under persistent workgroups

// Whole tiles of an expert's rows: the last may be a part of one, but more than half; less is made in quarters of 128 x 128.
constexpr int whole_tiles(int rows) { return (rows + 127) / 256; }
constexpr bool half_left(int rows) { return rows > whole_tiles(rows) * 256; }

// Of a launch's tiles those that stay whole, and all quarters: those of `halves` tiles of up to half the rows (two each), and behind them four each of a last
// round that would leave most workgroups without a tile.
constexpr unsigned QUARTER = 40; // time of a quarter in hundredths of a whole tile's (8 bits, 4096 deep: 26.6 us of 68; bf16: 42 of 105)
struct rounds_t {
    unsigned whole, quarters;
};
constexpr rounds_t split_rounds(unsigned tiles, unsigned halves, unsigned grid)
{
    const unsigned rest = tiles % grid, more = (4 * rest + 2 * halves + grid - 1) / grid, as_it_is = (2 * halves + grid - 1) / grid;
    if (rest && more * QUARTER < 100 + as_it_is * QUARTER) return {tiles - rest, 4 * rest + 2 * halves};
    return {tiles, 2 * halves};
}
// Quarter q: of tile `tile` or, `half`, of the tile-th row of half tiles; rows and columns from its first.
struct quarter_t {
    bool half;
    unsigned tile, row, col;
};
constexpr quarter_t quarter_of(unsigned q, const rounds_t &r, unsigned halves, unsigned nt)
{
    const unsigned of_whole = r.quarters - 2 * halves;
    if (q < of_whole) return {false, r.whole + q / 4, q % 2 * 128, q % 4 / 2 * 128};
    return {true, (q - of_whole) / (nt * 2), 0, (q - of_whole) % (nt * 2) * 128};
}
// Turn f of a launch of `grid` workgroups, every other round backwards.
constexpr unsigned back_and_forth(unsigned f, unsigned grid)
{
    const unsigned round = f / grid;
    return round & 1 ? round * grid + (grid - 1 - (f - round * grid)) : f;
}

// Scales of 8-bit floats under tiles of 256 x 256.  They lie in LDS in two places that runs of up to SCALE_RUN steps take by turns, a new
// run at each tile.  A run is requested two steps ahead of its first, while one group of wavefronts has yet to read for the step at hand: its
// place is free only if the run between has more than one step.  Reductions that would leave one step for their last run count their steps
// from 1 instead of 0, so that the first run is shorter by one and the last has two (9 blocks: 7 and 2).
constexpr int SCALE_RUN = 8;
constexpr int first_step(int steps) { return steps % SCALE_RUN == 1; } // of more than one
constexpr bool starts_run(int step, int first) { return step == first || step % SCALE_RUN == 0; }
constexpr int head_of_run(int step) { return step / SCALE_RUN * SCALE_RUN; } // the step, there or not, at the head of its place
