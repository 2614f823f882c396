// Index arithmetic of the products over rows by expert that the host walks too: no vector types, no memory.

// Scales of 8-bit floats under tiles of 256 x 256.  They lie in LDS in two places that runs of up to SCALE_RUN steps take by turns, a new
// run at each tile.  A run is requested two steps ahead of its first, while one group of wavefronts has yet to read for the step at hand: its
// place is free only if the run between has more than one step.  Reductions that would leave one step for their last run count their steps
// from 1 instead of 0, so that the first run is shorter by one and the last has two (9 blocks: 7 and 2).
constexpr int SCALE_RUN = 8;
constexpr int first_step(int steps) { return steps % SCALE_RUN == 1; } // of more than one
constexpr bool starts_run(int step, int first) { return step == first || step % SCALE_RUN == 0; }
constexpr int head_of_run(int step) { return step / SCALE_RUN * SCALE_RUN; } // the step, there or not, at the head of its place
