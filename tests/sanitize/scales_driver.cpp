// The places that the scales of 8-bit floats take under tiles of 256 x 256, phase by phase on the CPU: what gemm_ragged_phases.hip requests
// and reads in R0, M0, R1 and M1 of each step, its second group of wavefronts one phase late, with loads that land as early and as late as
// the waits allow.  Exit status 0 = every read finds the scale of its own tile and block.
#include "../../paper_2205_13603_amd/csrc/kernels/ragged_schedule.h"

#include <cstdio>
#include <vector>

struct Scale {
    int tile, block;
};
struct Request {
    int issued, landed, place; // phases: from `issued` on its old values may be gone, behind `landed` the new ones are there
    Scale of[SCALE_RUN];
};
struct Read {
    int phase, place, slot;
    Scale want;
};

// Requests and reads of `tiles` tiles of `steps` steps; `late` phases behind the first group.
static void walk(int steps, int tiles, int late, std::vector<Request> *requests, std::vector<Read> *reads)
{
    const int first = first_step(steps), end = first + steps;
    // the cursor of the loads: as place(), next_step(), advance() and load_scales()
    int lt = 0, lk = first, lplace = 0;
    bool more = true;
    auto request = [&](int phase, int by) {
        if (!starts_run(lk, first)) return;
        Request r = {phase, by, lplace, {}};
        const int start = head_of_run(lk) - first;
        for (int i = 0; i < SCALE_RUN; ++i) r.of[i] = {lt, start + i >= 0 && start + i < steps ? start + i : -1};
        requests->push_back(r);
    };
    auto advance = [&] {
        if (more && lk + 1 < end) {
            ++lk;
            if (lk % SCALE_RUN == 0) lplace ^= 1;
        } else if (more) {
            more = lt + 1 < tiles;
            if (more) ++lt, lk = first, lplace ^= 1;
        }
    };
    request(-2 + late, -1 + late); // ahead of the first phase, waited for
    advance();
    request(-2 + late, -1 + late);
    int n = 0, place = 0;
    for (int t = 0; t < tiles; ++t) {
        for (int k = first; k < end; ++k, ++n) {
            const int phase = 4 * n + late;
            if (k && k % SCALE_RUN == 0) place ^= 1;
            reads->push_back({phase, place, k % SCALE_RUN, {t, k - first}});
            advance();
            reads->push_back({phase + 2, place, k % SCALE_RUN, {t, k - first}});
            request(phase + 2, phase + 4); // the eight loads that the end of the next R0 leaves in flight are all younger
        }
        place ^= 1;
    }
}

int main()
{
    for (int steps = 2; steps <= 200; ++steps) {
        std::vector<Request> one, other;
        std::vector<Read> reads, late;
        walk(steps, 5, 0, &one, &reads);
        walk(steps, 5, 1, &other, &late);
        // rows: each group requests its own; columns: the first group requests for both
        auto check = [&](const std::vector<Request> &requests, const std::vector<Read> &rs, const char *what) {
            for (const Read &r : rs) {
                const Request *last = nullptr; // the one that surely landed ahead of the read; none other may have begun
                for (const Request &q : requests)
                    if (q.place == r.place && q.issued <= r.phase) last = &q;
                if (!last || last->landed >= r.phase || last->of[r.slot].tile != r.want.tile || last->of[r.slot].block != r.want.block) {
                    fprintf(stderr, "%d steps, %s: tile %d step %d reads place %d in phase %d, which holds tile %d from phase %d to %d on\n", steps, what, r.want.tile,
                            r.want.block, r.place, r.phase, last ? last->of[r.slot].tile : -1, last ? last->issued : 0, last ? last->landed : 0);
                    return false;
                }
            }
            return true;
        };
        if (!check(one, reads, "first group") || !check(other, late, "second group") || !check(one, late, "second group's columns")) return 1;
    }
    puts("scales ok");
    return 0;
}
