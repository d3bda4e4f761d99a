// How the tiles of a symmetric product are dealt out to workgroups.  Plain C++: of the host code, which plans, and of the kernels, which walk the plan.
//
// Workgroups take whole tiles as long as there is one for each of them.  The steps of the tiles that are left are dealt out: each of those tiles is cut into `slices` of
// `slice_steps` steps, a workgroup to each, and what that leaves of them (`rest` steps) goes to other workgroups, the helpers, so that all have about the same to do: helper h takes
// the rest of tile h, and of the further tiles' rests, behind each other, `share` steps.  Slices of one number run over the same steps at the same time: what their tiles share
// of the operands meets in the L2 caches.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace axo {

struct SymCut {
    int steps;   // of a tile
    int whole;   // tiles that are taken whole: a multiple of the workgroups, or all
    int cut;     // tiles that are cut, behind them
    int slices, slice_steps;
    int rest, helpers, share;

    // Helpers first..last have the rest of a further tile (helpers <= t < cut).
    constexpr int first_of(int t) const { return (int)((int64_t)(t - helpers) * rest / share); }
    constexpr int last_of(int t) const { return (int)(((int64_t)(t - helpers + 1) * rest - 1) / share); }
    // Parts of tile t, counted among those that are cut.
    constexpr int parts_of(int t) const { return rest == 0 ? slices : t < helpers ? slices + 1 : slices + last_of(t) - first_of(t) + 1; }
    // Where a part leaves its sums: the slices, the helpers' first parts, and their others, of which further tile u and helper h share number u + h.
    constexpr int slot_of(int t, int part) const {
        if (part < slices) return part * cut + t;
        const int base = slices * cut;
        return t < helpers ? base + t : base + helpers + (t - helpers) + first_of(t) + part - slices;
    }
    constexpr int slots() const { return cut == 0 ? 0 : cut * slices + (rest > 0 ? helpers + cut : 0); }
};

// A part of the work: steps from .. from + count of a tile.
struct SymPart {
    int tile, from, count;
    int cut;   // its number among the tiles that are cut, or -1: the tile is done by this part alone
    int slot, parts;
};

// The parts of one workgroup, in order.
struct SymWalk {
    int id, workgroups, whole, turn, at, end;
    constexpr SymWalk(const SymCut& c, int id_, int workgroups_) : id(id_), workgroups(workgroups_), whole(id_), turn(0), at(0), end(0) {
        const int h = id - c.cut * c.slices, all = c.cut > c.helpers ? (c.cut - c.helpers) * c.rest : 0;
        if (c.rest > 0 && h >= 0 && h < c.helpers) {
            at = h * c.share < all ? h * c.share : all;
            end = at + c.share < all ? at + c.share : all;
        }
    }
    constexpr bool next(const SymCut& c, SymPart& p) {
        p.cut = -1;
        p.from = 0;
        p.count = c.steps;
        if (whole < c.whole) {
            p.tile = whole;
            whole += workgroups;
            return true;
        }
        if (c.cut == 0) return false;
        const int h = id - c.cut * c.slices;
        int part = c.slices;
        if (h < 0) {
            if (turn++ > 0) return false;
            p.cut = id % c.cut;
            part = id / c.cut;
            p.from = part * c.slice_steps;
            p.count = c.slice_steps;
        } else {
            if (c.rest == 0 || h >= c.helpers) return false;
            if (turn++ == 0 && h < c.cut) {
                p.cut = h;
                p.from = c.slices * c.slice_steps;
                p.count = c.rest;
            } else {
                if (at >= end) return false;
                const int u = at / c.rest, in = at - u * c.rest;
                p.cut = c.helpers + u;
                p.from = c.slices * c.slice_steps + in;
                p.count = c.rest - in < end - at ? c.rest - in : end - at;
                at += p.count;
                part += h - c.first_of(p.cut);
            }
        }
        p.tile = c.whole + p.cut;
        p.parts = c.parts_of(p.cut);
        p.slot = c.slot_of(p.cut, part);
        if (p.parts == 1) p.cut = -1;
        return true;
    }
};

// A kind of tile: its rows; workgroups that run beside each other on a compute unit; us per step on a chip that is nearly idle, and what a full one adds; of a launch as a whole;
// to leave sums, and to add one part's.  Of launches of 3 to 528 tiles with 8 to 256 steps, whole and cut in up to sixteen parts, most are within 15 % of these:
//   64 x 64    128 columns, 8 steps 4.4 us; 576, 16 5.9; 1024, 64 14.4; in three slices 13.0
//   128 x 128  2048 columns, 32 steps 16.0; 96 40; in shares of 51 steps of up to ten parts 44; 4096, 64 steps, two rounds and sixteen tiles 90, those in nine slices 82; 256 steps 325 and 263
//   256 x 256  4096, 64 steps 86; 256 295; 8192, 128 steps 530, in slices of 16 to 26 steps 451 (of 128 x 128 ones 658)
struct SymKind {
    int size, beside;
    double step, busy, fixed, leave, add;
};
constexpr SymKind SYM_KINDS[4] = {{64, 1, 0.18, 0.0, 2.9, 1.0, 0.8}, {64, 2, 0.18, 0.13, 3.0, 1.0, 0.8}, {128, 1, 0.32, 0.20, 4.1, 0.5, 1.2}, {256, 1, 1.1, 0.5, 6.0, 2.0, 5.0}};
constexpr int SYM_MOST_PARTS = 16;  // of a tile
constexpr int SYM_MOST_CUT = 512;   // tiles that are cut: fewer than workgroups beside each other on 256 compute units
// Tiles of 256 rows and 128 columns, and the 128 x 128 ones that they leave of the diagonal, both in one launch: `size` of such a plan is SYM_HALF.
// (The same at half the size, 128 x 64 tiles of which 2048 columns have 256, is slower than 136 whole ones: 96 steps 45 us and 42, 32 steps 21 and 16.  The tiles take in 1.4 times as
// much, and 10 TB/s of operands already come from the caches.)
constexpr int SYM_HALF = 257, SYM_DIAGONAL = 129;

struct SymPlan {
    int size = 0, workgroups = 0;
    double us = 1e30;
    SymCut cut{}, diagonal{};
    int counters() const { return cut.cut + diagonal.cut; }
    // of the sums that parts of tiles leave
    int64_t partial_floats() const {
        return size == SYM_HALF ? (int64_t)diagonal.slots() * (128 * 128) : (int64_t)cut.slots() * size * size;
    }
};
// The quickest of all kinds for s rows and columns, the tiles that do not fill a round taken whole, in slices, or in slices and rests.
inline SymPlan sym_plan(int64_t s, int64_t steps, int64_t compute_units) {
    SymPlan best;
    {   // 32 x 32 tiles whose four waves split the reduction, five workgroups to a compute unit: bound by what a compute unit takes in, or by one wave's chain of steps
        // (256 columns, 16 steps; 512, 8; 576, 16; 1024, 16: see SLIM_MODEL, which these times are those of)
        const int64_t n = (s + 31) / 32, tiles = n * (n + 1) / 2, rounds = (tiles + compute_units - 1) / compute_units;
        const double chain = 0.7 + 0.24 * (double)((steps + 3) / 4);
        const double us = 2.5 + std::max((double)rounds * (0.2 + 0.08 * (double)steps), (double)((rounds + 4) / 5) * chain);
        if (tiles <= 5 * compute_units) best = {32, (int)tiles, us, {(int)steps, (int)tiles, 0, 1, 0, 0, 0, 1}, {}};
        for (int64_t q = 2; q <= SYM_MOST_PARTS && q * tiles <= compute_units && 4 * q <= steps; ++q) {
            const int64_t each = (steps + q - 1) / q, slices = steps / each, rest = steps - slices * each, parts = slices + (rest > 0);
            const double sliced = 2.5 + std::max(0.2 + 0.08 * (double)each, 0.7 + 0.24 * (double)((each + 3) / 4)) + 1.5 + 0.1 * (double)parts;
            if (sliced < best.us)
                best = {32, (int)(tiles * parts), sliced, {(int)steps, 0, (int)tiles, (int)slices, (int)each, (int)rest, rest > 0 ? (int)tiles : 0, 1}, {}};
        }
    }
    for (const SymKind& k : SYM_KINDS) {
        const int64_t n = (s + k.size - 1) / k.size, tiles = n * (n + 1) / 2, most = compute_units * k.beside, rounds = tiles / most, left = tiles % most;
        // so many steps one behind the other, on so many workgroups
        auto walked = [&](int64_t n_steps, int64_t workgroups) {
            const double share = (double)std::min(workgroups, most) / (double)most;
            return (double)n_steps * (k.step + k.busy * share * share);
        };
        const double full_us = k.fixed + walked(rounds * steps, most);
        auto consider = [&](int64_t workgroups, const SymCut& cut, double us) {
            if (us < best.us) best = {k.size, (int)workgroups, us, cut, {}};
        };
        consider(std::min(most, tiles), {(int)steps, (int)tiles, 0, 1, 0, 0, 0, 1}, full_us + (left > 0 ? walked(steps, left) : 0.0));
        if (left == 0) continue;
        const int whole = (int)(rounds * most), cut = (int)left;
        for (int64_t q = 2; q <= SYM_MOST_PARTS && q * left <= most && q <= steps; ++q) {
            // equal slices, of which the last may be shorter and then is a helper's
            const int64_t each = (steps + q - 1) / q, slices = steps / each, rest = steps - slices * each;
            consider(rounds > 0 ? most : left * (slices + (rest > 0)), {(int)steps, whole, cut, (int)slices, (int)each, (int)rest, rest > 0 ? cut : 0, 1},
                     full_us + walked(each, left * q) + k.leave + (double)q * k.add);
        }
        // slices and rests; the longer the slices the fewer parts the further rests come in
        const int64_t q = most / left, helpers = most - q * left, least = (left * steps + most - 1) / most;
        for (int64_t each = least; helpers > 0 && steps - q * each > 0 && each <= least + least / 2; each += std::max<int64_t>(1, least / 16)) {
            const int64_t rest = steps - q * each, further = std::max<int64_t>(0, left - helpers) * rest;
            const int64_t share = std::max<int64_t>({1, (further + helpers - 1) / helpers, std::min(rest, each - rest)}), pieces = further > 0 ? (rest - 1) / share + 2 : 1;
            if (q + pieces > SYM_MOST_PARTS) continue;
            consider(most, {(int)steps, whole, cut, (int)q, (int)each, (int)rest, (int)helpers, (int)share},
                     full_us + walked(std::max(each, rest + (further > 0 ? share : 0)), most) + 2.0 * k.leave + (double)(q + pieces) * k.add);
        }
    }
    {   // 256 x 128 tiles, all taken whole, and the diagonal's 128 x 128 ones in up to four slices behind them.  The 256 tiles of 4096 columns: 64 steps 80 us (128 x 128 tiles 92),
        // 256 steps 255 (256 x 256 ones in slices 282); 4000 columns, 125 steps 130 (128 x 128 ones in slices 147); the 1024 of 8192, 128 steps 485 (256 x 256 ones in slices 480)
        const int64_t n = (s + 255) / 256, tiles = n * n, rounds = (tiles + compute_units - 1) / compute_units, diagonal = s / 256 + (s % 256 > 128);
        const int64_t q = std::max<int64_t>(1, std::min<int64_t>({compute_units / std::max<int64_t>(1, diagonal), 4, steps}));
        const int64_t each = (steps + q - 1) / q, slices = steps / each, rest = steps - slices * each, parts = slices + (rest > 0);
        const double share = (double)tiles / (double)(rounds * compute_units);
        const double us = 8.0 + (double)(rounds * steps) * (0.70 + 0.18 * share * share) + (double)each * 0.4 + 1.5 * (double)parts;
        if (tiles >= compute_units && diagonal * parts <= compute_units && us < best.us) {
            const SymCut whole{(int)steps, (int)diagonal, 0, 1, 0, 0, 0, 1}, cut{(int)steps, 0, (int)diagonal, (int)slices, (int)each, (int)rest, rest > 0 ? (int)diagonal : 0, 1};
            best = {SYM_HALF, (int)compute_units, us, {(int)steps, (int)tiles, 0, 1, 0, 0, 0, 1}, parts == 1 ? whole : cut};
        }
    }
    return best;
}

}  // namespace axo
