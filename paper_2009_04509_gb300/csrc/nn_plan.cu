// How a launch of nn_mm.cu cuts its jobs into units of work and deals them to the CTA
// pairs.  Host arithmetic only: it compiles as plain C++, and a test runs it so.
//
// The costs below were checked against 18 shapes (256 x 92928 -> 128 to the gradients of
// 20000 x 2304 -> 512), each timed with both tile widths and the numbers of parts that
// this file considers: the plan chosen was the fastest or within 1% of it on 16 and
// within 3% on all.
#include <algorithm>

#include "nn_internal.h"

namespace emtk {
namespace {

// Time of a launch in chunks of a 256-wide tile (0.28 us), for a tile width and
// a number of parts: the most that any pair is given, plus what joining costs.
// A 128-wide tile's chunk takes 0.85 of it (half the products, but its a operand
// is staged all the same); a unit's set-up and epilogue count as 2.
double unit_cost(const MmPlan &p, const MmPlan::Piece &c) { return c.chunks_per_part * (p.tn == 256 ? 1.0 : 0.85) + 2; }

double cost_of(const MmPlan &p) {
    int at[3 * kMaxPieces + 1] = {0}, ats = 1;  // pairs where the number of some piece's units changes
    double most = 0, join = 0;
    for (int i = 0; i < p.pieces; ++i) {
        const MmPlan::Piece &c = p.piece[i];
        for (const int a : {c.pair_lo, c.pair_lo + c.pair_count, c.pair_lo + c.units % c.pair_count})
            if (a > 0 && a < p.pairs) at[ats++] = a;
        if (c.parts > 1) join += 8 + (double)c.units * (kMmTileRows * 8) * p.tn / 1.4e6;
    }
    for (int k = 0; k < ats; ++k) {
        double load = 0;
        for (int i = 0; i < p.pieces; ++i) {
            const MmPlan::Piece &c = p.piece[i];
            const int first = at[k] - c.pair_lo;
            if (first >= 0 && first < c.pair_count && first < c.units)
                load += ((c.units - first - 1) / c.pair_count + 1) * unit_cost(p, c);
        }
        most = std::max(most, load);
    }
    return most + join;
}

// Adds tiles [tile0, tile0 + tiles) of a job, their contraction in parts of at most
// `most` chunks.
void add_piece(MmPlan &p, int job, int tile0, int tiles, int most) {
    if (tiles == 0) return;
    MmPlan::Piece &c = p.piece[p.pieces++];
    const int total = p.job[job].total;
    c = {};
    c.job = job;
    c.tile0 = tile0;
    c.tiles = tiles;
    c.parts = std::max(1, (total + most - 1) / most);
    c.chunks_per_part = std::max(1, (total + c.parts - 1) / c.parts);
    c.parts = std::max(1, (total + c.chunks_per_part - 1) / c.chunks_per_part);
    c.units = tiles * c.parts;
    p.units += c.units;
}

// Deals the units out, the longest first, and returns the plan's cost.  Where a
// piece's last round leaves some pairs without one of its units, the next piece
// gives those pairs as many of its shorter units first as take the same time.
double finish_plan(MmPlan &p, int pairs) {
    p.pairs = std::min(pairs, p.units);
    MmPlan::Piece sorted[kMaxPieces];
    const int n = p.pieces;
    for (int i = 0; i < n; ++i) {
        int at = i;
        for (; at > 0 && sorted[at - 1].chunks_per_part < p.piece[i].chunks_per_part; --at) sorted[at] = sorted[at - 1];
        sorted[at] = p.piece[i];
    }
    p.pieces = 0;
    int longer = 0;  // pairs that have one of the last piece's units more than the others
    double cost = 0;
    for (int i = 0; i < n; ++i) {
        MmPlan::Piece c = sorted[i];
        const double mine = unit_cost(p, c);
        if (longer > 0 && p.pieces + (n - i) < kMaxPieces) {
            MmPlan::Piece even = c;
            even.pair_lo = longer;
            even.pair_count = p.pairs - longer;
            even.tiles = std::min(c.tiles, (int)(cost / mine + 0.5) * even.pair_count / c.parts);
            even.units = even.tiles * c.parts;
            if (even.tiles > 0) p.piece[p.pieces++] = even;
            c.tile0 += even.tiles;
            c.tiles -= even.tiles;
            c.units -= even.units;
        }
        if (c.tiles == 0) continue;
        c.pair_lo = 0;
        c.pair_count = p.pairs;
        p.piece[p.pieces++] = c;
        longer = c.units % p.pairs;
        cost = mine;
    }
    return cost_of(p);
}

}  // namespace

// Tries both tile widths and, for each, the jobs' contractions cut into parts of one
// length (few tiles, long sums) and, where the tiles fill the pairs at least once,
// the tiles of the last, partly filled round cut alone.
MmPlan plan_mm(const MmJob *jobs, int n, int sms) {
    const int pairs = std::max(1, sms / 2);
    MmPlan best{};
    double best_cost = 0;
    const bool gated = jobs[0].kind == kMmGated;
    for (const int tn : {256, 128}) {
        const int cols = gated ? tn / 2 : tn;
        MmPlan base{};
        base.tn = tn;
        int64_t tiles = 0;
        int longest = 0, long_job = 0;
        for (int i = 0; i < n; ++i) {
            MmPlan::Job &c = base.job[i];
            c.tiles_m = (int)(((int64_t)jobs[i].M + kMmTileRows - 1) / kMmTileRows);
            c.tiles_n = (int)(((int64_t)jobs[i].N + cols - 1) / cols);
            c.chunks = (int)(((int64_t)jobs[i].K + kMmStep - 1) / kMmStep);
            c.total = c.chunks * jobs[i].terms;
            tiles += (int64_t)c.tiles_m * c.tiles_n;
            if (c.total > longest) {
                longest = c.total;
                long_job = i;
            }
        }
        auto consider = [&](MmPlan &p) {
            const double cost = finish_plan(p, pairs);
            if (best.tn == 0 || cost < best_cost) {
                best = p;
                best_cost = cost;
            }
        };
        // parts of at least 4 chunks, as many as pairs at most
        for (int d = 1; d == 1 || (longest / d >= 4 && d <= pairs); d += std::max(1, d / 4)) {
            MmPlan p = base;
            for (int i = 0; i < n; ++i)
                add_piece(p, i, 0, p.job[i].tiles_m * p.job[i].tiles_n, std::max(1, (longest + d - 1) / d));
            consider(p);
        }
        // the last round's tiles, of the job with the longest units
        const int of_long = base.job[long_job].tiles_m * base.job[long_job].tiles_n;
        const int rest = (int)(tiles % pairs);
        if (tiles <= pairs || tiles > 40 * pairs || rest == 0 || rest > of_long) continue;
        for (int d = 2; longest / d >= 4 && d <= pairs; d += std::max(1, d / 2)) {
            MmPlan p = base;
            for (int i = 0; i < n; ++i) {
                const int all = p.job[i].tiles_m * p.job[i].tiles_n, cut = i == long_job ? rest : 0;
                add_piece(p, i, 0, all - cut, std::max(1, p.job[i].total));
                add_piece(p, i, all - cut, cut, (longest + d - 1) / d);
            }
            consider(p);
        }
    }
    for (int i = 0; i < best.pieces; ++i) {
        MmPlan::Piece &c = best.piece[i];
        if (c.parts == 1) continue;
        c.part_at = (int64_t)(best.workspace / sizeof(float));
        best.workspace += (size_t)c.units * kMmTileRows * best.tn * sizeof(float);
    }
    return best;
}

}  // namespace emtk
