// ortho_plan.cpp -- the split of a call's matrices over ortho.hip's kernels.
#include "ortho_plan.hpp"

#include <cmath>

#include "norm.hpp"

namespace qlayer {
namespace {

// What a launch with tiles of a size costs, in us, from measured kernels: a
// main-loop step of a workgroup that has its compute unit for itself, of one
// that shares it (two of the smaller tiles fit one), and what a tile costs
// besides its steps. fp64 has one tile size.
struct TileCost {
    double alone, shared, rest;
};
constexpr TileCost COST[4] = {{0.25, 0.45, 2}, {0.58, 1.10, 8}, {1.00, 1.00, 12}, {1.6, 1.6, 20}};
constexpr int UNITS = 256;  // compute units

double launch_cost(int mode, int which, int splits, const Chunk& c) {
    const TileCost& t = COST[which];
    const int64_t bt = TILES[which], slots = which < 2 ? 2 * UNITS : UNITS;
    double alone = 0, shared = 0, longest = 0;  // sums over workgroups, and the longest one
    int64_t tiles = 0;
    for (int k = 0; k < c.count; k++) {
        const int64_t n = c.batch[k] * tiles_of(mode, bt, c.shape[k].m, c.shape[k].n);
        const int64_t whole = up64(mode == GRAM ? c.shape[k].n : c.shape[k].m) * unit_of(TWO) / 128;
        const double steps = (double)((whole + splits - 1) / splits);
        tiles += n;
        alone += (double)(n * splits) * (steps * t.alone + t.rest);
        shared += (double)(n * splits) * (steps * t.shared + t.rest);
        longest = std::max(longest, steps * t.alone + t.rest);
    }
    if (!tiles) return 0;
    const int64_t groups = tiles * splits, rounds = groups / slots, rest = groups % slots;
    double cost = std::max(longest, rounds * shared / groups + (rest ? (rest <= UNITS ? alone : shared) / groups : 0));
    // the second launch, and the sums' way to memory (3 TB/s) and back
    if (splits > 1) cost += 3 + t.rest + 0.1 * splits + (double)groups * bt * bt * 8 / 3e6;
    return cost;
}

}  // namespace

bool is_small(int type, const Shape& s) {
    if (s.m > SMALL_M) return false;
    if (type == E_F64) return small_lds(s.m, s.n, 8) <= SMALL_LDS;
    return tiny_lds(s.m, s.n) <= TINY_LDS;
}

int chunks_of(const Shape& s) {
    return (int)std::min<int64_t>(std::min(s.m, 1024), std::max<int64_t>(1, (int64_t)s.m * s.n / 4096));
}

int64_t large_bytes(int format, const Shape& s) {
    return layout_of((int)up64(s.m), (int)up64(s.n), unit_of(format)).size;
}
int64_t norm_bytes(const Shape& s) { return ((chunks_of(s) + 1) * 8 + 255) / 256 * 256; }

bool all_small(int type, const ql_matrix* mats, int count) {
    for (int k = 0; k < count; k++)
        if (mats[k].batch > 0 && !is_small(type, shape_of(mats[k]))) return false;
    return true;
}

Scales scales_of(const OrthoCall& c) {
    double most_x = 1, most_q = 1;
    ortho_bounds(c.a, c.b, c.c, c.steps, most_x, most_q);
    // |a + b t + c t^2| over t = x^2 from 0 on, at its ends and its extremum
    const double most_t = most_x * most_x, inner = c.c != 0 ? -c.b / (2 * c.c) : 0;
    auto factor = [&](double t) { return std::fabs(c.a + t * (c.b + c.c * t)); };
    double most = std::max(factor(0), factor(most_t));
    if (inner > 0 && inner < most_t) most = std::max(most, factor(inner));
    const double growth = std::log2(std::max(most, 1e-30)) + std::log2(1 + 1.0 / 256);  // the margin of ortho_bounds
    return {std::exp2(std::floor(std::log2(32768 / most_x))), std::exp2(std::floor(std::log2(32768 / (most_x * most_x)))),
            std::exp2(std::floor(std::log2(32768 / std::max(most_q, 1e-3)))), growth};
}

int64_t tiles_of(int mode, int64_t bt, int m, int n) {
    const int64_t mt = (up64(m) + bt - 1) / bt, nt = (up64(n) + bt - 1) / bt;
    return mode <= POLY ? mt * (mt + 1) / 2 : mt * nt;
}

Choice choose(int format, int mode, const Chunk& c) {
    Choice best;
    if (format == DOUBLE) return best;
    // sums over a long side of few rows are for the tiles that fold them
    bool wide = false;
    for (int k = 0; k < c.count; k++) wide |= c.shape[k].n > std::max<int64_t>(FOLDED, 4 * (int64_t)c.shape[k].m);
    double least = 0;
    for (int which = 0; which < (mode == GRAM && wide ? 2 : 4); which++) {
        int64_t tiles = 0;
        for (int k = 0; k < c.count; k++) tiles += c.batch[k] * tiles_of(mode, TILES[which], c.shape[k].m, c.shape[k].n);
        for (int splits = 1; splits == 1 || (mode == GRAM && which < 2 && splits <= 64 && tiles * splits <= 2 * UNITS);
             splits = splits < 4 ? splits + 1 : splits * 3 / 2) {
            const double cost = launch_cost(mode, which, splits, c);
            if ((which == 0 && splits == 1) || cost < least) least = cost, best.which = which, best.splits = splits;
        }
    }
    if (best.splits > 1)
        for (int k = 0; k < c.count; k++)
            best.bytes += c.batch[k] * tiles_of(mode, TILES[best.which], c.shape[k].m, c.shape[k].n) * best.splits * TILES[best.which] * TILES[best.which] * 4;
    return best;
}

int next_chunk(const ql_matrix* mats, int count, int at, Chunk& c, const ql_matrix** entry) {
    for (c.count = 0; at < count && c.count < ENTRIES; at++)
        if (mats[at].batch > 0) {
            c.shape[c.count] = shape_of(mats[at]);
            c.batch[c.count] = mats[at].batch;
            if (entry) entry[c.count] = &mats[at];
            c.count++;
        }
    return at;
}

bool ortho_bounds(double a, double b, double c, int steps, double& most_x, double& most_q) {
    most_x = 1, most_q = 0;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    // over t = x^2: where p' = a + 3 b t + 5 c t^2 and q' = b + 2 c t vanish
    double inner[3];
    int n = 0;
    const double disc = 9 * b * b - 20 * a * c;
    if (c != 0) inner[n++] = -b / (2 * c);
    if (disc >= 0) {  // both roots without a difference of nearly equal numbers
        const double h = -(3 * b + std::copysign(std::sqrt(disc), b)) / 2;
        if (c != 0) inner[n++] = h / (5 * c);
        if (h != 0) inner[n++] = a / h;
    }
    double reach = 1;  // singular values lie in [0, reach]
    for (int s = 0; s < steps; s++) {
        double next = 0;
        for (int k = 0; k <= n; k++) {
            const double t = k < n ? inner[k] : reach * reach;
            if (!(t >= 0 && t <= reach * reach)) continue;
            const double q = t * (b + c * t), v = std::fabs(std::sqrt(t) * (a + q));
            if (!(v <= 1e6) || !(std::fabs(q) <= 1e5)) return false;
            next = std::max(next, v);
            most_q = std::max(most_q, std::fabs(q));
        }
        if (s + 1 == steps) break;  // what the last step gives is not held
        reach = next * (1 + 1.0 / 256);  // and a margin for the products' rounding
        most_x = std::max(most_x, reach);
        if (reach > 64) return false;
    }
    return true;
}

bool ortho_launchable(int type, const ql_matrix* mats, int count) {
    if (all_small(type, mats, count)) return true;
    // no launch has more workgroups than one for every 64x64 of X (the norm's take
    // 4096 elements or more, and what a split adds stays below 2 UNITS), of at most 512 threads
    int64_t tiles = 0;
    for (int k = 0; k < count; k++) {
        const Shape s = shape_of(mats[k]);
        tiles += mats[k].batch * tiles_of(APPLY, 64, s.m, s.n);
    }
    return tiles < ((int64_t)1 << 32) / 512;
}

size_t ortho_workspace(int type, const ql_matrix* mats, int count) {
    if (all_small(type, mats, count)) return 0;
    const int format = type == E_F64 ? DOUBLE : TWO;
    int64_t bytes = 0;
    for (int at = 0; at < count;) {
        Chunk c;
        at = next_chunk(mats, count, at, c, nullptr);
        for (int k = 0; k < c.count; k++) bytes += c.batch[k] * (large_bytes(format, c.shape[k]) + norm_bytes(c.shape[k]));
        bytes += choose(format, GRAM, c).bytes;
    }
    return (size_t)bytes;
}

}  // namespace qlayer
