// How the keys that groups of sequences have in common are cut into units, and the units dealt out to workgroups.  Nothing of HIP in here: the
// kernel and a host test that walks plans share the functions.
//
// Work is counted in weighted steps: a step is 64 keys met by one tile of columns of one KV head.  Shared keys weigh `shared` in all, the
// sequences' own ones `own`; of the launch's workgroups the first ones take units, the others own keys, and the launch takes as long as the
// slower kind.
#pragma once
#include <stdint.h>

#ifdef __HIP__
#define SHIFTATTN_BOTH __host__ __device__ inline   // (the compiler for the card takes no square roots in constant expressions)
#else
#define SHIFTATTN_BOTH inline
#endif

namespace shiftattn {
namespace shared_deal {

constexpr int kWorkgroups = 512;      // two resident per compute unit
constexpr int kMostShared = 508;      // workgroups that take shared keys at most
constexpr int kStep = 64;             // keys that shared ranges are counted in
constexpr int kTileCols = 128;        // (sequence, head) columns of a tile whose keys a workgroup's wavefronts share
// Columns of a tile that every wavefront takes with keys of its own, where a group has no more: 32 columns of one group of 20000 tokens 16.4
// us against 17.2 with a wide tile, 16 columns of 24 groups in FP8 27.1 against 29.9, in bf16 27.3 against 25.0.  With narrow tiles up to 64
// columns, 10 groups of 40 columns took 27.0 us against 25.4 with wide ones, one of 40 18.1 against 17.4, one of 64 18.9 against 17.9.
constexpr int kNarrowCols = 32;
// Least steps of a range, by the square root of a group's steps: a range that is too short costs more in the merge than it saves here (a step
// takes about as long as 16 parts of a row).  Between 0.12 and 0.6 no batch changes by more than 3 %.
constexpr float kRangeRoot = 0.25f;
// Time of a step of either kind of tile, and of 32 tokens for each of a workgroup's wavefronts, which have one group of 32 on its way each: 2 us
// in bf16 as in FP8.  With 2 for those, 180 sequences of up to 600 tokens behind 20000 took 55.0 us (39.6 with 4; FP8 50.9 and 42.7), 10 groups
// of 8 behind 6000 28.5 (24.5; 26.1 and 23.2), 8 groups over an FP8 cache 44.0 (44.1 to 45.5); with 6 these took 47.0.  Narrow steps at 2: within
// 1 % in those batches, 30 groups of 3 behind 3000 tokens 134 us against 121.
constexpr int kWideCost = 3, kNarrowCost = 1, kOwnCost = 4;
// What a unit takes beside its keys (block ids, queries, the first keys, the parts it writes: a chain of loads), and a step of a narrow tile among
// many, where memory sets the pace: half of the own keys' 128 tokens.  They count where workgroups take several units, and where it is asked if
// sharing pays.
constexpr int kUnitCost = 6, kNarrowAmong = 2;

// columns of a tile of a group that has so many, and its tiles
SHIFTATTN_BOTH int tile_cols(int cols) { return cols > kNarrowCols ? kTileCols : kNarrowCols; }
SHIFTATTN_BOTH int tiles_of(int cols) { return (cols + tile_cols(cols) - 1) / tile_cols(cols); }
SHIFTATTN_BOTH int cost_of(int cols) { return cols > kNarrowCols ? kWideCost : kNarrowCost; }
SHIFTATTN_BOTH int steps_of(int blocks) { return (blocks + 3) / 4; }

// steps of a unit that is one of many, and the unit
SHIFTATTN_BOTH int among(int steps, int cols) { return kUnitCost + steps * (cols > kNarrowCols ? kWideCost : kNarrowAmong); }
// Do the tiles of a group with so many blocks in common take less than its members take with those blocks each for itself?  512 pairs with four
// blocks in common: 212 us if they share those, 205 if they do not (the plain kernel 198).
SHIFTATTN_BOTH bool pays(int blocks, int members, int cols) {
    return static_cast<float>(tiles_of(cols)) * among(steps_of(blocks), cols) < 0.25f * kOwnCost * members * blocks / 2;
}

// The weight of a range: an even part of all work.  (Shared keys over whole workgroups, at least one, made 2000 tokens of 4 sequences one range that
// 60 others waited for: 43 us, where this takes 36.)
SHIFTATTN_BOTH int range_of(float shared, float own) { return static_cast<int>(__builtin_ceilf((shared + own) / kWorkgroups)); }

// ranges that the keys of a tile are cut into (range_min: steps that a range has at least), and steps of one of them
SHIFTATTN_BOTH int ranges_of(int steps, int cols, int range, int range_min) {
    const int cost = cost_of(cols), by_root = static_cast<int>(__builtin_sqrtf(static_cast<float>(steps)) * kRangeRoot);
    int per = (range + cost - 1) / cost;
    per = per > by_root ? per : by_root;
    per = per > range_min ? per : range_min;
    const int ranges = (steps + per - 1) / per;
    // workgroup i runs on die i % 8: with a multiple of 4 ranges the tiles and heads of a group find the same keys in the L2 of one die, or of
    // two (210 MB fetched from memory become 41 where 2048 columns meet 32768 tokens, 17 MB of keys)
    return ranges >= 16 && cols > kTileCols ? ranges & ~3 : ranges;
}
SHIFTATTN_BOTH int range_steps(int steps, int ranges) { return (steps + ranges - 1) / ranges; }

// Is a workgroup for each of `all` units, whose steps weigh `shared`, the best there is?  Where the own keys take no longer than the mean unit.
SHIFTATTN_BOTH bool one_each(int all, float shared, float own) {
    return all <= kMostShared && own * all <= (shared + static_cast<float>(kUnitCost) * all) * (kWorkgroups - all);
}

// Workgroups for `all` units of shared keys that weigh `shared` together and `longest` at most (by `among`).  With m of them, and units that follow
// each other, the shared part takes up to shared / m + longest, which meets the own keys' own / (kWorkgroups - m) at the root of
//     longest m^2 + (shared + own - longest kWorkgroups) m - kWorkgroups shared = 0;
// with a workgroup for one, two or three units it takes one, two or three times `longest`.  The fastest of these.
// 64 prompts of 1000 tokens with two answers each, 8 KV heads: 165 us (FP8 91), where a workgroup for every unit, however short, left four to
// the own keys and took 2585 (the plain kernel 182, 98); 30 groups of 3 behind 3000 tokens 106 (140, and 121 without the multiples of `longest`; plain 197).
SHIFTATTN_BOTH int workgroups_of(int all, float shared, float longest, float own) {
    const float b = shared + own - longest * kWorkgroups, root = __builtin_sqrtf(b * b + 4.f * kWorkgroups * longest * shared);
    const float meet = b > 0.f ? 2.f * kWorkgroups * shared / (b + root) : (root - b) / (2.f * longest);
    const int most = all < kMostShared ? all : kMostShared;
    int best = meet < 1.f ? 1 : meet < static_cast<float>(most) ? static_cast<int>(meet) : most;
    const float own_best = own / (kWorkgroups - best), shared_best = shared / best + longest;
    float least = own_best > shared_best ? own_best : shared_best;
    for (int k = 3; k > 0; --k) {
        const int n = (all + k - 1) / k;
        if (n > kMostShared) break;
        const float own_n = own / (kWorkgroups - n), time = own_n > k * longest ? own_n : k * longest;
        if (time <= least) best = n, least = time;
    }
    return best;
}

// Of n < all workgroups number i takes the units that begin at weights [first_of(i), first_of(i + 1)) of the line of all units.
SHIFTATTN_BOTH uint32_t first_of(uint32_t shared, int n, int i) { return shared / n * i + shared % n * i / n; }
// units of a group that begin in front of weight x: the group has n units of weight `each`, the first of which begins at `first`
SHIFTATTN_BOTH int units_before(uint32_t x, uint32_t first, uint32_t each, int n) {
    if (x <= first) return 0;
    const uint32_t k = (x - first + each - 1) / each;
    return k < static_cast<uint32_t>(n) ? static_cast<int>(k) : n;
}

}  // namespace shared_deal
}  // namespace shiftattn

#undef SHIFTATTN_BOTH
