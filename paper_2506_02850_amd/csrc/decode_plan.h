// How the attention of one new token is split over the chip and laid out in its workspace.  Plain C++, also for the kernels.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace metok {

constexpr int kAttendWaves = 4, kAttendThreads = 64 * kAttendWaves;
constexpr int kAttendRows = 16;                // query rows of a block: one MFMA's columns
// Blocks of a wave where a kv head has more than one: four where they fit the registers beside K, V and the sums and more than two are there
// (8 x 149990 rows of 64 elements, 24 query heads on one kv head: 85 us with four, 62 with two; 48 of them 84 and 97; 71 of them 147 and 159, but 48
// and 44 with 36990 rows, which stay in the caches between the turns).
constexpr int attend_blocks(int dh, int group) { return dh <= 64 && group > 2 * kAttendRows ? 4 : 2; }
// Cache rows of a tile: K and V of the next one are on their way in registers, 64 of them at most.
constexpr int attend_tile(int esize, int dh) { return esize * dh <= 256 && esize == 2 ? 32 : 16; }
// Workgroups of a large call: one per CU, two where a tile is only 4 KB (8 x 73980 rows of 4 heads of 32 bf16: 68 us with one, 57 with two, 57 with
// four; of 2 heads of 64: 58, 62).
constexpr int attend_groups(int esize, int dh) { return 2 * attend_tile(esize, dh) * esize * dh <= 4096 ? 512 : 256; }

// Capacities of up to so many tiles (no weights, at most 16 query heads to a kv head) take a workgroup of eight waves per pair and no second
// launch.  With more tiles than that few pairs leave most of the chip idle.  One video, 28 heads on 4 of 128: 128 rows 4.4 us (8.9 split over
// all CUs and joined), 512 rows 7.8 (8.9), 1024 rows, 33 tiles, 12.3 (9.0); 64 of them 6.0 (12.4), 13.0 (19.4), 27.6 (33.9), 256 17.4 (22.1),
// 51.4 (50.6), 96 (87); 2 videos of 14 heads on 2 of 64 in fp32, tiles of 16 rows: 256 rows 6.0 (8.4); 2 of 8 on 2 of 256: 512 rows, 33
// tiles, 12.7 (8.8).
constexpr int kAttendWholeWaves = 8, kAttendWhole = 32;

// The tiles of all (video, kv head, row block) pairs, one pair behind the other, are dealt out evenly to the waves, the workers.  The end of a
// pair takes a worker about as long as a tile, so every pair counts kAttendPairCost tiles more than it has; they lie behind its own (32 videos of 0
// to 8191 rows, 32 heads on 8: 41 us without, 32 with one, 31.5 with two; many short pairs fell to few workers).
// Worker w of n has units [w T / n, (w + 1) T / n), or kAttendMinTiles of them where there are few (2307 rows of 28 heads on 4: 9.2 us with one, 9.3
// with two, 11 with four; 2 x 5033 of 14 on 2 in fp32: 12.3, 10.7, 11.1: with one there are more parts to join).
constexpr int kAttendMinTiles = 2, kAttendPairCost = 1;
template <int GROUPS, int MIN_TILES = kAttendMinTiles, int PAIR_COST = kAttendPairCost> struct Deal {
    static constexpr int kWorkers = GROUPS * kAttendWaves, kPairCost = PAIR_COST;
    static_assert((kWorkers & (kWorkers - 1)) == 0, "a worker's first unit is a shift away");
    static constexpr int64_t workers(int64_t units) {
        const int64_t few = (units + MIN_TILES - 1) / MIN_TILES;
        return few < kWorkers ? few : kWorkers;
    }
    static constexpr int64_t first(int64_t worker, int64_t units) {
        const int64_t at = units < static_cast<int64_t>(MIN_TILES) * kWorkers ? worker * MIN_TILES : worker * units / kWorkers;
        return at < units ? at : units;
    }
    // Whether a worker's whole workgroup, of kAttendWaves workers that follow each other, is in the middle of the pair in which the worker begins at tile t.
    static constexpr bool in_the_middle(int64_t worker, int64_t units, int64_t t, int64_t tiles) {
        const int64_t group = worker / kAttendWaves * kAttendWaves, mine = first(worker, units);
        return t - (mine - first(group, units)) > 0 && t + (first(group + kAttendWaves, units) - mine) < tiles;
    }
};

// The partial results of a pair of the workers first .. last.  A worker leaves at most two: of the pair that an earlier worker began (slot 2 w) and of the one that
// it begins and a later one ends (slot 2 w + 1).  With teams a workgroup in the middle of the pair leaves one, its first worker's.
struct PairParts {
    int first, n, alone, teams;                    // `alone` of the first worker's workgroup, or all; behind them those of the teams
    constexpr int slot(int p) const {
        int worker = first + p;
        if (p >= alone) {
            const int behind = p - alone, team = behind < teams ? behind : teams;
            worker = (first / kAttendWaves + 1 + team) * kAttendWaves + (behind - team);
        }
        return 2 * worker + (p == 0);
    }
};
constexpr PairParts pair_parts(int first, int last, bool teams) {
    const int n = last - first + 1, between = last / kAttendWaves - first / kAttendWaves - 1;        // workgroups
    if (!teams || between <= 0) return {first, n, n, 0};
    return {first, n - (kAttendWaves - 1) * between, kAttendWaves - first % kAttendWaves, between};
}

struct AttendPlan {
    int tile;              // cache rows of a tile
    bool wide;             // several blocks of query heads of a kv head at a time
    int block_rows;        // query heads of a kv head that are taken at a time, at most
    int row_blocks;        // how often the rows are read for the query heads of a kv head
    int rows;              // query rows of a partial result
    int64_t pairs;         // (video, kv head, row block): what is split over the rows of the cache
    int64_t grid;          // workgroups
    int64_t workers;       // at most
    bool whole;            // a workgroup to a pair, no second launch and no workspace
    bool joined;           // false: every pair is one tile, whatever the lengths
    bool teams;            // a workgroup in the middle of a pair leaves one part
    int64_t logit_stride;  // logits of a (video, query head), 0: not kept
    size_t pair_workers, part_ml, part_o, lse2, logits, bytes;       // offsets in the workspace, and its size
                           // (lse2: a head's maximum and 1 / sum, what the logarithm of its sum is made of)
};

// What the split goes by beside the shapes: cache rows of a tile, workgroups of a large call, blocks of 16 query heads that a wave takes at a time where a
// kv head has more than one, up to how many tiles a pair is left to one workgroup, units a worker has at least and a pair's end counts, and whether the workers of
// a workgroup may join what they leave of a pair.
struct AttendSplit { int tile, groups, blocks, whole, min_tiles, pair_cost; bool teams; };

// `capacity` rows at most, one more with a new row.
constexpr AttendPlan plan_split(int B, int Hq, int Hkv, int64_t capacity, int dh, const AttendSplit& split, bool with_weight) {
    AttendPlan p{};
    const int group = Hq / Hkv;
    p.tile = split.tile;
    p.wide = group > kAttendRows;
    p.block_rows = kAttendRows * (p.wide ? split.blocks : 1);
    p.row_blocks = (group + p.block_rows - 1) / p.block_rows;
    p.rows = group < p.block_rows ? group : p.block_rows;
    p.pairs = static_cast<int64_t>(B) * Hkv * p.row_blocks;
    const int64_t most = (capacity + 1 + p.tile - 1) / p.tile;                       // tiles of the longest video
    p.whole = !p.wide && !with_weight && most <= split.whole;
    p.joined = most > 1 && !p.whole;
    const int groups = split.groups;
    const int64_t few = ((most + split.pair_cost) * p.pairs + split.min_tiles - 1) / split.min_tiles;      // workers, with a workgroup each
    p.grid = few < groups ? few : groups;
    p.teams = split.teams && few > groups;                                           // by the capacity, as the grid
    p.workers = static_cast<int64_t>(groups) * kAttendWaves;
    p.logit_stride = with_weight ? (capacity + 1 + 31) / 32 * 32 : 0;                // whole tiles are written, of 16 or 32 rows
    size_t at = 0;
    auto take = [&at](size_t floats) {
        const size_t here = at;
        at += (floats * sizeof(float) + 255) / 256 * 256;
        return here;
    };
    p.pair_workers = take(p.joined || with_weight ? static_cast<size_t>(p.pairs) * 2 : 0);
    const size_t slots = p.joined ? static_cast<size_t>(2 * p.workers) * p.rows : 0;
    p.part_ml = take(slots * 2);
    p.part_o = take(slots * dh);
    p.lse2 = take(with_weight ? static_cast<size_t>(B) * Hq * 2 : 0);
    p.logits = take(static_cast<size_t>(B) * Hq * static_cast<size_t>(p.logit_stride));
    p.bytes = at;
    return p;
}
constexpr AttendPlan plan_attend(int B, int Hq, int Hkv, int64_t capacity, int dh, int esize, bool with_weight) {
    return plan_split(B, Hq, Hkv, capacity, dh, {attend_tile(esize, dh), attend_groups(esize, dh), attend_blocks(dh, Hq / Hkv), kAttendWhole, kAttendMinTiles, kAttendPairCost, false}, with_weight);
}

// The same over a cache in 4 bits (kv4_attention.hip).  A row has a quarter of the bytes, so it takes two waves to a SIMD to keep enough of them on their way, and
// tiles of 32 rows at any width (28 heads on 4 of 128, 8 x 36992 rows: 31.3 us with 512 workgroups, 41.3 with 256; 32 videos of 0 to 8191 rows 15.6 and 19.5.  Tiles
// of 64 rows in 256 workgroups take as long at 8 x 36992, but 2307 rows 6.2 us against 5.4, 8 x 3000 of 256 elements 11.3 against 8.4).
constexpr int kAttend4Tile = 32, kAttend4Groups = 512;
static_assert(32 % kAttend4Tile == 0, "32 logits hold whole tiles");
// A pair per workgroup up to 32 tiles, as above.  28 heads on 4 of 128: 120 rows 5.0 us (9.6 split and joined), 1000 rows 8.2 (9.6), 16 of them 8.9
// (11.1), 64 of them 10.4 (18.1); 2000 rows 12.1 (9.6), 16 of them 14.1 (13.0).  The rule knows the tiles and not whether the pairs alone fill the chip: 64 videos of 2000
// rows, 256 pairs, would take 15.6 us in one launch and take 23.1.
constexpr int kAttend4Whole = 32;
// A tile is read in a quarter of the time, and what a worker does before the first and behind the last one counts for more: tiles go to workers one by one where they are
// few, and a pair's end is two of them (8 x 700 to 3000 rows of 256 elements 8.6 us with two tiles at least and an end of one, 7.7 with one and one, 7.4 with one
// and two, 7.2 with one and three; 32 videos of 0 to 8191 rows 15.8, 15.7, 14.0, 14.1; 2307 rows 5.5, 5.5, 5.3, 5.6).
constexpr int kAttend4MinTiles = 1, kAttend4PairCost = 2;
typedef Deal<kAttend4Groups, kAttend4MinTiles, kAttend4PairCost> Deal4;
constexpr AttendPlan plan_attend4(int B, int Hq, int Hkv, int64_t capacity, int dh, bool with_weight) {
    return plan_split(B, Hq, Hkv, capacity, dh, {kAttend4Tile, kAttend4Groups, 1, kAttend4Whole, kAttend4MinTiles, kAttend4PairCost, true}, with_weight);
}

}  // namespace metok
