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
template <int GROUPS> struct Deal {
    static constexpr int kWorkers = GROUPS * kAttendWaves;
    static_assert((kWorkers & (kWorkers - 1)) == 0, "a worker's first unit is a shift away");
    static constexpr int64_t workers(int64_t units) {
        const int64_t few = (units + kAttendMinTiles - 1) / kAttendMinTiles;
        return few < kWorkers ? few : kWorkers;
    }
    static constexpr int64_t first(int64_t worker, int64_t units) {
        const int64_t at = units < static_cast<int64_t>(kAttendMinTiles) * kWorkers ? worker * kAttendMinTiles : worker * units / kWorkers;
        return at < units ? at : units;
    }
};

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
    int64_t logit_stride;  // logits of a (video, query head), 0: not kept
    size_t pair_workers, part_ml, part_o, lse2, logits, bytes;       // offsets in the workspace, and its size
                           // (lse2: a head's maximum and 1 / sum, what the logarithm of its sum is made of)
};

// `capacity` rows at most, one more with a new row.
constexpr AttendPlan plan_attend(int B, int Hq, int Hkv, int64_t capacity, int dh, int esize, bool with_weight) {
    AttendPlan p{};
    const int group = Hq / Hkv;
    p.tile = attend_tile(esize, dh);
    p.wide = group > kAttendRows;
    p.block_rows = kAttendRows * (p.wide ? attend_blocks(dh, group) : 1);
    p.row_blocks = (group + p.block_rows - 1) / p.block_rows;
    p.rows = group < p.block_rows ? group : p.block_rows;
    p.pairs = static_cast<int64_t>(B) * Hkv * p.row_blocks;
    const int64_t most = (capacity + 1 + p.tile - 1) / p.tile;                       // tiles of the longest video
    p.whole = !p.wide && !with_weight && most <= kAttendWhole;
    p.joined = most > 1 && !p.whole;
    const int groups = attend_groups(esize, dh);
    const int64_t few = ((most + kAttendPairCost) * p.pairs + kAttendMinTiles - 1) / kAttendMinTiles;      // workers, with a workgroup each
    p.grid = few < groups ? few : groups;
    p.workers = static_cast<int64_t>(groups) * kAttendWaves;
    p.logit_stride = with_weight ? (capacity + 1 + 31) / 32 * 32 : 0;
    size_t at = 0;
    auto take = [&at](size_t floats) {
        const size_t here = at;
        at += (floats * sizeof(float) + 255) / 256 * 256;
        return here;
    };
    p.pair_workers = take(p.joined || with_weight ? static_cast<size_t>(p.pairs) * 2 : 0);
    // a worker leaves at most two partial results: of the pair that an earlier worker began (slot 2 w) and of the one that it begins and a
    // later one ends (slot 2 w + 1)
    const size_t slots = p.joined ? static_cast<size_t>(2 * p.workers) * p.rows : 0;
    p.part_ml = take(slots * 2);
    p.part_o = take(slots * dh);
    p.lse2 = take(with_weight ? static_cast<size_t>(B) * Hq * 2 : 0);
    p.logits = take(static_cast<size_t>(B) * Hq * static_cast<size_t>(p.logit_stride));
    p.bytes = at;
    return p;
}

}  // namespace metok
