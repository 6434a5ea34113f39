// How the attention of one new token is split over the chip and laid out in its workspace.  Plain C++, also for the kernels.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace metok {

constexpr int kAttendWaves = 4, kAttendThreads = 64 * kAttendWaves;
constexpr int kAttendRows = 16;                // query rows of a workgroup: one MFMA's columns
// Workgroups that share the rows of all videos, and the fewest tiles (of 32 or 16 rows) that one takes.
#ifndef TGT
#define TGT 512
#define MINT 4
#endif
constexpr int kAttendTarget = TGT, kAttendMinTiles = MINT;

// Cache rows of a wave's tile: K and V of the next one are on their way in registers, 64 of them at most.
constexpr int attend_tile(int esize, int dh) { return esize * dh <= 256 && esize == 2 ? 32 : 16; }

struct AttendPlan {
    int tile;              // cache rows of a tile
    int row_blocks;        // blocks of kAttendRows query heads of a kv head
    int rows;              // query rows of a partial result
    int64_t pairs;         // (video, kv head, row block): what is split over the rows of the cache
    int64_t grid;          // workgroups, and slots for partial results
    bool joined;           // false: every pair is one workgroup's, whatever the lengths
    int64_t logit_stride;  // logits of a (video, query head), 0: not kept
    size_t part_ml, part_o, lse2, logits, bytes;       // offsets in the workspace, and its size
};

// Tiles a workgroup takes at most, from the tiles of all pairs: kAttendTarget + pairs workgroups are enough for any lengths, because
// a pair has at most one workgroup more than its share.
constexpr int64_t attend_tiles_per_group(int64_t tiles_of_pairs) {
    const int64_t share = (tiles_of_pairs + kAttendTarget - 1) / kAttendTarget;
    return share > kAttendMinTiles ? share : kAttendMinTiles;
}

// `capacity` rows at most, one more with a new row.
constexpr AttendPlan plan_attend(int B, int Hq, int Hkv, int64_t capacity, int dh, int esize, bool with_weight) {
    AttendPlan p{};
    const int group = Hq / Hkv;
    p.tile = attend_tile(esize, dh);
    p.row_blocks = (group + kAttendRows - 1) / kAttendRows;
    p.rows = group < kAttendRows ? group : kAttendRows;
    p.pairs = static_cast<int64_t>(B) * Hkv * p.row_blocks;
    const int64_t most = (capacity + 1 + p.tile - 1) / p.tile;                       // tiles of the longest video
    const int64_t splits = (most + kAttendMinTiles - 1) / kAttendMinTiles;
    p.joined = splits > 1;
    p.grid = p.pairs + kAttendTarget;
    if (splits <= kAttendTarget && p.pairs * splits < p.grid) p.grid = p.pairs * splits;
    p.logit_stride = with_weight ? (capacity + 1 + 31) / 32 * 32 : 0;
    size_t at = 0;
    auto take = [&at](size_t floats) {
        const size_t here = at;
        at += (floats * sizeof(float) + 255) / 256 * 256;
        return here;
    };
    const size_t slots = p.joined ? static_cast<size_t>(p.grid) * p.rows : 0;
    p.part_ml = take(slots * 2);
    p.part_o = take(slots * dh);
    p.lse2 = take(with_weight ? static_cast<size_t>(B) * Hq : 0);
    p.logits = take(static_cast<size_t>(B) * Hq * static_cast<size_t>(p.logit_stride));
    p.bytes = at;
    return p;
}

}  // namespace metok
