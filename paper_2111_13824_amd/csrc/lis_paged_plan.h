// How a call of the attention over a paged cache is divided: chosen on the host from
// its sizes alone (lengths are device data).
#pragma once

#include <stdint.h>

#include "stream_internal.h"

namespace fqvit {
namespace paged {

constexpr int kTile = 64;           // keys a wavefront takes at a time

// One launch whose passes take the logits again; one for at most 16 rows, which keeps
// them in LDS; three launches over parts of the keys, without and (at most 16 rows) with
// the logits in the workspace.
enum Way { kOne, kOneFew, kParts, kPartsFew };

// Logits of a workgroup that LDS holds beside two stages, the buckets and the rest.
constexpr int64_t kLdsLogits = 16384;

// Logits that the workspace holds: 1 GiB.  They are as many as the table can name, whatever the
// lengths are (which are on the device), and tables of 2^20 keys for 128 key heads of 16 rows
// would take 8 GiB.  Calls beyond it take the logits again, as those of more rows do, which
// costs most with few rows and long sequences: tables of 131072 keys for 512 key heads of 64
// channels, stored to again, a row (256 MiB) 24 us to 25, 64 to 99 and 236 to 404 of 512, 4096 and
// 16384 keys, 4 rows (1 GiB) 26 to 25, 79 to 99 and 313 to 405, 8 rows (2 GiB) 31 to 25, 109 to
// 100 and 440 to 405; heads of 128, 8 rows, 39 to 32, 166 to 175 and 608 to 717.
constexpr int64_t kMostLogits = (int64_t)1 << 28;

struct Plan {
    Way way;
    int32_t splits;         // parts of the keys, each a workgroup's
    int32_t tile_rows;      // rows of a workgroup
    int32_t tiles;          // workgroups over the rows of a sequence and key head
    int32_t rows;           // rows of a sequence and key head
    int64_t units;          // sequences times key heads
    int64_t keys;           // keys a table names, up to a multiple of 64

    // workspace of a divided call: of every row its sum (64 bits), its maximum and its
    // parts' maxima (int32), then the logits [units, rows, keys] int32
    size_t all_rows() const { return way >= kParts ? (size_t)(units * tiles * tile_rows) : 0; }
    size_t logits() const { return way == kPartsFew ? (size_t)(units * rows * keys) : 0; }
    size_t bytes() const { return all_rows() * (12 + 4 * splits) + logits() * 4; }
};

// What a kernel is told of it.
struct Shape {
    int32_t splits, tiles, rows;
    int64_t keys;               // row stride of the stored logits
    uint64_t* row_sum;          // [units, tiles, rows of a tile]
    int32_t* row_max;           // likewise
    int32_t* part_max;          // [units, tiles, rows of a tile, splits]
    int32_t* logits;            // [units, rows, keys]
    int32_t shift, buckets;     // of the thresholds' buckets
};

inline Plan plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t L, int64_t max_keys) {
    Plan p{};
    p.units = (int64_t)B * Hkv;
    p.rows = L * (Hq / Hkv);
    p.keys = (max_keys + kTile - 1) / kTile * kTile;
    p.splits = 1;
    p.tile_rows = p.rows <= 16 ? 16 : 64;
    p.tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
    const int64_t groups = p.units * p.tiles;
    // One launch of a workgroup a unit takes 4 us and 2 more for every 512 keys, three launches
    // 18 to some thousands of keys: of few units, 1024, 2048 and 4096 keys 12, 16 and 24 us to 18.
    // With workgroups for half the compute units it is one launch as far as LDS goes: 4096 keys of
    // 128 units of a row 22 us to 28, of 256 of a row 27 to 37, of 256 of 4 rows 29 to 46.
    if (p.rows <= 16 && p.rows * p.keys <= kLdsLogits && (p.keys <= 2048 || p.units >= 128)) {
        p.way = kOneFew;
        return p;
    }
    const bool few = p.rows <= 16 && p.units * p.rows * p.keys <= kMostLogits;
    if (!few) p.tile_rows = 64;         // (one tile of at most 16 rows stays one)
    // Parts until every compute unit has a workgroup (two, of chunks): of a stage of few rows
    // (512 keys), of two tiles where they come one by one (24 workgroups of 64 rows over 1001 keys:
    // 30.7 us, 31.5 with four tiles).  Twice the parts of few rows cost more than they hide (each
    // adds to the results: 131072 keys, 58 us for 49).
    int64_t want = (few ? 256 : 512) / (groups > 0 ? groups : 1);
    const int64_t most = p.keys / (few ? 512 : 128);
    if (want > most) want = most;
    if (want > 256) want = 256;
    if (want > 1) p.splits = (int32_t)want;
    // three launches cost what four tiles in a row do: chunks of few keys stay in one
    if (!few && p.keys < 1024) p.splits = 1;
    p.way = few ? kPartsFew : (p.splits > 1 ? kParts : kOne);
    return p;
}

// The plan's arrays in a workspace of its bytes(); the sums first, which need the largest
// alignment.
inline Shape shape(const Plan& p, void* workspace) {
    Shape sh{};
    sh.splits = p.splits;
    sh.tiles = p.tiles;
    sh.rows = p.rows;
    sh.keys = p.keys;
    sh.row_sum = static_cast<uint64_t*>(workspace);
    sh.row_max = reinterpret_cast<int32_t*>(sh.row_sum + p.all_rows());
    sh.part_max = sh.row_max + p.all_rows();
    sh.logits = sh.part_max + p.all_rows() * p.splits;
    return sh;
}

}  // namespace paged
}  // namespace fqvit
