// scd_plan.h -- sizes and shares of the operators of learned features.  Arithmetic alone: the kernels and their host
// code use it, and it compiles for a host without HIP.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace scd {
namespace feat {

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// log2 of the smallest power of two that is at least n.
constexpr uint32_t log2_up(uint64_t n) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < n) ++l;
    return l;
}

// A launch has fewer than 2^32 threads along each of its axes; longer work goes in several launches.
constexpr int64_t kMaxThreads = 0xFFFFFFFFLL;

constexpr int kThreads = 256;  // of a workgroup of the lookup, and of the sums of narrow rows

// A row is `lanes` consecutive threads (a power of two, at most 256) with VEC elements each, and as many
// such column ranges (blockIdx.y) as it needs.  Rows narrower than 16 bytes go element by element (VEC = 1).
struct RowMap {
    uint32_t log2_lanes;
    uint32_t ranges;
};

inline RowMap row_map(int64_t dim, int vec) {
    RowMap m;
    m.log2_lanes = std::min<uint32_t>(8, log2_up((uint64_t)ceil_div(dim, vec)));
    m.ranges = (uint32_t)ceil_div(dim, (int64_t)vec << m.log2_lanes);
    return m;
}

// The lookup's rows in flight per thread: four once that still leaves eight workgroups to each CU.
inline int embed_unroll(int64_t n, const RowMap& m) {
    return ceil_div(n, (kThreads >> m.log2_lanes) * 4) * m.ranges >= 2048 ? 4 : 1;
}

// Tokens of one launch of the lookup at most, in which a workgroup takes `unroll` tokens for each of its groups of lanes.
inline int64_t embed_tokens(const RowMap& m, int unroll) { return kMaxThreads / kThreads * ((kThreads >> m.log2_lanes) * unroll); }

// ---------------------------------------------------------------------------------------- lookup gradient

constexpr int kFewMax = 1024;      // tokens that one launch does
constexpr int kBatch = 8;          // entries that a group of lanes sums at a time
constexpr int kPairBytes = 8;      // of an entry of a sorted list
constexpr int kSmallTile = 256;    // entries of a tile of the short lists' sort
constexpr int kTileThreads = 512;  // of a workgroup of the radix sort
constexpr int kMaxBits = 11;       // of a digit

// The bytes that workgroup `block` of `blocks` fills of `total` consecutive ones: a run of whole 64-byte lines, as long
// for each but the last of those that have any.
struct Piece {
    int64_t from, bytes;
};
constexpr Piece fill_piece(int64_t total, int64_t block, int64_t blocks) {
    const int64_t share = ceil_div(ceil_div(total, blocks), 64) * 64;
    const int64_t from = block * share < total ? block * share : total;
    return Piece{from, share < total - from ? share : total - from};
}

// Threads of a workgroup of the sums (k_sums): wide rows get workgroups of several groups of lanes all the same.
constexpr int kWideSums = 512;
inline int sums_threads(const RowMap& m) { return m.log2_lanes >= 6 ? kWideSums : kThreads; }

// Workgroups of the sums of n entries, of which each group of lanes takes `share`.
inline int64_t sums_blocks(int64_t n, uint32_t share, const RowMap& m) { return ceil_div(n, (int64_t)share * (sums_threads(m) >> m.log2_lanes)); }

// How a gradient call sorts and splits: a function of the sizes alone.
struct Plan {
    bool few;         // no sorted list: nothing below is used
    int64_t n;        // padded to whole batches
    bool tiled;       // a short list
    int passes, bits;
    int per_thread;
    int64_t tiles;
    uint32_t share;
    int64_t pairs;    // bytes of one list
    int64_t hist, pieces, bytes;
};

// Lists of up to this many entries are sorted by tiles, or up to twice as many where the radix sort takes several passes.
// Whole calls: 16,384 tokens into 1,000 x 256 (one pass) 28 us by tiles and 35 by radix, 30,000 46 and 38;
// 30,000 into 300,000 x 64 (two passes) 47 and 58, 16,384 into 75,000 x 1,024 46 and 71.
constexpr int64_t kTiledMax = 16384;

constexpr int64_t align16(int64_t b) { return (b + 15) / 16 * 16; }

inline Plan plan_for(int64_t n, int64_t rows, int64_t dim) {
    Plan p{};
    p.few = n <= kFewMax;
    if (p.few) return p;
    p.n = ceil_div(n, kBatch) * kBatch;
    const int key_bits = std::max(1, (int)log2_up((uint64_t)rows + 1));
    // As few passes as digits of at most 11 bits take, which share the key's bits evenly: the more digits, the shorter the
    // runs that a tile writes.
    p.passes = (int)ceil_div(key_bits, kMaxBits);
    p.tiled = p.n <= kTiledMax * (p.passes > 1 ? 2 : 1);
    p.bits = (int)ceil_div(key_bits, p.passes);
    // Entries of a tile's thread: enough tiles for the CUs while the list is short, few counts of digits where it is long.
    // Whole calls with 2, 4 and 8: 131,072 into 50,000 x 512 74, 77 and 84 us; 300,000 into 1.5 M x 32 78, 76 and 84;
    // 600,000 into 1.5 M x 16 96, 89 and 90; 1.28 M into 1.5 M x 16 (4 and 8) 135 and 120.
    p.per_thread = p.n <= 200'000 ? 2 : p.n <= 800'000 ? 4 : 8;
    p.tiles = ceil_div(p.n, kTileThreads * p.per_thread);
    // Entries per group: as many as keep about 4,096 waves in work, 8 at least, 64 at most.
    const int64_t work = p.n * ceil_div(dim, 4) / 64;
    p.share = (uint32_t)std::min<int64_t>(64, std::max<int64_t>(8, work / 4096 / 8 * 8));
    // A share has at most 256 threads (and the last workgroup may have one group without): the longest lists take larger
    // ones, so that they fit a launch.
    while (ceil_div(p.n, p.share) >= kMaxThreads / kThreads) p.share *= 2;
    p.pairs = align16(p.n * kPairBytes);
    // The tiles' keys, or the counts of digits and their totals.
    p.hist = p.tiled ? ceil_div(p.n, kSmallTile) * kSmallTile * 4 : align16(((p.tiles + 1) << p.bits) * 4);
    // The pieces of runs: a row for each workgroup of the sums, as many as there are with vectors of 1, 4 or 8 elements.
    int64_t blocks = dim < 8 ? sums_blocks(p.n, p.share, row_map(dim, 1)) : 0;
    for (int vec = 4; vec <= 8; vec += 4)
        if (dim >= vec) blocks = std::max(blocks, sums_blocks(p.n, p.share, row_map(dim, vec)));
    p.pieces = align16(blocks * dim * 4);
    p.bytes = 2 * p.pairs + p.hist + 2 * p.pieces;
    return p;
}

}  // namespace feat
}  // namespace scd
