// kv_units.h -- how attention over the cache is cut into units of work: the
// rules that the host's bounds and the kernels' plans have in common.  Plain C++
// apart from the qualifiers, so that they are tested against each other on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "kv_common.h"

namespace msi {

// Blocks of a unit for `work` blocks in all (times heads and row tiles): one
// workgroup per CU as long as each has at most 16 blocks, four a wavefront;
// then units of 16, which hide their start and their partial results' way
// through memory, until there are 2048 of them (131072 tokens of one sequence, 2 heads
// of 256: 36 us with 16 blocks, 46 with 4; 48 sequences of up to 16384, 8 heads of 128:
// 246, 233, 223 and 219 us with 256, 512, 1024 and 2048 workgroups).
// Sequences of up to 8 blocks are not cut (4 to 16 sequences of 500 tokens: 9.3 and 10.1 us,
// 11.6 and 13.5 cut; of 1000 tokens with heads of 256 17.0, 14.1 cut).
constexpr int DIRECT_BLOCKS = 8, LEAST_BLOCKS = 4, ENOUGH_BLOCKS = 16, FILL_WORKGROUPS = 256, MOST_WORKGROUPS = 2048;

MSI_HD int unit_chunk(int64_t work)
{
    const int64_t fill = (work + FILL_WORKGROUPS - 1) / FILL_WORKGROUPS;
    if (fill <= ENOUGH_BLOCKS)
        return fill < LEAST_BLOCKS ? LEAST_BLOCKS : int(fill);
    const int64_t most = (work + MOST_WORKGROUPS - 1) / MOST_WORKGROUPS;
    return most < ENOUGH_BLOCKS ? ENOUGH_BLOCKS : int(most);
}

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// ---------------------------------------------------------------- shared pages

struct KvGroups {
    const int32_t *cu;           // [n + 1] first sequence of every group
    const int32_t *blocks;       // [n] shared blocks
    int n, max_rows, max_blocks;
    int usable;                  // blocks that rows can stand behind (max_len / 64): groups with more serve nobody
};
// What units are cut from: the shared pages of a group with the rows of its sequences, or the other pages of a sequence
// with its rows.
struct alignas(16) KvOwner {
    int row0, n, len, seq;       // rows, tokens up to the last of these pages, sequence whose table is read
    int b0, blocks;              // pages
    int units, tiles;            // row tiles of a unit
    int64_t part;                // first partial result; a unit's are [H, n * G]
    int group;                   // of a sequence: its group, -1 if it shares nothing
    int all;                     // every row sees every token
};
struct SharedCut {
    bool few_p, few_s;           // form of the shared pages' units, of the sequences'
    bool both;                   // one launch for both
    int tile_p, tile_s;          // packed rows of a workgroup
    int items_p, items_s;        // bounds of units times row tiles
    int most_p, most_s;          // workgroups that units are cut for, at most
    bool small;                  // every wavefront lays out the units by itself
    int64_t parts;               // bound of the partial results (rows)
    size_t first, part_ml, part_o, bytes;   // workspace offsets and size (the owners come first)
};

constexpr int LEAST_MANY = 8;                // blocks of a 128-row unit: below, its partial results outweigh the codes
constexpr int SMALL_OWNERS = 64;
constexpr int64_t SMALL_PARTS = 1 << 23;     // sums over the lanes stay in 32 bits

MSI_HD int log2_of(int power) { return __builtin_ctz(unsigned(power)); }

// Row tiles of n rows (n G <= 2^29), tiles being powers of two.
MSI_HD int tiles_of(int n, int G, int tile_rows)
{
    return int((unsigned(n) * unsigned(G) + unsigned(tile_rows - 1)) >> log2_of(tile_rows));
}

// Blocks of a unit of shared pages' calls: a least one, from which `balanced_chunk` goes up.
MSI_HD int shared_chunk(int64_t work, bool few, int most)
{
    if (few)
        return unit_chunk(work);
    const int64_t least = (work + most - 1) >> log2_of(most);
    return least < LEAST_MANY ? LEAST_MANY : int(least);
}

// How a call with shared pages is cut, by its host-side bounds alone.  Units are cut on the device so that at most `most`
// workgroups (times heads and row tiles) come of them, besides one for every owner's row tile; that bounds the items and
// the rows of partial results.
inline SharedCut shared_cut(const KvSeqs &s, const KvGroups &g, int H, int G, int D)
{
    SharedCut c{};
    // Up to three tiles of 32 rows read the pages as often, mostly from L2, in less time than a tile of 128 rows takes, which
    // converts and multiplies for all of them (tokens of its own, 12 rows of 8 heads behind 200 shared blocks: heads of 64,
    // 128, 256 42, 52, 59 us by 128 rows, 38, 47, 49; shared blocks, 72 rows: 26, 30, 42 and 28, 32, 31).
    auto tile = [](int64_t rows, int most) { return rows <= 16 ? 16 : rows <= most ? 32 : 128; };
    c.tile_p = tile(int64_t(g.max_rows) * G, D == 256 ? 96 : 64);
    c.tile_s = tile(int64_t(s.max_rows) * G, 96);
    c.few_p = c.tile_p != 128;
    c.few_s = c.tile_s != 128;
    c.both = c.few_p && c.few_s;
    if (c.both)
        c.tile_p = c.tile_s = std::max(c.tile_p, c.tile_s);
    const int rounds = 4 * (D == 256 ? 256 : 512);          // four times the 128-row workgroups that the card holds at once
    c.most_p = c.few_p ? MOST_WORKGROUPS : rounds;
    c.most_s = c.few_s ? MOST_WORKGROUPS : rounds;
    const int64_t packed = int64_t(s.n_rows) * G;
    auto bound = [&](int64_t owners, int64_t blocks, int tile_rows, int most, bool few, int64_t &parts) {
        const int64_t tiles = packed / tile_rows + owners, least = few ? LEAST_BLOCKS : LEAST_MANY,
                      units = (blocks + least - 1) / least;
        const int64_t items = std::min(most / H + tiles, units * tiles);
        parts += std::min(units * packed, items * tile_rows) * H;
        return int(std::min<int64_t>(items, 0x7fffffff));
    };
    const bool any = g.n && g.max_rows && g.usable;
    c.items_p = any ? bound(g.n, g.usable, c.tile_p, c.most_p, c.few_p, c.parts) : 0;
    c.items_s = bound(s.S, (s.max_len + KV_BLOCK - 1) / KV_BLOCK, c.tile_s, c.most_s, c.few_s, c.parts);
    auto work = [&](int64_t owners, int64_t blocks, int tile_rows) { return (packed / tile_rows + owners) * blocks * H; };
    c.small = g.n <= SMALL_OWNERS && s.S <= SMALL_OWNERS && c.parts < SMALL_PARTS && int64_t(c.items_p) + c.items_s < SMALL_PARTS &&
              work(g.n, g.usable, c.tile_p) + work(s.S, (s.max_len + KV_BLOCK - 1) / KV_BLOCK, c.tile_s) < int64_t(1) << 30;
    size_t off = up256(size_t(g.n + s.S) * sizeof(KvOwner));
    c.first = off;
    off += up256(size_t(g.n + s.S + 1) * sizeof(int32_t));
    c.part_ml = off;
    off += up256(size_t(c.parts) * 2 * sizeof(float));
    c.part_o = off;
    off += up256(size_t(c.parts) * D * sizeof(float));
    c.bytes = off;
    return c;
}

}  // namespace msi
