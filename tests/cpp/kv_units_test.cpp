// What the plans of attention over shared pages make of batches, against what the host reserves for them: items (which size
// the grids), partial results (which size the workspace) and sums that small batches take in 32 bits.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2608_23805_amd/csrc/kv_units.h"

using namespace msi;

static int failures = 0;
#define CHECK(c)                                                     \
    do {                                                             \
        if (!(c)) {                                                  \
            std::printf("line %d: %s\n", __LINE__, #c);              \
            ++failures;                                              \
        }                                                            \
    } while (0)

struct Owner {
    int n, blocks;                    // rows, blocks
};

struct Made {
    int64_t work = 0, items = 0, parts = 0;
};

// Items and rows of partial results of owners in units of `chunk` blocks.
static Made cut_in(const std::vector<Owner> &owners, int G, int H, int tile_rows, int chunk)
{
    Made m;
    for (const Owner &o : owners) {
        const int64_t tiles = tiles_of(o.n, G, tile_rows), units = o.n ? (o.blocks + chunk - 1) / chunk : 0;
        m.work += o.blocks * tiles * H;
        m.items += units * tiles;
        m.parts += units * o.n * G * H;
    }
    return m;
}

int main()
{
    // chunks: never under the least, whatever a sum of a batch that breaks its bounds has become
    for (const int64_t work : {int64_t(0), int64_t(1), int64_t(-1), -(int64_t(1) << 31), int64_t(1) << 40}) {
        CHECK(unit_chunk(work) >= LEAST_BLOCKS);
        for (const int most : {1024, 2048})
            CHECK(shared_chunk(work, false, most) >= LEAST_MANY && shared_chunk(work, true, most) >= LEAST_BLOCKS);
    }
    CHECK(unit_chunk(4 * 256) == 4 && unit_chunk(16 * 256) == 16 && unit_chunk(16 * 256 + 1) == 16 && unit_chunk(17 * 2048) == 17);
    CHECK(tiles_of(0, 7, 16) == 0 && tiles_of(5, 13, 32) == 3 && tiles_of(1 << 29, 1, 128) == 1 << 22);

    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return int(std::uniform_int_distribution<int>(lo, hi)(rng)); };
    auto any_of = [&](std::initializer_list<int> v) { return v.begin()[pick(0, int(v.size()) - 1)]; };
    int small = 0, both = 0, many = 0;
    for (int round = 0; round < 20000; ++round) {
        const int S = any_of({1, 2, 7, 63, 64, 65, 200}), H = any_of({1, 2, 3, 8, 128, 256}), G = any_of({1, 4, 7, 8, 13}), D = any_of({64, 128, 256});
        const int most_rows = any_of({1, 1, 2, 5, 13, 70, 300}), most_own = any_of({1, 2, 9, 40, 900}), most_shared = any_of({0, 1, 9, 30, 2000});
        std::vector<Owner> seqs(S), groups;
        int n_rows = 0, max_rows = 0, own = 1;
        for (Owner &o : seqs) {
            o = Owner{pick(0, most_rows), pick(1, most_own)};
            n_rows += o.n, max_rows = std::max(max_rows, o.n), own = std::max(own, o.blocks);
        }
        if (!n_rows)
            continue;
        int group_rows = 0, blocks = 0;
        const int length = any_of({1, 3, 64, 1000});
        std::vector<Owner> rest;                             // the sequences' other pages
        for (int a = 0; a < S;) {
            const int z = std::min(S, a + pick(0, length));
            Owner g{0, pick(0, most_shared)};
            for (int i = a; i < z; ++i)
                g.n += seqs[i].n;
            groups.push_back(g);
            group_rows = std::max(group_rows, g.n), blocks = std::max(blocks, g.blocks);
            if (z == a && pick(0, 3) == 0)                   // (a sequence of no group: all of its pages are its own)
                rest.push_back(Owner{seqs[a].n, seqs[a].blocks + pick(0, most_shared)}), ++a;
            for (; a < z; ++a)
                rest.push_back(pick(0, 5) ? seqs[a] : Owner{seqs[a].n, seqs[a].blocks + g.blocks});   // (some by themselves)
        }
        for (const Owner &o : rest)
            own = std::max(own, o.blocks);
        // the host's bounds: as tight as they may be, or loose
        const int loose = pick(0, 1) * pick(0, 100);
        KvSeqs s{nullptr, nullptr, nullptr, S, 1 << 20, n_rows, max_rows + loose % 3, 0, false};
        s.max_rows = std::min(s.max_rows, n_rows);
        s.max_len = 64 * std::max(own, blocks + 1) - pick(0, 63) + 64 * loose;
        KvGroups g{nullptr, nullptr, int(groups.size()), std::min(group_rows + loose, n_rows), blocks + loose, 0};
        g.usable = std::min(g.max_blocks, s.max_len / KV_BLOCK);
        const SharedCut c = shared_cut(s, g, H, G, D);
        if (c.both)
            CHECK(c.tile_p == c.tile_s);
        Made p = cut_in(groups, G, H, c.tile_p, 1), q = cut_in(rest, G, H, c.tile_s, 1);
        const int64_t work_p = c.both ? p.work + q.work : p.work, work_s = c.both ? p.work + q.work : q.work;
        int chunk_p = shared_chunk(work_p, c.few_p, c.most_p), chunk_s = shared_chunk(work_s, c.few_s, c.most_s);
        if (!c.few_p)
            chunk_p += pick(0, 1) * pick(0, 300);            // (what the balancing makes of it)
        if (!c.few_s)
            chunk_s += pick(0, 1) * pick(0, 300);
        p = cut_in(groups, G, H, c.tile_p, chunk_p), q = cut_in(rest, G, H, c.tile_s, chunk_s);
        CHECK(p.items <= c.items_p && q.items <= c.items_s);
        CHECK(p.parts + q.parts <= c.parts);
        CHECK(c.bytes >= size_t(c.parts) * 4 * (D + 2) + (groups.size() + S) * (sizeof(KvOwner) + 4));
        CHECK(c.first % 256 == 0 && c.part_ml % 256 == 0 && c.part_o % 256 == 0);
        if (c.small) {
            CHECK(S <= 64 && groups.size() <= 64 && p.work + q.work < int64_t(1) << 30 && c.parts < int64_t(1) << 23);
            CHECK(64 * (int64_t(c.items_p) + c.items_s + 1) < int64_t(1) << 31);
        }
        small += c.small, both += c.both, many += !c.few_s;
        if (failures)
            return 1;
        // blocks that no rows can stand behind take nothing
        g.usable = 0;
        CHECK(shared_cut(s, g, H, G, D).items_p == 0);
    }
    CHECK(small > 1000 && both > 1000 && many > 1000);
    if (!failures)
        std::puts("ok");
    return failures != 0;
}
