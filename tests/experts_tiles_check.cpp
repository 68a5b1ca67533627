// Experts' rows in tiles (sparq_mx_tiles.h), on the host: 64 lanes, or a table's workgroup, as threads, against plain counting in 64 bits.
//   experts_tiles_check ROWS TILE offset...            up to 64 experts: by lanes, and by a table; more: by a table
// Prints "ok <tiles>" or what differs.  Offsets that fall: nothing outside of the table is written and no tile leaves the rows.
#define __shared__
#include <stdio.h>
#include <stdlib.h>

#include "../paper_2105_11010_amd/csrc/sparq_mx_tiles.h"

using namespace sparq::mx;

void gpu::load(const Buffer&, uint32_t, uint32_t, int) {}

int main(int argc, char** argv) {
    const int64_t rows = atoll(argv[1]);
    const int tile = atoi(argv[2]), experts = argc - 4;
    std::vector<int32_t> offsets;
    for (int i = 3; i < argc; ++i) offsets.push_back((int32_t)atoll(argv[i]));
    bool rising = true;
    for (int i = 0; i < experts; ++i) rising &= offsets[i] <= offsets[i + 1];
    const int64_t most = most_tiles(rows, experts, tile);
    // the tiles, as they should be
    struct Range {
        int64_t first, count, tiles_before;
    };
    std::vector<Range> ranges;
    int64_t total = 0;
    for (int e = 0; e < experts; ++e) {
        const auto cut = [&](int64_t v) { return v < 0 ? 0 : v > rows ? rows : v; };
        const int64_t a = cut(offsets[e]), b = cut(offsets[e + 1]), n = b > a ? b - a : 0;
        ranges.push_back({a, n, total});
        total += (n + tile - 1) / tile;
    }
    const auto is = [&](int64_t i, const ExpertTile& t) {
        int e = experts - 1;
        while (ranges[e].tiles_before > i || ranges[e].count == 0) --e;
        const int64_t in = (i - ranges[e].tiles_before) * tile, left = ranges[e].count - in;
        if (t.row == ranges[e].first + in && t.rows == (left < tile ? left : tile) && t.expert == e) return true;
        printf("tile %lld of %lld: row %d, rows %d, expert %d\n", (long long)i, (long long)total, t.row, t.rows, t.expert);
        return false;
    };
    bool ok = true;
    // Every tile of small calls, the first and last of each expert in any
    std::vector<int64_t> looked_at;
    for (int e = 0; e < experts; ++e) {
        const int64_t n = (ranges[e].count + tile - 1) / tile;
        for (int64_t i = 0; i < n; ++i)
            if (i < 5 || i >= n - 5) looked_at.push_back(ranges[e].tiles_before + i);
    }
    if (experts <= kExpertsOfLanes)
        gpu::run_workgroup(64, dim3(0), [&] {
            const LaneTiles t = tiles_of_lanes(offsets.data(), experts, rows, tile);
            const int64_t count = (uint32_t)tile_count(t);
            if (threadIdx.x == 0 && count != total) ok = false, printf("%lld tiles by lanes, not %lld\n", (long long)count, (long long)total);
            for (const int64_t i : looked_at) {
                const ExpertTile of = expert_tile(t, tile, (uint32_t)i);
                if (threadIdx.x == 0) ok = is(i, of) && ok;
            }
        });
    constexpr int kGuard = 1 << 16;              // entries before and behind the table
    std::vector<ExpertTile> memory(most + 1 + 2 * kGuard, ExpertTile{7, 7, 7, 7});
    ExpertTile* const table = memory.data() + kGuard;
    int64_t sums[kTableThreads / 64];
    gpu::run_workgroup(kTableThreads, dim3(0), [&] { write_tiles(offsets.data(), experts, rows, tile, (int)most, table, sums); });
    const int64_t count = table[0].row;
    if (count != (total < most ? total : most)) ok = false, printf("%lld tiles in the table, not %lld, at most %lld\n", (long long)count, (long long)total, (long long)most);
    if (rising)
        for (const int64_t i : looked_at) ok = is(i, table[1 + i]) && ok;
    for (int64_t i = 0; i < count && i < most; ++i) {
        const ExpertTile& t = table[1 + i];
        if (t.row < 0 || t.rows < 1 || t.rows > tile || t.row + (int64_t)t.rows > rows || t.expert < 0 || t.expert >= experts) {
            ok = false;
            printf("tile %lld leaves the rows: row %d, rows %d, expert %d\n", (long long)i, t.row, t.rows, t.expert);
            break;
        }
    }
    for (int64_t i = 0; i < kGuard; ++i)
        if (memory[i].unused != 7 || memory[memory.size() - 1 - i].unused != 7) return printf("written outside of the table\n"), 1;
    if (!ok) return 1;
    printf("ok %lld\n", (long long)total);
    return 0;
}
