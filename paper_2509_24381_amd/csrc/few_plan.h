// Host side of attend_few_kernel's launches: how many parts the requests' key ranges become, and whose wavefronts share tiles, so that all sums have
// room in the workspace's slots.  No device code (a test compiles this file on its own).
#pragma once
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <vector>

constexpr int FEW_WAVES = 4;
constexpr int FEW_MAX_PARTS = 64;
constexpr int FEW_GROUP = 64;          // stacked rows of an item
constexpr int NOBODY = 0xffff, SEVERAL = 0xfffe;   // (FewShared::with)
// Blocks of 16 rows that `rows` of them are handled as: 1, 2 or 4.
constexpr int few_row_blocks(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

struct FewRequest {
    int kv, row0, T;       // index into kvs, first row, rows
    int units, tiles;      // items per part, tiles
    int row_blocks;        // of 16 rows: 1, 2 or 4
    int parts;
    bool once = false;     // its tiles are read once
    double weight = 1.0;   // of a tile
    int tile0 = 0;         // first of its tiles
    int with = NOBODY;     // (FewShared)
    int together = 0;      // (FewShared)
    bool in_slots() const { return parts > 1 || with != NOBODY; }
    double work() const { return tiles * weight; }
    int parts_of(int len) const { return std::min((int)std::ceil(work() / len), FEW_MAX_PARTS); }
};

// Slots, of 16 rows each, that the sums of requests on shared pages take if nothing is cut.
inline size_t fewest_slots(const std::vector<FewRequest>& reqs) {
    size_t n = 0;
    for (const FewRequest& r : reqs)
        if (r.with != NOBODY) n += (size_t)r.units * r.row_blocks;
    return n;
}

// Wavefronts of a workgroup share tiles (attend_shared.h) where a request has more than 32 stacked rows, and where it has more than 16 if the call's requests of
// that kind have this many tiles, times KV heads.  us a pass, wavefronts apart / together, (g) 28 query and 4 KV heads, (h) 64 and 8: (g) 4 beams each, 1 on 8000 (500) 15.7 / 16.6, 4 on 2000 (300)
// 13.0 / 13.8, 1 on 32000 (2000) 22.9 / 25.8, 16 on 8000 (4520) 51.4 / 43.5, 8 bits 34.7 / 32.7; 8 beams, 8 on 8000 (2130) 37.7 / 32.0.
constexpr long TOGETHER_TILES = 3000;
// That takes more slots: 17 to 32 rows are two blocks of 16 apart and eight together, more rows up to twice as many.  So those of up to 32 rows are only
// together if all sums have room then (51 prompts with 3 beams, (h): 4488 of 4096 slots together, 2040 apart; on 4000 209 us a pass apart, 331 with each request
// alone), and share_pages leaves twice the slots that are taken apart.  Sets units and row_blocks of those that are together; returns FewShared::together.
inline int share_tiles(std::vector<FewRequest>& reqs, int g, int hkv, long from, size_t slots) {
    long tiles = 0;
    for (const FewRequest& r : reqs)
        if (r.with == SEVERAL) tiles += (long)r.units * r.tiles;
    for (int above = tiles >= from ? 1 : 2; above <= 2; ++above) {
        int together = 0;
        for (const FewRequest& r : reqs)
            if (r.with == SEVERAL && r.row_blocks > above) together = std::max(together, (long)r.T * g > FEW_GROUP ? 2 : 1);
        if (together == 0) return 0;
        std::vector<FewRequest> now = reqs;
        for (FewRequest& r : now) {
            if (r.with != SEVERAL || r.row_blocks <= above) continue;
            r.together = together;
            r.units = (int)(((long)r.T * g + FEW_GROUP * together - 1) / (FEW_GROUP * together)) * hkv;
            r.row_blocks = 2 * FEW_GROUP / 16;   // (slots: of 128 rows, or of 64 twice)
        }
        if (fewest_slots(now) > slots && above < 2) continue;
        reqs.swap(now);
        return together;
    }
    return 0;
}

// Parts of the key ranges, of `len` tiles at most.  Estimated in tiles of a place (a workgroup's room on a compute unit) when all places stream:
// an item costs 1.5 beside its tiles, joining 2.  With no more items than places the longest ends last, but the fewer are left the
// faster they stream: a tile then takes 0.66 of one.  With more, the last ones start late: a share of the longest comes on top.  Where two or
// all four wavefronts need every tile it takes 2 and 3 times as long (wavefronts of 32 rows: 1.5 and 2), and parts are that much shorter (us a
// pass, all alike -> so: 30 single tokens on up to 8000 beside 4 requests of 5 on 3000, 64 query heads, 8 KV heads, 142.7 -> 115.5, 8 bits
// 91.3 -> 55.8; 24 requests of 3 on up to 6000 beside one of 12 on 5000 68.4 -> 53.4; one of 4 on 8000, alone, 15.8 -> 17.2).
// us a pass, parts of 4 / 8 / 16 / 24 / 48 tiles, and with this estimate's: 64 requests on up to 8000 tokens 97.4 / 93.2 / 86.0 / 86.6 / 89.0,
// 88.3; 16 on up to 32000, 8 bits, 73.2 / 68.6 / 66.1 / 64.6 / 59.4, 60.2; 24 of 3 tokens on up to 6000 and one of 12, 64 and 8 heads, 79.6 / 69.5 / 58.3 / 56.6 / 67.0, 54.3.
// False: however few the parts are, their sums do not fit the slots.
inline bool plan_few(std::vector<FewRequest>& reqs, int places, size_t slots) {
    double total = 0.0;
    int longest = 1;
    for (const FewRequest& r : reqs) {
        total += r.units * r.work();
        longest = std::max(longest, (int)std::ceil(r.work()));
    }
    double best = 1e30;
    int best_len = longest;
    for (int len = FEW_WAVES; ; len = std::min(longest, len + std::max(1, len / 8))) {
        long items = 0, split = 0;
        double most = 0.0;
        for (const FewRequest& r : reqs) {
            const int p = r.parts_of(len);
            items += (long)r.units * p;
            if (p > 1 || r.with != NOBODY) split += (long)r.units * p * r.row_blocks;
            most = std::max(most, (r.tiles + p - 1) / p * r.weight * 0.66);
        }
        const double share = total / places;
        const double cost = (items <= places ? std::max(share, most) + 1.5 : share + 1.5 * items / places + 0.5 * most) + (split ? 2.0 : 0.0);
        if ((size_t)split <= slots && cost < best) {
            best = cost;
            best_len = len;
        }
        if (len >= longest) break;
    }
    for (FewRequest& r : reqs) r.parts = r.parts_of(best_len);
    return best < 1e30;
}
