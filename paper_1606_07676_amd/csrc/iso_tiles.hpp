// Tiles of ranks for the matrix kernels of attention: which keys a tile of the torus needs, in which order, and which
// (rank, key) pairs of a tile are neighbours.  The neighbourhood is the same at every rank, so one table serves all tiles.
// Pure host code.
#pragma once

#include <algorithm>
#include <array>
#include <cmath>
#include <cstdint>
#include <unordered_map>
#include <vector>

#include "iso_plan.hpp"

namespace iso {

constexpr int kTileWaves = 4;              // wavefronts of a workgroup, 16 columns (rank, head) each
constexpr int kTileColumns = 16 * kTileWaves;
constexpr int kChunkRows = 64;             // rows (keys) that a workgroup holds in LDS at a time
constexpr int kTileMaxRows = 4096;         // rows of a tile

struct TilePlan {
    int heads = 1;                         // columns of one rank: column c is rank c / heads, head c % heads
    std::array<int32_t, ISO_MAX_DIMS> tile{}, tiles{};      // ranks per tile and tiles, by dimension
    int64_t n_tiles = 1;
    int rows = 0, chunks = 0;              // rows in use; chunks of kChunkRows
    // positions relative to the tile's first rank, the last dimension first, in words of four
    std::vector<int16_t> column_at;        // [kTileColumns / heads][words * 4]
    std::vector<int16_t> row_at;           // [chunks * kChunkRows][words * 4]
    std::vector<uint32_t> active;          // [chunks]: bit 4 * wave + group: that block holds a neighbour
    // The bias's gradient, for columns that are ranks.  A slot is (head of the column) * s + neighbour; its pairs among 32 rows and
    // the 16 columns of a wavefront, at most one a column, are places in what the wavefront's lanes wrote (slot_place).
    // [chunks * 2][kTileWaves][slot_rounds]: 64 slots, one a lane, then [slot_words][64][8] places as 16-bit numbers.  Lanes
    // without a slot name the one behind the last, and places without a pair the zero behind the last.
    int slot_rounds = 0, slot_words = 0;
    std::vector<uint32_t> slots;
    // [chunks * 2][kTileWaves][64][2][4]: of (lane's column, row 4 * (lane / 16) + r) of the 16 rows of either group of a pair, four
    // times (column's head) * (s + 1) + neighbour, with s for the neighbour where it is none
    std::vector<uint16_t> index;
};

// Lane (row % 16 / 4) * 16 + column writes four rows of either half at once.
inline uint32_t slot_place(int column, int row) { return (uint32_t)((row / 16 * 64 + row % 16 / 4 * 16 + column) * 4 + row % 4); }
constexpr uint32_t kSlotZero = 512;

struct TileShape {
    std::array<int32_t, ISO_MAX_DIMS> tile{}, wave{}, tiles{};
    int64_t n_tiles = 1;
};

// The tile: dimensions are doubled where that keeps the rows of all tiles together fewest; the ranks of a wavefront the same way.
// reach: highest less lowest step to a neighbour, by dimension.
inline TileShape tile_shape(const Comm &c, int ranks, int per_wave, const std::array<int64_t, ISO_MAX_DIMS> &reach) {
    TileShape s;
    const auto grow = [&](std::array<int32_t, ISO_MAX_DIMS> &t, int total, const std::array<int32_t, ISO_MAX_DIMS> *limit) {
        t.fill(1);
        for (int have = 1; have < total; have *= 2) {
            int best = -1;
            double best_cost = 0;
            for (int j = c.d - 1; j >= 0; --j) {
                if (limit && t[j] * 2 > (*limit)[j]) continue;
                const double n = c.dims[j], e = (double)reach[j], w = t[j];
                const auto cost = [&](double x) { return (limit ? n / x : std::ceil(n / x)) * (x + e); };
                const double gain = cost(2 * w) / cost(w);
                if (best < 0 || gain < best_cost) best = j, best_cost = gain;
            }
            t[best] *= 2;
        }
    };
    grow(s.tile, ranks, nullptr);
    grow(s.wave, per_wave, &s.tile);
    for (int j = 0; j < c.d; ++j) {
        s.tiles[j] = (c.dims[j] + s.tile[j] - 1) / s.tile[j];
        s.n_tiles *= s.tiles[j];
    }
    return s;
}

// Steps from a rank to its sources, signed, and how far they reach; what no rank of a mesh can have is left out.
struct Steps {
    std::vector<std::array<int32_t, ISO_MAX_DIMS>> step;
    std::vector<uint8_t> used;
    std::array<int32_t, ISO_MAX_DIMS> low{}, high{};
    std::array<int64_t, ISO_MAX_DIMS> reach{};
};
inline Steps source_steps(const Comm &c) {
    Steps s;
    s.step.resize((size_t)c.s);
    s.used.assign((size_t)c.s, 1);
    bool any = false;
    for (int i = 0; i < c.s; ++i) {
        s.step[i].fill(0);
        for (int j = 0; j < c.d; ++j) {
            const int64_t n = c.dims[j];
            int64_t x = c.c(i, j);
            if (c.periodic[j]) x = x > n / 2 ? x - n : x;
            else if (x >= n || x <= -n) s.used[i] = 0;
            s.step[i][j] = s.used[i] ? (int32_t)-x : 0;
        }
        if (!s.used[i]) continue;
        for (int j = 0; j < c.d; ++j) {
            s.low[j] = any ? std::min(s.low[j], s.step[i][j]) : s.step[i][j];
            s.high[j] = any ? std::max(s.high[j], s.step[i][j]) : s.step[i][j];
        }
        any = true;
    }
    for (int j = 0; j < c.d; ++j) s.reach[j] = (int64_t)s.high[j] - s.low[j];
    return s;
}
inline TileShape tile_shape(const Comm &c, int heads) { return tile_shape(c, kTileColumns / heads, 16 / heads, source_steps(c).reach); }

// The index holds byte offsets of biases in 16 bits.
inline bool tile_table_holds(int heads, int s) { return (int64_t)heads * (s + 1) * 4 <= 65535; }

// back = false: columns are ranks, rows their sources R (-) C^i.  back = true: columns are sources, rows the ranks that read
// them.  False where no table of that form exists (neighbours too many, or too far apart) or nothing would be in it (a mesh on
// which no neighbour has a source at any rank): a tile that the kernels are given has one chunk of rows or more.
//
// pays(rows, n_tiles) is asked before any table is made, with the fewest rows that there can be and then with those that there
// are: false ends it.
template <typename Pays>
inline bool build_tile_plan(const Comm &c, int heads, bool back, bool bias_slots, TilePlan &out, Pays &&pays) {
    const int d = c.d, ranks = kTileColumns / heads, per_wave = 16 / heads;
    if (c.s < 1 || !tile_table_holds(heads, c.s)) return false;
    Steps steps = source_steps(c);
    if (back)                              // from a source to its readers
        for (int i = 0; i < c.s; ++i)
            for (int j = 0; j < d; ++j) steps.step[i][j] = -steps.step[i][j];
    std::array<int32_t, ISO_MAX_DIMS> low = steps.low, high = steps.high;
    for (int j = 0; back && j < d; ++j) low[j] = -steps.high[j], high[j] = -steps.low[j];
    const auto &step = steps.step;
    const auto &used = steps.used;
    TilePlan p;
    p.heads = heads;
    const TileShape shape = tile_shape(c, ranks, per_wave, steps.reach);
    const auto &wave = shape.wave;
    p.tile = shape.tile;
    p.tiles = shape.tiles;
    p.n_tiles = shape.n_tiles;
    if (p.n_tiles > 0x7FFFFFFF) return false;
    // sums of a of one kind and b of another are a + b - 1 or more
    std::vector<std::array<int32_t, ISO_MAX_DIMS>> distinct;
    for (int i = 0; i < c.s; ++i)
        if (used[i]) distinct.push_back(step[i]);
    std::sort(distinct.begin(), distinct.end());
    const int steps_apart = (int)(std::unique(distinct.begin(), distinct.end()) - distinct.begin());
    const int fewest = steps_apart + ranks - 1;
    if (!steps_apart || fewest > kTileMaxRows || !pays(fewest, p.n_tiles)) return false;
    // columns: the wavefronts' boxes one after the other, the last dimension fastest inside and outside
    const int width = (d + 3) / 4 * 4;
    std::vector<int32_t> column_at((size_t)ranks * d);
    p.column_at.assign((size_t)ranks * width, 0);
    for (int r = 0; r < ranks; ++r) {
        int inside = r % per_wave, box = r / per_wave;
        for (int j = d - 1; j >= 0; --j) {
            const int boxes = p.tile[j] / wave[j];
            column_at[(size_t)r * d + j] = box % boxes * wave[j] + inside % wave[j];
            p.column_at[(size_t)r * width + d - 1 - j] = (int16_t)column_at[(size_t)r * d + j];
            inside /= wave[j];
            box /= boxes;
        }
    }
    // rows by position: a number in the box that all positions span
    std::array<int64_t, ISO_MAX_DIMS> span{};
    int64_t volume = 1;
    for (int j = 0; j < d; ++j) {
        if (c.dims[j] > 1 << 30) return false;                      // a tile's place and a position add up in 32 bits
        span[j] = (int64_t)high[j] - low[j] + p.tile[j];
        if (low[j] < -32768 || (int64_t)high[j] + p.tile[j] > 32768 || span[j] > (int64_t(1) << 40) / volume) return false;
        volume *= span[j];
    }
    struct Row {
        std::array<int32_t, ISO_MAX_DIMS> at;
        int copy;                          // a pair that is listed twice finds its second neighbour in a second row
    };
    std::vector<Row> rows;
    std::unordered_map<int64_t, std::vector<int>> by_place;
    std::unordered_map<int64_t, int> taken;                 // rank and row -> neighbour
    for (int r = 0; r < ranks; ++r)
        for (int i = 0; i < c.s; ++i) {
            if (!used[i]) continue;
            Row row;
            row.at.fill(0);
            int64_t place = 0;
            for (int j = 0; j < d; ++j) {
                row.at[j] = column_at[(size_t)r * d + j] + step[i][j];
                place = place * span[j] + (row.at[j] - low[j]);
            }
            std::vector<int> &copies = by_place[place];
            row.copy = 0;
            while ((size_t)row.copy < copies.size() && taken.count((int64_t)r << 32 | copies[row.copy])) ++row.copy;
            if ((size_t)row.copy == copies.size()) {
                if (rows.size() == (size_t)kTileMaxRows) return false;
                copies.push_back((int)rows.size());
                rows.push_back(row);
            }
            taken[(int64_t)r << 32 | copies[row.copy]] = i;
        }
    if (!pays((int)rows.size(), p.n_tiles)) return false;
    // Order: boxes of a wavefront's shape, so that the groups of 16 rows that a wavefront has no neighbour in are many.  Where
    // neighbours are few and far apart, so that few rows serve more than one column, the rows of one wavefront after those of
    // the other (as they were found) leave fewer blocks.
    std::vector<int> order(rows.size()), found(rows.size());
    for (size_t u = 0; u < order.size(); ++u) order[u] = found[u] = (int)u;
    const auto blocks_of = [&](const std::vector<int> &o) {
        std::vector<int> place(o.size());
        for (size_t u = 0; u < o.size(); ++u) place[o[u]] = (int)u;
        std::vector<uint8_t> hit((o.size() + 15) / 16 * kTileWaves, 0);
        for (const auto &[pair, i] : taken) hit[place[(size_t)(pair & 0xFFFFFFFF)] / 16 * kTileWaves + (int)(pair >> 32) / per_wave] = 1;
        return std::count(hit.begin(), hit.end(), 1);
    };
    std::sort(order.begin(), order.end(), [&](int a, int b) {
        for (int pass = 0; pass < 2; ++pass)
            for (int j = 0; j < d; ++j) {
                const int x = rows[a].at[j] - low[j], y = rows[b].at[j] - low[j];
                const int u = pass ? x % wave[j] : x / wave[j], v = pass ? y % wave[j] : y / wave[j];
                if (u != v) return u < v;
            }
        return rows[a].copy < rows[b].copy;
    });
    if (blocks_of(found) < blocks_of(order)) order = found;
    p.rows = (int)rows.size();
    p.chunks = (p.rows + kChunkRows - 1) / kChunkRows;
    p.row_at.assign((size_t)p.chunks * kChunkRows * width, 0);
    p.active.assign((size_t)p.chunks, 0);
    p.index.resize((size_t)p.chunks * 4 * kTileWaves * 64 * 4);
    for (size_t i = 0; i < p.index.size(); ++i) p.index[i] = (uint16_t)(4 * ((int)(i / 8 % 16) % heads * (c.s + 1) + c.s));
    std::vector<int> rank_of((size_t)p.rows);
    for (int u = 0; u < p.rows; ++u) {
        rank_of[order[u]] = u;
        for (int j = 0; j < d; ++j) p.row_at[(size_t)u * width + d - 1 - j] = (int16_t)rows[order[u]].at[j];
    }
    for (const auto &[pair, i] : taken) {
        const int r = (int)(pair >> 32), u = rank_of[(size_t)(pair & 0xFFFFFFFF)];
        const int group = u / 16, lane_row = u % 16;
        for (int h = 0; h < heads; ++h) {
            const int column = r * heads + h, w = column / 16;
            const int lane = lane_row / 4 * 16 + column % 16;
            p.index[(((size_t)(group / 2) * kTileWaves + w) * 64 + lane) * 8 + group % 2 * 4 + lane_row % 4] = (uint16_t)(4 * (h * (c.s + 1) + i));
            p.active[group / 4] |= 1u << (4 * w + group % 4);
        }
    }
    if (bias_slots) {
        std::vector<std::vector<std::pair<uint32_t, uint32_t>>> of((size_t)p.chunks * 2 * kTileWaves);
        for (const auto &[pair, i] : taken) {
            const int r = (int)(pair >> 32), u = rank_of[(size_t)(pair & 0xFFFFFFFF)];
            for (int h = 0; h < heads; ++h) {
                const int column = r * heads + h;
                of[(size_t)(u / 32) * kTileWaves + column / 16].push_back({(uint32_t)(h * c.s + i), slot_place(column % 16, u % 32)});
            }
        }
        size_t most = 1;
        for (auto &list : of) {
            std::sort(list.begin(), list.end());
            size_t n = 0;
            for (size_t k = 0; k < list.size(); ++k) n += !k || list[k].first != list[k - 1].first;
            most = std::max(most, n);
        }
        p.slot_rounds = (int)((most + 63) / 64);
        p.slot_words = 16 / heads > 8 ? 2 : 1;
        const size_t round = 64 + 256 * (size_t)p.slot_words;
        p.slots.assign(of.size() * p.slot_rounds * round, kSlotZero | kSlotZero << 16);
        for (size_t l = 0; l < of.size(); ++l) {
            uint32_t *at = p.slots.data() + l * p.slot_rounds * round;
            for (int n = 0; n < p.slot_rounds; ++n) std::fill_n(at + n * round, 64, (uint32_t)(heads * c.s));
            int lane = -1, count = 0;
            for (size_t k = 0; k < of[l].size(); ++k) {
                const auto &[slot, place] = of[l][k];
                if (!k || slot != of[l][k - 1].first) ++lane, count = 0;
                uint32_t *mine = at + lane / 64 * round;
                mine[lane % 64] = slot;
                uint32_t &word = mine[64 + count / 8 * 256 + lane % 64 * 4 + count % 8 / 2];
                word = count % 2 ? (word & 0xFFFF) | place << 16 : (word & 0xFFFF0000) | place;
                ++count;
            }
        }
    }
    out = std::move(p);
    return true;
}

}  // namespace iso
