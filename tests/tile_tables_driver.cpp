// The tables of attention's tile kernels against the neighbourhood itself, for random tori, meshes, offsets and heads: every
// pair of a column and one of its neighbours is in the index exactly once, at a row whose position is that neighbour's; the
// groups that hold one are the active ones; and the slots of the bias's gradient hold every pair once, at the place where its
// lane writes.  Positions are followed as the kernels do.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>

#include "iso_tiles.hpp"

using namespace iso;

#define CHECK(x)                                                                       \
    do {                                                                               \
        if (!(x)) {                                                                    \
            std::printf("%s:%d: %s does not hold (%s)\n", __FILE__, __LINE__, #x, what.c_str()); \
            std::exit(1);                                                              \
        }                                                                              \
    } while (0)

static std::string what;

// The rank at a position of a tile; -1 outside.  Only rows wrap, and once.
static int64_t rank_at(const Comm &c, const TilePlan &p, int64_t tile, const int16_t *at, bool column) {
    int64_t rank = 0;
    bool there = true;
    for (int i = 0; i < c.d; ++i) {
        const int j = c.d - 1 - i, n = c.dims[j];
        int64_t x = tile % p.tiles[j] * p.tile[j] + at[i];
        tile /= p.tiles[j];
        if (!column && c.periodic[j]) {
            x += x < 0 ? n : 0;
            x -= x >= n ? n : 0;
        }
        there = there && x >= 0 && x < n;
        rank += x * c.inner[j];
    }
    return there ? rank : -1;
}

// R (-) C^i, or R (+) C^i; -1 where a mesh has none.
static int64_t neighbour(const Comm &c, int64_t rank, int i, bool back) {
    int64_t out = 0;
    for (int j = 0; j < c.d; ++j) {
        const int64_t n = c.dims[j], at = rank / c.inner[j] % n, by = c.raw[(size_t)i * c.d + j];
        int64_t x = back ? at + by : at - by;
        if (c.periodic[j]) x = (x % n + n) % n;
        else if (x < 0 || x >= n) return -1;
        out += x * c.inner[j];
    }
    return out;
}

static void check(const Comm &c, const TilePlan &p, int heads, bool back, bool slots) {
    const int width = (c.d + 3) / 4 * 4, ranks = kTileColumns / heads;
    CHECK(p.heads == heads && p.rows > 0 && p.rows <= kTileMaxRows && p.chunks == (p.rows + kChunkRows - 1) / kChunkRows);
    CHECK(p.column_at.size() == (size_t)ranks * width && p.row_at.size() == (size_t)p.chunks * kChunkRows * width);
    CHECK(p.active.size() == (size_t)p.chunks && p.index.size() == (size_t)p.chunks * 4 * kTileWaves * 64 * 4);
    // the index: (column, neighbour) -> row
    std::map<std::pair<int, int>, int> row_of;
    std::set<std::pair<int, int>> column_row;
    std::vector<uint32_t> active((size_t)p.chunks, 0);
    for (int u = 0; u < p.chunks * kChunkRows; ++u)
        for (int column = 0; column < kTileColumns; ++column) {
            const int group = u / 16, lane = u % 16 / 4 * 16 + column % 16;
            const size_t at = (((size_t)(group / 2) * kTileWaves + column / 16) * 64 + lane) * 8 + group % 2 * 4 + u % 4;
            CHECK(p.index[at] % 4 == 0);
            const int value = p.index[at] / 4, h = value / (c.s + 1), i = value % (c.s + 1);
            CHECK(h == column % heads);
            if (i == c.s) continue;
            CHECK(u < p.rows && row_of.insert({{column, i}, u}).second);
            active[(size_t)(u / kChunkRows)] |= 1u << (column / 16 * 4 + group % 4);
        }
    CHECK(active == p.active);
    // positions, tile by tile: every rank is one column (of each head), and its neighbours are where the index says
    std::vector<int> seen((size_t)c.p, 0);
    for (int64_t tile = 0; tile < p.n_tiles; ++tile)
        for (int r = 0; r < ranks; ++r) {
            const int64_t rank = rank_at(c, p, tile, &p.column_at[(size_t)r * width], true);
            if (rank < 0) continue;
            ++seen[(size_t)rank];
            for (int i = 0; i < c.s; ++i) {
                const int64_t want = neighbour(c, rank, i, back);
                for (int h = 0; h < heads; ++h) {
                    const auto it = row_of.find({r * heads + h, i});
                    const int64_t got = it == row_of.end() ? -1 : rank_at(c, p, tile, &p.row_at[(size_t)it->second * width], false);
                    CHECK(got == want);
                }
            }
        }
    for (int n : seen) CHECK(n == 1);
    if (!slots) return;
    // the slots: each pair once, where its lane writes it
    const size_t round = 64 + 256 * (size_t)p.slot_words;
    CHECK(p.slots.size() == (size_t)p.chunks * 2 * kTileWaves * p.slot_rounds * round);
    std::set<std::tuple<int, int, int>> from_index, from_slots;
    for (const auto &[pair, u] : row_of) {
        const auto [column, i] = pair;
        const int place = (u % 32 / 16 * 64 + u % 16 / 4 * 16 + column % 16) * 4 + u % 4;
        from_index.insert({u / 32 * kTileWaves + column / 16, column % heads * c.s + i, place});
    }
    for (size_t l = 0; l < (size_t)p.chunks * 2 * kTileWaves; ++l) {
        std::set<uint32_t> used;
        for (int n = 0; n < p.slot_rounds; ++n) {
            const uint32_t *at = p.slots.data() + (l * p.slot_rounds + n) * round;
            for (int lane = 0; lane < 64; ++lane) {
                const uint32_t slot = at[lane];
                CHECK(slot <= (uint32_t)(heads * c.s));
                CHECK(slot == (uint32_t)(heads * c.s) || used.insert(slot).second);         // two lanes never add to one
                for (int w = 0; w < 4 * p.slot_words; ++w) {
                    const uint32_t two = at[64 + w / 4 * 256 + lane * 4 + w % 4];
                    for (uint32_t place : {two & 0xFFFF, two >> 16}) {
                        CHECK(place <= kSlotZero);
                        if (place == kSlotZero) continue;
                        CHECK(slot < (uint32_t)(heads * c.s) && from_slots.insert({(int)l, (int)slot, (int)place}).second);
                    }
                }
            }
        }
    }
    CHECK(from_slots == from_index);
}

int main() {
    std::mt19937 rng(7);
    const auto draw = [&](int64_t lo, int64_t hi) { return (int)((int64_t)(rng() % (uint64_t)(hi - lo + 1)) + lo); };
    int made = 0, refused = 0, without = 0;
    for (int k = 0; k < 400; ++k) {
        const int d = draw(1, 10) > 7 ? draw(4, 9) : draw(1, 3);
        const int most = d == 1 ? 300 : d == 2 ? 24 : d == 3 ? 9 : d < 6 ? 4 : 3;
        std::vector<int32_t> dims((size_t)d), periodic((size_t)d);
        for (auto &n : dims) n = draw(1, most);
        const bool mesh = draw(0, 1);
        for (auto &x : periodic) x = mesh ? draw(0, 1) : 1;
        const int s = draw(0, 9) ? draw(1, 40) : draw(100, 200), reach = draw(0, 3) ? draw(1, 4) : 400;
        std::vector<int32_t> rel((size_t)s * d);
        for (auto &x : rel) x = draw(0, 30) ? draw(-reach, reach) : draw(-2000000000, 2000000000);
        Comm c;
        if (build_comm(d, dims.data(), periodic.data(), s, rel.data(), c) != ISO_SUCCESS) return 2;
        what = "";
        for (int j = 0; j < d; ++j) what += std::to_string(dims[j]) + (periodic[j] ? "x" : "|x");
        what += " s " + std::to_string(s) + " reach " + std::to_string(reach);
        bool any = false;
        for (int64_t rank = 0; rank < c.p && !any; ++rank)
            for (int i = 0; i < s && !any; ++i) any = neighbour(c, rank, i, false) >= 0;
        for (int heads : {1, 2, 4, 8})
            for (int back = 0; back < (heads == 1 ? 2 : 1); ++back) {
                TilePlan p;
                std::vector<int> asked;
                const auto pays = [&](int rows, int64_t) { asked.push_back(rows); return true; };
                if (!build_tile_plan(c, heads, back, !back, p, pays)) {
                    CHECK(p.index.empty());
                    ++refused;
                    without += !any;
                    continue;
                }
                CHECK(any);                                         // nothing to stage: no tiles
                CHECK(asked.size() == 2 && asked[0] <= asked[1] && asked[1] == p.rows);
                check(c, p, heads, back, !back);
                ++made;
                // a no ends it at either question, and leaves no table
                for (size_t no = 0; no < 2; ++no) {
                    TilePlan none;
                    size_t n = 0;
                    CHECK(!build_tile_plan(c, heads, back, !back, none, [&](int, int64_t) { return n++ < no; }) && none.index.empty());
                }
            }
    }
    if (made < 1000 || !without || refused == without) return 3;
    std::printf("%d tables ok, %d refused, %d of them without any neighbour\n", made, refused, without);
    return 0;
}
