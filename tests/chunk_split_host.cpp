// The work split of prompt and tree attention on the host: what every worker of a call takes, from
// the arithmetic that the kernel uses (chunk_split.h).  Lanes and threads are loops here.

#include "chunk_split.h"

#include <vector>

using namespace hck;

namespace {

template <int BLOCK>
struct Config {
    static constexpr int kBlock = BLOCK;
};

template <class C, bool TREE>
int split(int tok, int heads, int most, int batch, const int* ctx, const int* n, const int* bad, int* whole,
          int64_t* out, int cap) {
    std::vector<Row> rows;
    for (int b = 0, start = 0; b < batch; start += n[b++])
        rows.push_back(make_row<C, TREE>(tok, start, n[b], bad[b] ? 0 : ctx[b], bad[b]));
    int count = 0;
    const auto put = [&](int k, int b, int g, int tile, int k0, int k1, int nb, int parts) {
        if (count < cap) {
            const int64_t v[8] = {k, b, g, tile, k0, k1, nb, parts};
            for (int i = 0; i < 8; ++i) out[8 * count + i] = v[i];
        }
        ++count;
    };
    // a worker's walk from `at` to `end`
    const auto walk = [&](int k, Place at, Place end, int parts) {
        while (before(at, end) && at.b < batch) {
            const Row& r = rows[at.b];
            if (at.g >= heads || r.tiles == 0) {
                at = Place{at.b + 1, 0, 0, 0};
                continue;
            }
            const int nb = tile_blocks<C, TREE>(tok, r, at.tile);
            const bool to_end = end.b == at.b && end.g == at.g && end.tile == at.tile;
            put(k, at.b, at.g, at.tile, at.blk, to_end ? end.blk : nb, nb, parts);
            if (to_end) break;
            at.blk = 0;
            if (++at.tile == r.tiles) {
                at.tile = 0;
                ++at.g;
            }
        }
    };
    *whole = 0;
    bool even = batch <= 64;
    for (const Row& r : rows) even = even && even_tiles(r) && static_cast<int64_t>(heads) * r.tiles <= most;
    if (even) {
        float t[64] = {}, u[64];
        for (int b = 0; b < batch; ++b) t[b] = tile_cost(rows[b]) * (heads * rows[b].tiles);
        for (int d = 1; d < 64; d <<= 1) {
            for (int i = 0; i < 64; ++i) u[i] = t[i] + t[i ^ d];
            for (int i = 0; i < 64; ++i) t[i] = u[i];
        }
        float longest = 0.f;
        int64_t all = 0;
        for (const Row& r : rows) {
            const int w = tile_parts<C, TREE>(tok, r, most, t[0]);
            const float part = tile_cost(r) / w;
            longest = part > longest ? part : longest;
            all += static_cast<int64_t>(heads) * r.tiles * w;
        }
        if (all <= most && !parts_too_long(longest, t[0], most)) {
            *whole = 1;
            int k = 0;
            for (int b = 0; b < batch; ++b) {
                const int w = tile_parts<C, TREE>(tok, rows[b], most, t[0]);
                for (int rem = 0; rem < heads * rows[b].tiles * w; ++rem, ++k) {
                    Place from, to;
                    part_place<C, TREE>(tok, rows[b], b, rem, w, from, to);
                    walk(k, from, to, w);
                }
            }
            return count;
        }
    }
    int64_t keys = 0, tiles = 0;
    for (const Row& r : rows) {
        keys += heads * r.head_units(0);
        tiles += static_cast<int64_t>(heads) * r.tiles;
    }
    const Cuts cuts = cuts_of<C>(most, keys, tiles);
    const auto find = [&](int64_t u, int64_t& more) {
        int64_t first = 0;
        for (int b = 0; b < batch; ++b) {
            const int64_t units = heads * rows[b].head_units(cuts.cost);
            if (u < first + units) return place_of<C, TREE>(tok, rows[b], b, u - first, cuts.cost, more);
            first += units;
        }
        return Place{batch, 0, 0, 0};
    };
    for (int k = 0; k < cuts.workers; ++k) {
        int64_t more = 0;
        const Place from = find(cuts.at(k), more), to = find(cuts.at(k + 1), more);
        walk(k, from, to, cuts.at(k + 1) < cuts.total && to.blk > 0 ? worker_at(cuts, cuts.at(k + 1) + more) - k + 1 : 0);
    }
    return count;
}

}  // namespace

// Pieces as [worker, row, KV head, tile, first block, end, the tile's blocks, parts]; their number.
// `parts` is what the worker gives for a tile cut at its range's end.
extern "C" int chunk_split(int tree, int block, int tok, int heads, int most, int batch, const int* ctx, const int* n,
                           const int* bad, int* whole, int64_t* out, int cap) {
    const auto f = block == 64 ? (tree ? split<Config<64>, true> : split<Config<64>, false>)
                               : (tree ? split<Config<32>, true> : split<Config<32>, false>);
    return f(tok, heads, most, batch, ctx, n, bad, whole, out, cap);
}
