// The work split of prompt and tree attention in plain integers: rows, their tiles and blocks, and
// the cuts between workers.  Every worker computes its range from these, and a tile's parts are
// joined by them, so they hold nothing of the device and compile for the host as well.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define HCK_HD __host__ __device__ __forceinline__
#else
#define HCK_HD inline
#endif

namespace hck {

// What one row b brings: n tokens (or drafts), `ctx` tokens before them, the row's units.
struct Row {
    int start;     // first query of the row in q (tokens)
    int n;         // queries
    int ctx;       // cached tokens that every query sees
    int bad;       // 1: lengths that do not fit, the row's outputs are NaN
    int tiles;     // tiles per KV head
    int64_t base;  // keys of tile i < tiles - 1: base + slope (i + 1)
    int64_t slope;
    int64_t last;  // keys of the last tile
    // First unit of tile i, and all units of one KV head, where a tile costs its keys and `cost` more.
    HCK_HD int64_t tile_start(int64_t i, int cost) const {
        return i * (base + cost) + slope * (i * (i + 1) / 2);
    }
    HCK_HD int64_t head_units(int cost) const { return tiles ? tile_start(tiles - 1, cost) + last + cost : 0; }
};

// What a tile costs beside its keys, in keys: its queries' load, its output, the pipeline's
// start and the masked blocks.  kTileCost is what balances calls with work for every worker
// (twelve packed prompts: 64: 1510 us, 192: 1195, 320: 1037, 448: 1041, 640: 1060; with 64 dims
// 985, 778, 711, 740 and 768; in float32, where a key costs more, 6 prompts of 100-2000 tokens over
// up to 2000: 507, 537, 528, 550 and 559).  Calls with less than that are cut finer, with
// kTileCostFine (2 x 5 float32 drafts: 64: 13.5 us, 320: 13.9; 12 chunks of 20-300 tokens 56.3 and
// 56.0; 7 chunks of 1-701 tokens, 3 heads of 64 dims: 32.7 and 31.1).
constexpr int kTileCost = 320, kTileCostFine = 64;

// The units of a row that brings n queries after ctx tokens.
template <class C, bool TREE>
HCK_HD Row make_row(int tile_tokens, int start, int n, int ctx, int bad) {
    Row r;
    r.start = start;
    r.n = n;
    r.ctx = ctx;
    r.bad = bad;
    r.tiles = (n + tile_tokens - 1) / tile_tokens;
    r.slope = 0;
    if (bad) {
        r.base = r.last = 0;
    } else if constexpr (TREE) {
        r.base = r.last = static_cast<int64_t>((n + C::kBlock - 1) / C::kBlock) * C::kBlock + ctx;
    } else {
        r.base = ctx;
        r.slope = tile_tokens;
        r.last = r.base + n;
    }
    return r;
}

// Blocks of tile i: the drafts' first (trees), then the context's.
template <class C, bool TREE>
HCK_HD int draft_blocks(const Row& r) {
    return TREE && !r.bad ? (r.n + C::kBlock - 1) / C::kBlock : 0;
}
template <class C, bool TREE>
HCK_HD int tile_keys(int tile_tokens, const Row& r, int i) {
    if (r.bad) return 0;
    if (TREE) return r.ctx;
    const int64_t hi = static_cast<int64_t>(i + 1) * tile_tokens;
    return r.ctx + (hi < r.n ? static_cast<int>(hi) : r.n);
}
template <class C, bool TREE>
HCK_HD int tile_blocks(int tile_tokens, const Row& r, int i) {
    return draft_blocks<C, TREE>(r) + (tile_keys<C, TREE>(tile_tokens, r, i) + C::kBlock - 1) / C::kBlock;
}

// A place in the order of blocks: block `blk` of tile `tile` of (row b, KV head g).
struct Place {
    int b, g, tile, blk;
};

// How the call's units are cut: `total` units over `workers` equal ranges, a tile costing its
// keys and `cost` more.
struct Cuts {
    int64_t total;
    int workers, cost;
    HCK_HD int64_t at(int k) const {   // floor(k total / workers), in 32 bits where they do
        if ((total >> 32) == 0) {
            const unsigned t = static_cast<unsigned>(total), w = static_cast<unsigned>(workers);
            const unsigned q = t / w, m = t - q * w, n = static_cast<unsigned>(k);
            return static_cast<int64_t>(n * q + n * m / w);
        }
        return k * (total / workers) + k * (total % workers) / workers;
    }
};

// Enough units for a block or more in every range (see place_of).
template <class C>
HCK_HD Cuts cuts_of(int most, int64_t keys, int64_t tiles) {
    Cuts c;
    c.cost = kTileCost;
    if (keys + c.cost * tiles < static_cast<int64_t>(c.cost + 2 * C::kBlock) * most) c.cost = kTileCostFine;
    c.total = keys + c.cost * tiles;
    const int64_t n = (c.total >> 32) == 0
                          ? static_cast<int64_t>(static_cast<unsigned>(c.total) / static_cast<unsigned>(c.cost + 2 * C::kBlock))
                          : most;
    c.workers = c.total <= 0 ? 0 : static_cast<int>(n < 1 ? 1 : (n > most ? most : n));
    return c;
}

// The place of unit `u` of row b (0 <= u < its units).  Both workers at a cut compute it
// from the same numbers, so their ranges meet without a gap; a place past a tile's last
// block is the next tile's first.  A tile without blocks belongs to the worker that has
// its first unit.  Ranges of at least cost + 2 kBlock units hold one block or more.
// `more`: for a place inside a tile, how many units further a cut still lies inside it.
template <class C, bool TREE>
HCK_HD Place place_of(int tile_tokens, const Row& r, int b, int64_t u, int cost, int64_t& more) {
    Place p;
    p.b = b;
    const int64_t h = r.head_units(cost);
    if (((u | h) >> 32) == 0) {
        p.g = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(h));
    } else {
        p.g = static_cast<int>(u / h);
    }
    int64_t rem = u - p.g * h;
    int lo = 0, hi = r.tiles - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (r.tile_start(mid, cost) <= rem) lo = mid; else hi = mid - 1;
    }
    rem -= r.tile_start(lo, cost);
    p.tile = lo;
    p.blk = 0;
    more = 0;
    if (rem > 0) {
        const int64_t x = rem - cost;
        const int nb = tile_blocks<C, TREE>(tile_tokens, r, lo);
        const int64_t k = x <= 0 ? 0 : (x + C::kBlock - 1) / C::kBlock;
        p.blk = k < nb ? static_cast<int>(k) : nb;
        more = static_cast<int64_t>(nb - 1) * C::kBlock - x;
        if (p.blk == nb) {
            p.blk = 0;
            if (++p.tile == r.tiles) {
                p.tile = 0;
                ++p.g;    // may be the number of KV heads: the walk moves on to the next row
            }
        }
    }
    return p;
}

HCK_HD bool before(const Place& x, const Place& y) {
    if (x.b != y.b) return x.b < y.b;
    if (x.g != y.g) return x.g < y.g;
    if (x.tile != y.tile) return x.tile < y.tile;
    return x.blk < y.blk;
}

// The last worker whose range begins at unit `u` or before.
HCK_HD int worker_at(const Cuts& c, int64_t u) {
    const int64_t n = (u + 1) * c.workers - 1;
    const int64_t k = ((n | c.total) >> 32) == 0
                          ? static_cast<int64_t>(static_cast<unsigned>(n) / static_cast<unsigned>(c.total))
                          : n / c.total;
    return k < c.workers ? static_cast<int>(k) : c.workers - 1;
}

// Where no more than `workers` tiles have about the same cost in each row (drafts, short
// chunks over long contexts) and equal parts of them differ little, every tile is cut into
// whole parts, as many as its share of the workers: no worker then has parts of two tiles,
// whose starts and ends follow each other.  8 sessions x 8 drafts over 2K tokens: 23.9 us with
// ranges, 19.3 so; 2 x 5 drafts in float32: 17.0 and 13.5.  Taken without looking at
// the longest part, 32 sessions of 8K to 32K tokens lose (240 us with ranges, 305 so).  Parts
// up to an eighth longer than even ones are taken: tiles of one row, cut alike, read the same
// keys at the same time, from one L2 (4 sessions x 49-64 drafts, two tiles a row: 192 us with
// ranges, 180 so); with one tile a row the difference is small (4 x 32 drafts over 8K: 43.7 and 44.9).
HCK_HD bool even_tiles(const Row& r) {
    return r.tiles <= 1 || r.slope == 0 || static_cast<int64_t>(r.n) * 4 <= r.ctx;
}
HCK_HD float tile_cost(const Row& r) { return r.tiles ? static_cast<float>(r.last) : 0.f; }
// Parts of each of a row's tiles; `total` is the cost of all tiles of the call.
template <class C, bool TREE>
HCK_HD int tile_parts(int tile_tokens, const Row& r, int most, float total) {
    const int w = static_cast<int>(most * tile_cost(r) / (total > 1.f ? total : 1.f));
    const int half = (r.tiles ? tile_blocks<C, TREE>(tile_tokens, r, 0) : 0) / 2;      // of its shortest tile
    const int least = w < half ? w : half;
    return least > 1 ? least : 1;
}
HCK_HD bool parts_too_long(float longest, float total, int most) {
    return longest > 1.125f * (total / most) + kTileCost;
}
// Blocks [from, to) of the `rem`-th part of row b's tiles, which are cut into `parts` each.
template <class C, bool TREE>
HCK_HD void part_place(int tile_tokens, const Row& r, int b, int rem, int parts, Place& from, Place& to) {
    const unsigned at = static_cast<unsigned>(rem) / static_cast<unsigned>(parts);
    const int part = rem - at * parts;
    const int g = at / static_cast<unsigned>(r.tiles), tile = at - g * r.tiles;
    const int blocks = tile_blocks<C, TREE>(tile_tokens, r, tile);
    const auto cut = [&](int p) {      // p blocks / parts
        return static_cast<int>(static_cast<unsigned>(p * (blocks % parts)) / static_cast<unsigned>(parts)) +
               p * (blocks / parts);
    };
    const int end = cut(part + 1);
    from = Place{b, g, tile, cut(part)};
    to = end == blocks ? Place{b, g, tile + 1, 0} : Place{b, g, tile, end};
}

}  // namespace hck
