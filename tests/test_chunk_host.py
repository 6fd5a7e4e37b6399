"""Prompt chunks, draft trees and accepted drafts on the host: calls that must be refused before
any device is touched, and the work split's arithmetic (CPU only)."""

import random

import pytest


@pytest.fixture
def kv():
    import torch  # noqa: F401  (its HIP runtime has to be the one that the library finds)
    from paper_2609_25782_amd import hotcold_kv
    return hotcold_kv


@pytest.fixture
def meta(kv):
    d = kv.kv_pool_desc(2, 2, 64, 16, kv.KV_DTYPE_BF16, 8, 8, 0, 4, 4, 0, kv.KV_POOL_METADATA_ONLY)
    p = kv.kv_pool_create(d, 0, 0, 0, 0, 0)
    yield p
    kv.kv_pool_destroy(p)


def test_metadata_only_pools_are_refused(kv, meta):
    for pool in (meta, 0):
        for call in (lambda: kv.paged_prefill_attention(pool, 0, 16, 16, 4, 16, 4, 16, 1, 4, 0.1, 16, 256, 1 << 30),
                     lambda: kv.paged_tree_attention(pool, 0, 16, 16, 16, 16, 0, 4, 16, 4, 16, 1, 4, 0.1, 16, 256,
                                                     1 << 30),
                     lambda: kv.kv_accept_drafts(pool, 0, 1, 16, 4, 16, 16, 16, 1, 4, 16, 16)):
            with pytest.raises(kv.KVError) as e:
                call()
            assert e.value.status == kv.KV_ERR_INVALID
        assert kv.paged_prefill_workspace_bytes(pool, 1, 4, 4) == 0
        assert kv.paged_tree_workspace_bytes(pool, 1, 4, 4) == 0


# -- the work split: tiles laid end to end, cut into equal ranges --------------
# The same arithmetic as the kernel's (a tile's fixed cost, places of units), on plain integers.


def row_units(ctx, n, tok, block, tree, fixed):
    """Costs of a row's tiles of one KV head, and their numbers of blocks."""
    tiles = -(-n // tok)
    cost, blocks = [], []
    for i in range(tiles):
        if tree:
            nd = -(-n // block)
            cost.append(fixed + nd * block + ctx)
            blocks.append(nd + -(-ctx // block))
        else:
            keys = ctx + min((i + 1) * tok, n)
            cost.append(fixed + keys)
            blocks.append(-(-keys // block))
    return cost, blocks


def place(tiles, u, block, fixed):
    """Block that unit u begins with: (tile, block) over the flat list of (cost, blocks)."""
    for i, (cost, nb) in enumerate(tiles):
        if u < cost:
            if u == 0:
                return i, 0
            x = u - fixed
            k = min(nb, 0 if x <= 0 else -(-x // block))
            return (i, k) if k < nb else (i + 1, 0)
        u -= cost
    return len(tiles), 0


@pytest.mark.parametrize("tree", [False, True])
def test_every_block_belongs_to_one_worker(tree):
    rng = random.Random(5)
    for trial in range(300):
        block = rng.choice([32, 64])
        group = rng.choice([1, 2, 3, 5, 8, 16])
        tok = rng.choice([64, 256]) // group
        heads = rng.choice([1, 2, 4])
        fixed = rng.choice([64, 320])
        tiles = []
        for _ in range(rng.randint(1, 6)):
            ctx = rng.choice([0, 1, rng.randint(0, 100), rng.randint(0, 5000)])
            n = rng.choice([0, 1, rng.randint(1, 64)] if tree else [0, 1, rng.randint(1, 3000)])
            tiles += list(zip(*row_units(ctx, n, tok, block, tree, fixed))) * heads
        total = sum(c for c, _ in tiles)
        most = rng.choice([1, 7, 256, 512])
        workers = max(1, min(most, total // (fixed + 2 * block))) if total else 0
        cuts = [place(tiles, k * total // workers, block, fixed) for k in range(workers)] + [(len(tiles), 0)]
        assert not workers or cuts[0] == (0, 0)
        done = []
        for k in range(workers):
            at, end = cuts[k], cuts[k + 1]
            assert at < end, "worker %d of %d has nothing" % (k, workers)
            heads_cut = 0
            while at < end:
                tile, k0 = at
                nb = tiles[tile][1]
                k1 = end[1] if end[0] == tile else nb
                done.append((tile, k0, k1))
                heads_cut += k0 > 0
                if end[0] == tile:
                    break
                at = (tile + 1, 0)
            assert heads_cut <= 1           # one slot for a tile begun by another worker
        want = 0
        flat = iter(done)
        for tile, (_, nb) in enumerate(tiles):
            upto = 0
            while True:
                t, k0, k1 = next(flat)
                assert t == tile and k0 == upto and (k1 > k0 or nb == 0)
                upto = k1
                if upto == nb:
                    break
            want += 1
        assert next(flat, None) is None


# -- the other split: every tile in whole parts ---------------------------------


def whole_parts(rows, heads, tok, block, tree, most, tile_cost=320):
    """Kernel's rule on float32 numbers: [(row, head, tile, first block, end)] per worker, or None."""
    import numpy as np
    f = np.float32
    infos = []
    for ctx, n in rows:
        tiles = -(-n // tok)
        slope = 0 if tree else tok
        last = -(-n // block) * block + ctx if tree else ctx + n
        if not (tiles <= 1 or slope == 0 or n * 4 <= ctx) or heads * tiles > most:
            return None
        infos.append((ctx, n, tiles, f(last) if tiles else f(0)))
    total = f(sum(c * f(heads * t) for _, _, t, c in infos))
    split, longest = [], f(0)
    for ctx, n, tiles, cost in infos:
        blocks = row_units(ctx, n, tok, block, tree, 0)[1]
        w = max(1, min(int(f(most) * cost / max(total, f(1))), blocks[0] // 2 if tiles else 0))
        split.append((tiles, w, blocks))
        longest = max(longest, cost / f(w))
    if sum(heads * t * w for t, w, _ in split) > most or longest > f(1.125) * (total / f(most)) + f(tile_cost):
        return None
    out = []
    for b, (tiles, w, blocks) in enumerate(split):
        for g in range(heads):
            for t in range(tiles):
                nb = blocks[t]
                cut = [p * (nb % w) // w + p * (nb // w) for p in range(w + 1)]
                out += [(b, g, t, cut[p], cut[p + 1]) for p in range(w)]
    return out


@pytest.mark.parametrize("tree", [False, True])
def test_equal_parts_cover_every_tile_once(tree):
    rng = random.Random(8)
    taken = 0
    for trial in range(600):
        block = rng.choice([32, 64])
        group = rng.choice([1, 2, 3, 5, 8, 16])
        tok = rng.choice([128, 256]) // group
        heads = rng.choice([1, 2, 4, 8])
        most = rng.choice([8, 256, 304])
        base = rng.choice([0, 5, 300, 5000, 100000])
        rows = [(base + rng.randint(0, 1 + base // rng.choice([2, 50])),
                 rng.choice([0, 1, rng.randint(1, 64), rng.randint(1, 64 if tree else 300)]))
                for _ in range(rng.randint(1, 12))]
        parts = whole_parts(rows, heads, tok, block, tree, most)
        if parts is None:
            continue
        taken += 1
        assert len(parts) <= most
        want = []
        for b, (ctx, n) in enumerate(rows):
            blocks = row_units(ctx, n, tok, block, tree, 0)[1]
            want += [(b, g, t, nb) for g in range(heads) for t, nb in enumerate(blocks)]
        got = iter(parts)
        for b, g, t, nb in want:
            upto = 0
            while True:
                part = next(got)
                assert part[:4] == (b, g, t, upto)
                assert part[4] >= upto + 2 or part[3:] == (0, nb)     # a whole tile, or two blocks or more
                upto = part[4]
                if upto == nb:
                    break
        assert next(got, None) is None
    assert taken > 100
