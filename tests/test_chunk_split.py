"""The work split of prompt and tree attention as the kernel computes it (csrc/chunk_split.h,
compiled here for the host): every block of every tile belongs to one worker, and the workers
that the merge joins are those that hold a part (CPU only)."""

import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_25782_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("split") / "chunk_split.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-Wall", "-I", CSRC, "-o",
                           out, os.path.join(HERE, "chunk_split_host.cpp")])
    return ctypes.CDLL(out)


def split(lib, tree, block, tok, heads, most, rows):
    """(whole parts?, pieces) of rows (ctx, n, bad)."""
    ctx, n, bad = (np.array(x, np.int32) for x in zip(*rows))
    cap = most * 2 + heads * int(sum(-(-int(x) // tok) for x in n))
    out, whole = np.zeros((cap, 8), np.int64), ctypes.c_int(0)
    p = [x.ctypes.data_as(ctypes.c_void_p) for x in (ctx, n, bad, out)]
    count = lib.chunk_split(int(tree), block, tok, heads, most, len(rows), p[0], p[1], p[2], ctypes.byref(whole), p[3],
                            cap)
    assert count <= cap
    return bool(whole.value), out[:count].tolist()


def blocks_of(tree, block, tok, row, tile):
    ctx, n, bad = row
    if bad:
        return 0
    if tree:
        return -(-n // block) + -(-ctx // block)
    return -(-(ctx + min(n, (tile + 1) * tok)) // block)


def verify(tree, block, tok, heads, most, rows, pieces):
    got = iter(pieces)
    parts_of = {}                # worker: the slots that it fills
    last = 0
    for b, row in enumerate(rows):
        for g in range(heads):
            for tile in range(-(-row[1] // tok)):
                nb = blocks_of(tree, block, tok, row, tile)
                upto, holders, parts = 0, [], None
                while True:
                    k, pb, pg, pt, k0, k1, pn, p = next(got)
                    assert (pb, pg, pt, pn) == (b, g, tile, nb) and last <= k < most
                    assert k0 == upto and (k1 > k0 or nb == 0)
                    last = k
                    holders.append(k)
                    if not (k0 == 0 and k1 == nb):
                        slot = (k, k0 == 0)
                        assert slot not in parts_of       # one place in the workspace, one part
                        parts_of[slot] = (b, g, tile)
                        if k0 == 0:
                            parts = p
                    upto = k1
                    if upto == nb:
                        break
                if len(holders) > 1:                      # what the merge reads is what was written
                    assert holders == list(range(holders[0], holders[0] + parts))
    assert next(got, None) is None


def random_rows(rng, tree, many):
    kind = rng.randrange(4)
    base = rng.choice([0, 5, 300, 5000, 100000, 1 << 24])
    rows = []
    for _ in range(rng.randint(65, 200) if many else rng.randint(1, 64 if kind == 0 else 8)):
        ctx = base + rng.randint(0, 1 + base // 50) if kind < 2 else rng.choice([0, 1, rng.randint(0, 100), rng.randint(0, 1 << rng.randint(1, 20))])
        n = rng.choice([0, 1, rng.randint(1, 64), rng.randint(1, 64 if tree else 1 << rng.randint(1, 13))])
        rows.append((ctx, n, int(rng.random() < 0.05)))
    return rows


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_every_block_has_one_worker(lib, tree, many):
    rng = random.Random(60 + 2 * tree + many)
    seen = {False: 0, True: 0}
    for trial in range(1500 if not many else 200):
        block, group = rng.choice([32, 64]), rng.choice([1, 2, 3, 5, 8, 16])
        args = tree, block, rng.choice([128, 256]) // group, rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 7, 8, 256, 304])
        rows = random_rows(rng, tree, many)
        whole, pieces = split(lib, *args, rows)
        verify(*args, rows, pieces)
        seen[whole] += 1
    assert seen[False] > 100 and (many or seen[True] > 100)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("shift", [-3, -1, 0, 1, 700])
def test_units_around_2_32(lib, tree, shift):
    """Totals on both sides of 32 bits, where other divisions are taken."""
    rng = random.Random(70)
    for heads in (1, 4, 16):
        for trial in range(20):
            tok, block = rng.choice([16, 256]), rng.choice([32, 64])
            rows = []
            for _ in range(rng.randint(2, 5)):
                rows.append([0, rng.randint(1, 64 if tree else 40 * tok), 0])
            # one long row brings the total (keys and tiles' costs) to about 2^32
            tiles = [-(-r[1] // tok) for r in rows]
            spent = sum(heads * t * 320 for t in tiles) + sum(heads * t * r[1] // (1 if tree else 2) for r, t in zip(rows, tiles))
            i = rng.randrange(len(rows))
            rows[i][0] = min(1 << 30, max(0, (2 ** 32 - spent) // (heads * tiles[i]) + shift))
            rows = [tuple(r) for r in rows]
            for most in (7, 256):
                whole, pieces = split(lib, tree, block, tok, heads, most, rows)
                verify(tree, block, tok, heads, most, rows, pieces)


def test_the_longest_rows(lib):
    """Rows of 2^30 tokens, in many heads: totals far past 2^32."""
    for heads in (1, 16):
        for rows in ([(1 << 30, 64, 0)] * 3, [((1 << 30) - 5000, 5000, 0), (0, 1, 0), (1 << 29, 300, 0)],
                     [(3, 2, 0), (1 << 30, 0, 0), (1 << 30, 0, 1), ((1 << 30) - 1, 1, 0)]):
            for tree in (False, True):
                if tree and max(r[1] for r in rows) > 64:
                    continue
                whole, pieces = split(lib, tree, 64, 16, heads, 256, rows)
                verify(tree, 64, 16, heads, 256, rows, pieces)
