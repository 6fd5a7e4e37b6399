"""Speculative steps whose sessions are evicted and resumed between them: every accepted draft is
still there, whatever was rejected (kv_session_reserve before each step's drafts)."""

import numpy as np
import pytest
import torch

from chunk_reference import TORCH, attend, check, i32, mask_tensor, random_tree, tree_reference
from paper_2609_25782_amd.pool import HotColdPool

pytestmark = pytest.mark.gpu


class Mirror:
    """What tree_reference reads: the sessions' K and V on the CPU."""

    def __init__(self, d, dtype, k, v):
        self.d, self.dtype, self.k, self.v = d, dtype, k, v


@pytest.mark.parametrize("cold", ["device", "host"])
@pytest.mark.parametrize("lazy", [False, True])
@pytest.mark.parametrize("dtype,width", [("bf16", 6), ("f32", 6), ("bf16", 40)])
def test_accepted_tokens_survive_evictions(dtype, width, lazy, cold):
    layers, hq, hkv, d = 2, 4, 2, 64
    t = TORCH[dtype]
    g = torch.Generator().manual_seed(40 + width)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(t)

    lens = [10, 100, 16, 31]
    B = len(lens)
    pool = HotColdPool(layers, hkv, d, dtype, 120, 200, B, 32, cold_location=cold)
    pool.set_spill(lazy)
    pool.hot.view(t).fill_(float("nan"))
    s = Mirror(d, dtype, [normal(layers, n, hkv, d) for n in lens], [normal(layers, n, hkv, d) for n in lens])
    for b, n in enumerate(lens):
        pool.create_session(n)
        pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    rng = np.random.default_rng(41)
    for turn in range(6):
        for b in range(B):
            pool.reserve(b, lens[b], lens[b] + width)
        table = pool.page_table.clone()
        q, hk, hv = normal(layers, B, width, hq, d), normal(layers, B, width, hkv, d), normal(layers, B, width, hkv, d)
        masks = [random_tree(rng, width, width) for _ in range(B)]
        # none, few, all, any
        n = [0, min(2, width), width if turn % 2 else 1, int(rng.integers(0, width, endpoint=True))]
        n = [n[(b + turn) % B] for b in range(B)]
        path = np.zeros((B, width), np.int32)
        for b in range(B):
            path[b, :n[b]] = np.sort(rng.permutation(width)[:n[b]])
        d_lens, kd, vd = i32(lens), hk.cuda(), hv.cuda()
        for layer in range(layers):
            got = pool.tree_decode(layer, q[layer].cuda(), kd[layer], vd[layer], mask_tensor(masks), d_lens, page_table=table)
            check(got, *tree_reference(s, q[layer], hk[layer], hv[layer], masks, lens, [width] * B, layer),
                  what="turn %d layer %d" % (turn, layer))
        pool.accept_drafts(0, table, d_lens, torch.from_numpy(path).cuda(), i32(n), kd, vd)
        for b in range(B):
            s.k[b] = torch.cat([s.k[b], hk[:, b, path[b, :n[b]]]], dim=1)
            s.v[b] = torch.cat([s.v[b], hv[:, b, path[b, :n[b]]]], dim=1)
            lens[b] += n[b]
        if turn % 3 != 1:
            torch.cuda.synchronize()
            pool.evict(list(range(B)))
            pool.hot.view(t).fill_(float("nan"))
            if lazy:
                pool.resume_lazy(list(range(B)))
                pool.promote(int(rng.integers(0, 12)))
            else:
                pool.resume([2, 0, 3, 1])
    for b in range(B):
        pool.reserve(b, lens[b], lens[b])
        assert len(pool.info(b)[2]) == -(-lens[b] // 16) and pool.info(b)[1] == lens[b]
    torch.cuda.synchronize()
    rows = pool.page_table.cpu().numpy()
    for b in range(B):
        assert (rows[b, -(-lens[b] // 16):] == -1).all()
    for layer in range(layers):
        q = normal(B, hq, d)
        got = pool.decode(layer, q.cuda(), i32(lens))
        for b in range(B):
            ref, bound = attend(q[b:b + 1], s.k[b][layer], s.v[b][layer], np.ones((1, lens[b]), bool), d ** -0.5, dtype)
            check(got[b:b + 1], ref, 2 * bound, what="decode, session %d layer %d" % (b, layer))


@pytest.mark.parametrize("pages", [20, 3000])     # ids in the kernel arguments, an uploaded list
def test_released_pages_wait_for_the_stream(pages):
    """A session gives its pages back on a stream with other work before it; the session that takes
    them on a second stream, and the room made again in the first one's row, come after that."""
    pool = HotColdPool(1, 1, 64, "bf16", pages, 0, 2, pages)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    old = torch.ones((16 * pages, 1, 64), dtype=torch.bfloat16, device="cuda")
    new = torch.full_like(old, 2.0)
    m = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
    torch.mm(m, m)
    torch.cuda.synchronize()
    sid = pool.create_session(16 * pages, stream=a)
    with torch.cuda.stream(a):
        for _ in range(60):
            torch.mm(m, m)
    pool.write_tokens(sid, 0, 0, old, old, stream=a)
    pool.reserve(sid, 16, 16, stream=a)
    released = torch.cuda.Event()
    released.record(a)
    other = pool.create_session(16 * (pages - 2), stream=b)
    pool.write_tokens(other, 0, 0, new[32:], new[32:], stream=b)
    pool.reserve(sid, 16, 17, stream=b)
    assert not released.query(), "the delay was too short for the test to show anything"
    torch.cuda.synchronize()
    row = pool.page_table.cpu()
    first, rest = pool.info(sid)[2], pool.info(other)[2]
    assert row[sid, :3].tolist() == first + [-1] and row[other, :pages - 2].tolist() == rest
    held = pool.hot_page_bytes().view(torch.bfloat16).view(pages, -1)
    assert (held[torch.tensor(rest)] == 2).all() and (held[first[0]] == 1).all()
