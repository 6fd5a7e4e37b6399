"""Decode attention over listed pages (paged_sparse_attention) against the definition, and the
run of bounds, choice and attention as a serving loop has it."""

import numpy as np
import pytest
import torch

from chunk_reference import Sessions, check, i32, pages_for
from paper_2609_25782_amd import hotcold_kv as kv
from sparse_reference import attend_pages, choose, page_bounds, scores, values

pytestmark = pytest.mark.gpu

SHAPES = [(8, 1, 128, "bf16"), (32, 4, 128, "bf16"), (6, 2, 64, "bf16"), (16, 1, 64, "bf16"), (3, 3, 128, "bf16"),
          (16, 16, 64, "bf16"), (4, 1, 64, "f32"), (10, 2, 128, "f32")]


def reference(s, q, lens, lists, scale=None, layer=0):
    scale = s.d ** -0.5 if scale is None else scale
    out, bound = np.zeros(tuple(q.shape)), np.zeros(tuple(q.shape))
    for b, n in enumerate(lens):
        out[b], bound[b] = attend_pages(q[b], s.k[b][layer], s.v[b][layer], n, lists[b], scale, s.dtype)
    return out, bound


def tensors(lists, width, hkv):
    """(picks, counts) of lists[b][g], padded with -1."""
    picks = np.full((len(lists), hkv, width), -1, np.int32)
    for b, row in enumerate(lists):
        for g, pages in enumerate(row):
            picks[b, g, :len(pages)] = pages
    return torch.from_numpy(picks).cuda(), i32([len(p) for row in lists for p in row]).view(len(lists), hkv)


def random_lists(rng, lens, hkv, width):
    lists = []
    for n in lens:
        P = pages_for(n)
        lists.append([sorted(rng.permutation(P)[:min(P, int(rng.integers(0, width + 1)))].tolist()) for _ in range(hkv)])
    return lists


def call(s, q, lens, lists, width, scale=None, with_counts=True, **kw):
    picks, counts = tensors(lists, width, s.hkv)
    kw.setdefault("out", torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"))
    return s.pool.sparse_decode(0, q.cuda(), i32(lens), picks, counts if with_counts else None, scale=scale, **kw)


@pytest.mark.parametrize("width", [1, 3, 31, 100, 700])
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_matches_definition(hq, hkv, d, dtype, width):
    lens = [1, 15, 16, 17, 0, 333, 1600, 5000]
    s = Sessions(lens, hq, hkv, d, dtype, seed=1)
    q = s.normal(len(lens), hq, d)
    lists = random_lists(np.random.default_rng(width), lens, hkv, width)
    lists[7] = [list(range(pages_for(5000)))[-width:]] * hkv
    for counts in (True, False):
        check(call(s, q, lens, lists, width, with_counts=counts), *reference(s, q, lens, lists), "counts %s" % counts)


def test_order_and_repetition():
    """Lists need no order; a page listed twice counts twice; entries outside the row are passed over."""
    lens = [100, 100, 100, 40]
    s = Sessions(lens, 4, 2, 64, "f32", seed=2)
    q = s.normal(4, 4, 64)
    lists = [[[6, 0, 3], [2, 2, 5]], [[7, 1, -3, 1 << 30], [-1, -1]], [[1] * 9, [6, 6]], [[2, 1, 0], [3, 2]]]
    check(call(s, q, lens, lists, 9), *reference(s, q, lens, lists))


def test_empty_lists_and_bad_lengths():
    lens = [100, 50, 70, 0]
    s = Sessions([100, 50, 70, 30], 8, 2, 128, "bf16", seed=3)
    q = s.normal(4, 8, 128)
    lists = [[[], [1]], [[0, 1], [2]], [[1], [0]], [[0], [1]]]
    ref, bound = reference(s, q, lens, lists)
    assert not ref[0, :4].any() and not ref[3].any()
    check(call(s, q, lens, lists, 4), ref, bound)
    picks, _ = tensors(lists, 4, 2)
    counts = i32([-3, 99, 2, 1, 1, 1, 0, 0]).view(4, 2)     # past the ends: none, and all of the four
    check(s.pool.sparse_decode(0, q.cuda(), i32(lens), picks, counts), ref, bound)
    bad = [-1, 50, 16 * s.pool.stride + 1, 0]
    ref[[0, 2]] = np.nan
    check(call(s, q, bad, lists, 4), ref, bound)


@pytest.mark.parametrize("bad", [-1, 1 << 20, (1 << 29) | 1, (1 << 30) | 3])
def test_bad_pages(bad):
    """A list with a page outside the pools is NaN; lists without it are not."""
    s = Sessions([200, 90], 8, 2, 128, "bf16", seed=4, cold=8)
    q = s.normal(2, 8, 128)
    table = s.pool.page_table[:2].clone()
    table[0, 3] = bad
    lists = [[[1, 3, 7], [0, 2, 12]], [[3], [5, 1]]]
    ref, bound = reference(s, q, [200, 90], lists)
    ref[0, :4] = np.nan
    check(call(s, q, [200, 90], lists, 5, page_table=table), ref, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_not_listed_do_not_matter(dtype):
    lens = [16 * 12 + 5]
    s = Sessions(lens, 4, 2, 64, dtype, seed=5)
    q = s.normal(1, 4, 64)
    lists = [[[0, 5, 12], [3, 12]]]
    ref, bound = reference(s, q, lens, lists)
    for page, value in ((1, float("nan")), (4, float("inf")), (11, float("-inf"))):
        s.k[0][0, page * 16:page * 16 + 16] = value
        s.v[0][0, page * 16:page * 16 + 16] = value
    s.pool.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())
    check(call(s, q, lens, lists, 3), ref, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype):
    """Such tokens weigh nothing, wherever in a list they come; with no others the output is NaN."""
    lens = [160, 32]
    s = Sessions(lens, 2, 1, 64, dtype, seed=6)
    q = s.normal(2, 2, 64).abs() + 0.1
    s.k[0][0, :48] = float("-inf")
    s.k[1][0] = float("-inf")
    for b in range(2):
        s.pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    q = q.to(s.k[0].dtype)
    lists = [[[0, 1, 2, 5, 9]], [[0, 1]]]
    ref, bound = reference(s, q, lens, [[[5, 9]], [[]]])
    ref[1] = np.nan
    check(call(s, q, lens, lists, 5), ref, bound)
    check(call(s, q, lens, [[[9, 5, 2, 1, 0]], [[0, 1]]], 5), ref, bound)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_scales(scale):
    lens = [70, 33]
    s = Sessions(lens, 4, 2, 64, "bf16", seed=7)
    q = s.normal(2, 4, 64)
    lists = [[[0, 4], [1, 2, 4]], [[2], [0, 1, 2]]]
    check(call(s, q, lens, lists, 3, scale=scale), *reference(s, q, lens, lists, scale=scale))


def test_spilled_pages_are_read_in_place():
    lens = [300]
    s = Sessions(lens, 8, 2, 128, "bf16", seed=8, cold=30)
    s.pool.set_spill(True)
    s.pool.evict(0)
    s.pool.resume_lazy(0)
    assert s.pool.promote(7) == 7
    q = s.normal(1, 8, 128)
    lists = [[[0, 6, 7, 18], [3, 9, 10, 11, 17]]]
    check(call(s, q, lens, lists, 6), *reference(s, q, lens, lists))


def test_every_page_listed_is_the_dense_decode():
    lens = [500, 1200, 31]
    s = Sessions(lens, 32, 4, 128, "bf16", seed=9)
    q = s.normal(3, 32, 128)
    lists = [[list(range(pages_for(n)))] * 4 for n in lens]
    ref, bound = reference(s, q, lens, lists)
    check(call(s, q, lens, lists, 75), ref, bound)
    check(s.pool.decode(0, q.cuda(), i32(lens), page_table=s.pool.page_table[:3].contiguous()), ref, bound)


def test_many_rows():
    lens = [int(x) for x in np.random.default_rng(10).integers(0, 300, 900)]
    s = Sessions(lens, 4, 1, 64, "bf16", seed=10)
    q = s.normal(900, 4, 64)
    lists = random_lists(np.random.default_rng(11), lens, 1, 8)
    check(call(s, q, lens, lists, 8), *reference(s, q, lens, lists))


@pytest.mark.parametrize("lens,hkv,width", [([9000], 1, 16), ([9000], 1, 17), ([9000], 1, 500), ([9000, 8000], 2, 64),
                                            ([2000] * 40, 4, 64), ([700] * 70, 4, 32)])
def test_splits(lens, hkv, width):
    """Lists in one part, in several, and in as many as there are pages to give away; parts past a
    short list's end."""
    s = Sessions(lens, 2 * hkv, hkv, 64, "f32", seed=17)
    q = s.normal(len(lens), 2 * hkv, 64)
    lists = random_lists(np.random.default_rng(18), lens, hkv, width)
    lists[0] = [sorted(np.random.default_rng(g).permutation(pages_for(lens[0]))[:width].tolist()) for g in range(hkv)]
    lists[-1][0] = lists[-1][0][:1]
    check(call(s, q, lens, lists, width), *reference(s, q, lens, lists))


def test_results_do_not_depend_on_where_pages_sit():
    lens = [3000]
    outs = []
    for spare in (0, 50):
        s = Sessions(lens, 8, 2, 128, "bf16", seed=12, spare=spare)
        s.k[0], s.v[0] = (torch.randn(1, 3000, 2, 128, generator=torch.Generator().manual_seed(i)).bfloat16() for i in (1, 2))
        s.pool.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())
        q = torch.randn(1, 8, 128, generator=torch.Generator().manual_seed(3)).bfloat16()
        outs.append(call(s, q, lens, [[list(range(0, 180, 2)), list(range(60))]], 90))
    assert torch.equal(*outs)


def step(s, q, lens, width, layer=0):
    """The reference of a sparse decode step: lists by the definition, then the attention."""
    lists = []
    for b, n in enumerate(lens):
        sc = scores(q[b], *page_bounds(s.k[b][layer], n))
        lists.append([choose(list(sc[g]), width, 1, 2) for g in range(s.hkv)])
    return reference(s, q, lens, lists, layer=layer)


def test_serving_loop():
    """Prompts with bounds, then steps that append a token, renew its page's bounds, pick and attend;
    one session is evicted and resumed in between, and its bounds with it."""
    lens = [700, 450, 1000]
    s = Sessions(lens, 8, 2, 128, "bf16", seed=13, layers=2, cold=200, spare=60, stride=80, max_sessions=4)
    p = s.pool
    p.set_bounds(True)
    p.update_bounds(0, 2, i32(lens))
    sids = i32([0, 1, 2])
    for turn in range(20):
        if turn == 9:
            p.evict(1)
            p.create_session(64)
            p.resume(1)
        for b in range(3):
            p.extend(b, lens[b] + 1)
            s.k[b] = torch.cat([s.k[b], s.normal(2, 1, 2, 128)], dim=1)
            s.v[b] = torch.cat([s.v[b], s.normal(2, 1, 2, 128)], dim=1)
        table = p.gather_table(sids)
        k = torch.stack([s.k[b][:, lens[b]] for b in range(3)], dim=1).cuda()
        v = torch.stack([s.v[b][:, lens[b]] for b in range(3)], dim=1).cuda()
        p.append_tokens_table(0, table, i32([0, 1, 2]), i32(lens), k.contiguous(), v.contiguous())
        before, lens = lens, [n + 1 for n in lens]
        p.update_bounds(0, 2, i32(lens), starts=i32(before), page_table=table)
        for layer in range(2):
            q = s.normal(3, 8, 128)
            picks, counts = p.select_pages(layer, q.cuda(), i32(lens), 12, page_table=table)
            out = p.sparse_decode(layer, q.cuda(), i32(lens), picks, counts, page_table=table)
            check(out, *step(s, q, lens, 12, layer), "turn %d layer %d" % (turn, layer))


def test_captured_steps():
    """A step (append, bounds, choice, attention) captured once and replayed while lengths, queries and
    the table change, with eager steps in between; two graphs share no workspace."""
    lens = [200, 330]
    s = Sessions(lens, 8, 2, 64, "bf16", seed=14, spare=80, stride=64)
    p = s.pool
    p.set_bounds(True)
    p.update_bounds(0, 1, i32(lens))
    for b in range(2):
        p.extend(b, lens[b] + 20)
    table = p.gather_table(i32([0, 1]))
    at, now, rows = i32(lens), i32([n + 1 for n in lens]), i32([0, 1])
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def run():
        p.append_tokens_table(0, table, rows, at, k, v)
        p.update_bounds(0, 1, now, starts=at, page_table=table)
        picks, counts = p.select_pages(0, q, now, 7, page_table=table)
        return p.sparse_decode(0, q, now, picks, counts, page_table=table)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        run()
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(run())
            graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(8):
        for b in range(2):
            s.k[b] = torch.cat([s.k[b][:, :lens[b]], s.normal(1, 1, 2, 64)], dim=1)
            s.v[b] = torch.cat([s.v[b][:, :lens[b]], s.normal(1, 1, 2, 64)], dim=1)
        new_q = s.normal(2, 8, 64)
        q.copy_(new_q)
        k.copy_(torch.stack([s.k[b][:, lens[b]] for b in range(2)], dim=1))
        v.copy_(torch.stack([s.v[b][:, lens[b]] for b in range(2)], dim=1))
        at.copy_(i32(lens))
        lens = [n + 1 for n in lens]
        now.copy_(i32(lens))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0].replay()
            graphs[1].replay()
        torch.cuda.synchronize()
        ref = step(s, new_q, lens, 7)
        for out in outs:
            check(out, *ref, "turn %d" % turn)
        assert torch.equal(run(), outs[0])
        torch.cuda.synchronize()


def test_profiling_counts_the_kernels():
    s = Sessions([9000, 300], 4, 1, 64, "bf16", seed=21, spare=40, max_sessions=4)
    p, q = s.pool, s.normal(2, 4, 64).cuda()
    lens = i32(s.lens)
    p.set_bounds(True)
    kv.kv_pool_set_profiling(p.handle, True)
    p.update_bounds(0, 1, lens)
    picks, counts = p.select_pages(0, q, lens, 40)                                  # a table of over 512 pages a row
    p.select_pages(0, q, i32([300, 300]), 4, page_table=p.page_table[1].repeat(2, 1)[:, :30].contiguous())
    p.sparse_decode(0, q, lens, picks, counts)                                      # in parts
    p.sparse_decode(0, q, lens, picks[:, :, :4].contiguous())                       # in one
    p.fork([1, 1], [300, 20])
    torch.cuda.synchronize()
    for kernel, launches in ((kv.KV_KERNEL_BOUNDS, 1), (kv.KV_KERNEL_PAGE_SCORES, 1), (kv.KV_KERNEL_PAGE_PICK, 2),
                             (kv.KV_KERNEL_SPARSE, 2), (kv.KV_KERNEL_SPARSE_MERGE, 1), (kv.KV_KERNEL_FORK_COPY, 1)):
        n, ms = kv.kv_pool_profile_read(p.handle, kernel)
        assert n == launches and ms > 0, (kernel, n)


def test_pages_and_records_past_32_bits():
    """A row on the last pages of a pool of 71 GB, whose records lie past 2 GiB as well."""
    from paper_2609_25782_amd.pool import HotColdPool
    hkv, d, n, pages = 16, 128, 330, 540_000
    assert pages * (hkv * 2 * d + 16) > 2 ** 31
    p = HotColdPool(1, hkv, d, "bf16", pages, 0, 2, 30)
    p.set_bounds(True)
    rng = np.random.default_rng(22)
    row = (pages - 1 - rng.permutation(5000)[:pages_for(n)]).astype(np.int32)
    row[0] = 0
    table = torch.from_numpy(np.pad(row, (0, 30 - len(row)), constant_values=-1)[None]).cuda()
    g = torch.Generator().manual_seed(22)
    k, v, q = (torch.randn(shape, generator=g).to(torch.bfloat16) for shape in ((n, hkv, d), (n, hkv, d), (1, 32, d)))
    positions = torch.arange(n, dtype=torch.int32, device="cuda")
    p.append_tokens_table(0, table, torch.zeros_like(positions), positions, k[None].cuda(), v[None].cuda())
    lens = i32([n])
    p.update_bounds(0, 1, lens, page_table=table)
    lo, hi, e = page_bounds(k, n)
    got = p.key_bounds(0, 1, i32(row.tolist()))[0].cpu().double().numpy()
    assert np.array_equal(got, values(lo, hi, e))
    picks, counts = p.select_pages(0, q.cuda(), lens, 7, page_table=table)
    want = [choose(list(x), 7, 1, 2) for x in scores(q[0], lo, hi, e)]
    assert picks[0].tolist() == want
    out, bound = attend_pages(q[0], k, v, n, want, d ** -0.5, "bf16")
    check(p.sparse_decode(0, q.cuda(), lens, picks, counts, page_table=table), out[None], bound[None])
    del p
    torch.cuda.empty_cache()


def test_two_streams_at_once():
    """Calls of two streams run side by side, each with its own workspace."""
    s = Sessions([4000] * 4, 8, 2, 128, "bf16", seed=15)
    s.pool.set_bounds(True)
    lens = i32([4000] * 4)
    s.pool.update_bounds(0, 1, lens)
    qs = [s.normal(4, 8, 128).cuda() for _ in range(2)]

    def one(q, stream=None):
        picks, counts = s.pool.select_pages(0, q, lens, 40, stream=stream)
        return s.pool.sparse_decode(0, q, lens, picks, counts, stream=stream)
    want = [one(q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = [one(q, st) for q, st in zip(qs, streams)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    s = Sessions([100], 4, 2, 64, "bf16", seed=16)
    p, q, lens = s.pool, s.normal(1, 4, 64).cuda(), i32([100])
    picks, counts = tensors([[[0, 1], [2]]], 3, 2)
    out, ws = torch.zeros_like(q), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    good = [p.handle, 0, q.data_ptr(), p.page_table.data_ptr(), p.stride, lens.data_ptr(), picks.data_ptr(),
            counts.data_ptr(), 3, 1, 4, 0.125, out.data_ptr(), ws.data_ptr(), ws.numel()]
    kv.paged_sparse_attention(*good)
    for i, bad in ((1, 1), (1, -1), (2, 0), (2, q.data_ptr() + 8), (3, 0), (4, 0), (4, 1 << 31), (5, 0), (6, 0), (8, 0),
                   (9, -1), (9, 8193), (10, 3), (10, 0), (10, 34), (12, 0), (12, out.data_ptr() + 8), (13, 0),
                   (13, ws.data_ptr() + 16), (14, 255)):
        args = list(good)
        args[i] = bad
        with pytest.raises(kv.KVError) as e:
            kv.paged_sparse_attention(*args)
        assert e.value.status == kv.KV_ERR_INVALID, i
    args = list(good)
    args[9] = 0
    kv.paged_sparse_attention(*args)          # no rows
    with pytest.raises(AssertionError):
        p.sparse_decode(0, q, lens, picks.long(), counts)
    with pytest.raises(AssertionError):
        p.sparse_decode(0, q, lens, picks[:, :1].contiguous(), counts)


def test_captured_steps_have_workspaces_of_their_own():
    """Two graphs whose calls need workspaces (scores of a wide table, partial results of a long list), with
    queries of their own, replayed side by side and between eager calls."""
    lens = [9000, 7000]
    s = Sessions(lens, 4, 1, 128, "bf16", seed=23)
    p = s.pool
    width, n = 60, i32(lens)
    assert kv.paged_select_workspace_bytes(p.handle, 2, p.stride, width) > 256
    assert kv.paged_sparse_workspace_bytes(p.handle, 2, 4, width) > 256
    p.set_bounds(True)
    p.update_bounds(0, 1, n)
    qs = [torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3)]

    def run(q):
        picks, counts = p.select_pages(0, q, n, width)
        return picks, p.sparse_decode(0, q, n, picks, counts)
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for q, st in zip(qs, streams):
        with torch.cuda.stream(st):
            run(q)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                outs.append(run(q))
            graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(6):
        for q in qs:
            q.copy_(s.normal(2, 4, 128))
        want = [run(q) for q in qs]
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        eager = run(qs[2])
        torch.cuda.synchronize()
        for got, ref in zip(outs + [eager], want):
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]), turn
    for q, out in zip(qs, outs):
        lists = []
        for b, m in enumerate(lens):
            sc = scores(q[b].cpu(), *page_bounds(s.k[b][0], m))
            lists.append([choose(list(sc[0]), width, 1, 2)])
        check(out[1], *reference(s, q.cpu(), lens, lists))


def test_two_streams_have_workspaces_of_their_own():
    s = Sessions([9000] * 2, 4, 1, 128, "f32", seed=24)
    p, n, width = s.pool, i32([9000] * 2), 60
    assert kv.paged_select_workspace_bytes(p.handle, 2, p.stride, width) > 256
    assert kv.paged_sparse_workspace_bytes(p.handle, 2, 4, width) > 256
    p.set_bounds(True)
    p.update_bounds(0, 1, n)
    qs = [s.normal(2, 4, 128).cuda() for _ in range(2)]

    def one(q, stream=None):
        picks, counts = p.select_pages(0, q, n, width, stream=stream)
        return picks, p.sparse_decode(0, q, n, picks, counts, stream=stream)
    want = [one(q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = [one(q, st) for q, st in zip(qs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_spilled_pages_in_host_memory(dtype):
    """Bounds, choice and attention over pages that lie in pinned host memory."""
    from paper_2609_25782_amd.pool import HotColdPool
    lens = [300, 16 * 20]
    s = Sessions(lens, 8, 2, 128, dtype, seed=25)
    p = s.pool = HotColdPool(1, 2, 128, dtype, 44, 44, 3, 24, cold_location="host")
    for b in range(2):
        p.create_session(lens[b])
        p.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    p.set_spill(True)
    p.evict([0, 1])
    p.resume_lazy([0, 1])
    assert p.promote(7) == 7
    p.set_bounds(True)
    p.update_bounds(0, 1, i32(lens))
    q = s.normal(2, 8, 128)
    picks, counts = p.select_pages(0, q.cuda(), i32(lens), 6)
    lists = [[choose(list(x), 6, 1, 2) for x in scores(q[b], *page_bounds(s.k[b][0], lens[b]))] for b in range(2)]
    assert picks.tolist() == lists
    check(p.sparse_decode(0, q.cuda(), i32(lens), picks, counts), *reference(s, q, lens, lists))
    entries = p.page_table[1, :20].contiguous()
    assert (entries & kv.KV_PAGE_COLD != 0).all()
    assert np.array_equal(p.key_bounds(0, 1, entries)[0].cpu().double().numpy(), values(*page_bounds(s.k[1][0], 320)))
    all_pages = [[list(range(pages_for(n)))] * 2 for n in lens]
    check(call(s, q, lens, all_pages, 20), *reference(s, q, lens, all_pages))
