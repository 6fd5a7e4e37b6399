"""Key bounds of pages (kv_update_bounds, kv_read_bounds) and the choice of pages by them
(paged_select_pages): whole numbers, equal to the definition."""

import numpy as np
import pytest
import torch

from chunk_reference import PAGE, TORCH, Sessions, i32, pages_for
from paper_2609_25782_amd import hotcold_kv as kv
from sparse_reference import choose, page_bounds, scores, values

pytestmark = pytest.mark.gpu

SHAPES = [(8, 1, 128, "bf16"), (32, 4, 128, "bf16"), (6, 2, 64, "bf16"), (16, 1, 64, "bf16"), (3, 3, 128, "bf16"),
          (16, 16, 64, "bf16"), (4, 1, 64, "f32"), (10, 2, 128, "f32"), (8, 8, 128, "f32")]
LENS = [1, 15, 16, 17, 200, 0, 333]


def spread(s, seed):
    """Keys of very different sizes: channels from 2^-6 to 2^6, tokens that stand out."""
    g = torch.Generator().manual_seed(seed)
    for b, n in enumerate(s.lens):
        if n == 0:
            continue
        size = torch.exp2(torch.randint(-6, 7, (s.d,), generator=g).float())
        k = s.k[b].float() * size
        k[:, torch.randint(0, n, (1 + n // 50,), generator=g)] *= 8
        s.k[b] = k.to(TORCH[s.dtype])
        s.pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    return s


def expected(s, lens=None):
    """[layer][session] -> (lo, hi, e)."""
    lens = s.lens if lens is None else lens
    return [[page_bounds(s.k[b][layer], n) for b, n in enumerate(lens)] for layer in range(len(s.k[0]))]


def read(s, b, layers=1, first=0, upto=None):
    pages = i32(s.pages[b][first:pages_for(s.lens[b]) if upto is None else upto])
    return s.pool.key_bounds(0, layers, pages).cpu().double().numpy()


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_bounds_match_the_definition(hq, hkv, d, dtype):
    s = spread(Sessions(LENS, hq, hkv, d, dtype, seed=1, layers=2), 2)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 2, i32(LENS))
    want = expected(s)
    for b, n in enumerate(LENS):
        got = read(s, b, layers=2)
        for layer in range(2):
            assert np.array_equal(got[layer], values(*want[layer][b])), (b, layer)
            low, high = values(*want[layer][b])[:, :, 0], values(*want[layer][b])[:, :, 1]
            k = s.k[b][layer].double().numpy()
            for p in range(pages_for(n)):      # they are bounds
                part = k[p * PAGE:min(n, (p + 1) * PAGE)]
                assert (low[p] <= part.min(axis=0)).all() and (high[p] >= part.max(axis=0)).all()


def test_ranges_of_tokens():
    """Only pages with tokens of [starts, lens) change, and a page's earlier tokens stay in."""
    s = Sessions([100, 100, 100, 100, 40], 8, 2, 128, "bf16", seed=3)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([37, 100, 16, 100, 1000000]), starts=i32([20, 96, -5, 100, 0]))
    zero = np.zeros((2, 2, 128))

    def page(b, upto, p):
        return values(*(x[p:p + 1] for x in page_bounds(s.k[b][0], upto)))[0]
    for b, upto, pages in ((0, 37, [1, 2]), (1, 100, [6]), (2, 16, [0]), (3, 0, []), (4, 0, [])):
        got = read(s, b)[0]
        for p in range(pages_for(s.lens[b])):
            assert np.array_equal(got[p], page(b, upto, p) if p in pages else zero), (b, p)


def test_entries_that_name_no_page():
    s = Sessions([90, 33], 8, 2, 64, "bf16", seed=4, cold=4)
    s.pool.set_bounds(True)
    table = s.pool.page_table[:2].clone()
    table[0, 1], table[0, 2], table[0, 3] = -1, 1 << 20, (1 << 30) | 2     # spill is off
    s.pool.update_bounds(0, 1, i32([90, 33]), page_table=table)
    got = read(s, 0)[0]
    want = values(*page_bounds(s.k[0][0], 90))
    want[1:4] = 0
    assert np.array_equal(got, want)
    named = s.pool.key_bounds(0, 1, i32([-1, 1 << 20, (1 << 30) | 4, (1 << 29) | 1, (1 << 30) | 3]))
    assert torch.isnan(named[0, :4]).all() and (named[0, 4] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_any_size(dtype):
    """Zeros, infinities, NaN, and values past both ends of the powers."""
    s = Sessions([16 * 9], 4, 2, 64, dtype, seed=5)
    k = s.k[0][0]
    k[0:16] = 0
    k[16:32, 0, 3] = float("inf")
    k[32:48, 1, 5] = float("-inf")
    k[50, 0, 7] = float("nan")
    k[51, 1, 9] = -torch.tensor(float("nan")) if dtype == "f32" else torch.copysign(torch.tensor(float("nan")), torch.tensor(-1.0))
    k[64:80] *= 2.0 ** 60
    k[80:96] *= 2.0 ** -70
    k[96:112] = -0.0
    k[112:128, :, 1:] = 0           # one channel alone
    k[128:144, 0] = 127.0           # the largest that a power of 0 holds
    s.pool.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([144]))
    lo, hi, e = page_bounds(k, 144)
    assert e[8, 0] == 0 and e[4, 0] > 50 - 2 and e[5, 0] < -50 + 2 and e[1, 0] == 50 and e[0, 0] == -7
    assert np.array_equal(read(s, 0)[0], values(lo, hi, e))


def picks_of(s, q, lens, width, first, recent, want, **kw):
    picks, counts = s.pool.select_pages(0, q.cuda(), i32(lens), width, first=first, recent=recent, **kw)
    picks, counts = picks.cpu().numpy(), counts.cpu().numpy()
    for b in range(len(lens)):
        for g in range(s.hkv):
            exp = want[b][g]
            assert counts[b, g] == len(exp), (b, g)
            assert picks[b, g].tolist() == exp + [-1] * (width - len(exp)), (b, g)


def choices(s, q, lens, width, first, recent):
    out = []
    for b, n in enumerate(lens):
        sc = scores(q[b], *page_bounds(s.k[b][0], n))
        out.append([choose(list(sc[g]), width, first, recent) for g in range(s.hkv)])
    return out


@pytest.mark.parametrize("width,first,recent", [(1, 0, 0), (1, 0, 1), (5, 2, 3), (9, 1, 2), (16, 0, 0), (40, 3, 1)])
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_picks_match_the_definition(hq, hkv, d, dtype, width, first, recent):
    lens = [1, 0, 16, 150, 333, 16 * 40, 16 * 41, 1000]
    s = spread(Sessions(lens, hq, hkv, d, dtype, seed=6), 7)
    q = s.normal(len(lens), hq, d)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32(lens))
    picks_of(s, q, lens, width, first, recent, choices(s, q, lens, width, first, recent))


@pytest.mark.parametrize("tokens,stride", [(16 * 512, 512), (16 * 1024, 1024), (16 * 1025, 1025), (16 * 4096, 4096), (16 * 5000, 5000),
                                           (70001, 20000)])
def test_long_rows(tokens, stride):
    """Both sides of every size at which the choice holds its keys in another way."""
    s = Sessions([tokens, 40], 2, 1, 64, "bf16", seed=8, stride=stride)
    q = s.normal(2, 2, 64)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([tokens, 40]))
    for width in (3, 257):
        picks_of(s, q, [tokens, 40], width, 1, 2, choices(s, q, [tokens, 40], width, 1, 2))


def test_ties_go_to_the_lowest_pages():
    """Equal pages: the choice is by page number; pages that stand out come first."""
    s = Sessions([16 * 300], 4, 2, 64, "bf16", seed=9)
    s.k[0][0] = s.k[0][0, :1]
    s.k[0][0, 16 * 200:16 * 201] = s.normal(1, 2, 64)
    q = s.normal(1, 4, 64)
    s.pool.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([4800]))
    for width, first, recent in ((1, 0, 0), (64, 0, 0), (65, 1, 1), (299, 0, 0)):
        picks_of(s, q, [4800], width, first, recent, choices(s, q, [4800], width, first, recent))
    zero = torch.zeros_like(q)
    picks_of(s, zero, [4800], 70, 0, 0, [[list(range(70))] * 2])


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 2.0 ** 80, 2.0 ** -80])
def test_queries_of_any_size(value):
    s = Sessions([16 * 60], 4, 2, 128, "f32", seed=10)
    q = s.normal(1, 4, 128)
    if value == value and abs(value) != float("inf"):
        q = q * value
    else:
        q[0, 1, 17] = value
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([960]))
    picks_of(s, q, [960], 11, 1, 1, choices(s, q, [960], 11, 1, 1))


def test_pages_outside_the_pools_are_picked_first():
    s = Sessions([16 * 50], 8, 2, 64, "bf16", seed=11)
    q = s.normal(1, 8, 64)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([800]))
    table = s.pool.page_table[:1].clone()
    table[0, 20], table[0, 33] = -1, 1 << 25
    sc = scores(q[0], *page_bounds(s.k[0][0], 800))
    sc[:, [20, 33]] = np.inf
    for width in (1, 2, 7):
        picks_of(s, q, [800], width, 0, 0, [[choose(list(sc[g]), width, 0, 0) for g in range(2)]], page_table=table)


def test_lengths_that_do_not_fit_pick_nothing():
    s = Sessions([200, 200, 200, 200], 4, 2, 64, "bf16", seed=12)
    q = s.normal(4, 4, 64)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([200] * 4))
    lens = [-1, 0, 16 * s.pool.stride + 1, 200]
    want = [[[], []]] * 3 + choices(s, q, [0, 0, 0, 200], 5, 1, 1)[3:]
    picks_of(s, q, lens, 5, 1, 1, want)


def test_bounds_go_with_evicted_and_resumed_pages():
    """Eviction, other sessions' use of the pages, resume: the bounds are where the pages are."""
    for host in ("device", "host"):
        lens = [150, 90]
        s = Sessions(lens, 8, 2, 64, "bf16", seed=13, layers=2, cold=40, max_sessions=4)
        if host == "host":
            from paper_2609_25782_amd.pool import HotColdPool
            s.pool = HotColdPool(2, 2, 64, "bf16", 40, 40, 4, 16, cold_location="host")
            for b, n in enumerate(lens):
                s.pool.create_session(n)
                s.pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
        p = s.pool
        p.set_bounds(True)
        p.update_bounds(0, 2, i32(lens))
        want = [values(*page_bounds(s.k[0][layer], 150)) for layer in range(2)]
        p.evict(0)
        cold = i32([c | kv.KV_PAGE_COLD for c in p.info(0)[3]])
        got = p.key_bounds(0, 2, cold).cpu().double().numpy()
        assert all(np.array_equal(got[layer], want[layer]) for layer in range(2))
        other = p.create_session(16)         # takes a page that the resume then cannot have
        p.resume(0)
        got = p.key_bounds(0, 2, i32(p.info(0)[2])).cpu().double().numpy()
        assert all(np.array_equal(got[layer], want[layer]) for layer in range(2))
        p.destroy_session(other)


@pytest.mark.parametrize("pages", [100, 128, 129, 300])
def test_bounds_go_with_lists_of_any_length(pages):
    """Copy lists in the kernels' arguments and uploaded ones, with and without profiling events."""
    n = 16 * pages
    s = Sessions([n], 4, 2, 64, "bf16", seed=18, cold=pages, spare=pages, max_sessions=2)
    p = s.pool
    p.set_bounds(True)
    lens = i32([n])
    p.update_bounds(0, 1, lens)
    want = read(s, 0)
    for prof in (False, True):
        kv.kv_pool_set_profiling(p.handle, prof)
        p.evict(0)
        p.key_bounds(0, 1, i32([0]))
        other = p.create_session(16 * 7)        # other pages for the resume
        p.resume(0)
        s.pages = [p.info(0)[2]]
        assert np.array_equal(read(s, 0), want)
        p.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())     # so that the next eviction copies again
        p.destroy_session(other)


def test_bounds_go_with_a_captured_eviction():
    """Replays after other calls have used the pool's copy lists move the same records."""
    s = Sessions([200, 300, 100], 4, 2, 64, "bf16", seed=19, cold=60, max_sessions=6, spare=60)
    p = s.pool
    p.set_bounds(True)
    lens = i32([200, 300, 100])
    p.update_bounds(0, 1, lens)
    want = read(s, 1)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p.evict(1, stream=st)
    cold = i32([c | kv.KV_PAGE_COLD for c in p.info(1)[3]])
    saved = p.bounds.clone()
    for turn in range(3):
        p.bounds.copy_(saved)               # the session's old pages are free: resumes below may take them
        p.bounds.view(-1)[p.num_hot_pages * (2 * 2 * 64 + 16):] = 0
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(p.key_bounds(0, 1, cold).cpu().double().numpy(), want), turn
        p.evict(0), p.resume(0)                 # eager calls between the replays
        p.evict(2), p.resume(2)
        torch.cuda.synchronize()


def test_spilled_pages_have_bounds():
    s = Sessions([200], 8, 2, 64, "bf16", seed=14, cold=40)
    p = s.pool
    p.set_spill(True)
    p.set_bounds(True)
    p.evict(0)
    p.resume_lazy(0)
    p.update_bounds(0, 1, i32([200]))       # of the pages where they are: in the cold tier
    want = values(*page_bounds(s.k[0][0], 200))
    cold = i32([c | kv.KV_PAGE_COLD for c in p.info(0)[3]])
    assert np.array_equal(p.key_bounds(0, 1, cold)[0].cpu().double().numpy(), want)
    q = s.normal(1, 8, 64)
    picks_of(s, q, [200], 4, 1, 1, choices(s, q, [200], 4, 1, 1))
    assert p.promote(5) == 5
    s.pages = [p.info(0)[2][:5]]
    assert np.array_equal(read(s, 0, upto=5)[0], want[:5])
    picks_of(s, q, [200], 4, 1, 1, choices(s, q, [200], 4, 1, 1))


def test_layers_are_apart():
    s = Sessions([500], 4, 2, 64, "bf16", seed=15, layers=3)
    s.pool.set_bounds(True)
    s.pool.update_bounds(1, 2, i32([500]))
    got = read(s, 0, layers=3)
    assert (got[0] == 0).all()
    for layer in (1, 2):
        assert np.array_equal(got[layer], values(*page_bounds(s.k[0][layer], 500)))
    q = s.normal(1, 4, 64)
    picks, _ = s.pool.select_pages(2, q.cuda(), i32([500]), 6, first=0, recent=0)
    sc = scores(q[0], *page_bounds(s.k[0][2], 500))
    assert [picks[0, g].tolist() for g in range(2)] == [choose(list(sc[g]), 6, 0, 0) for g in range(2)]


def test_many_rows():
    lens = [int(x) for x in np.random.default_rng(16).integers(0, 400, 700)]
    s = Sessions(lens, 2, 1, 64, "bf16", seed=16)
    q = s.normal(700, 2, 64)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32(lens))
    picks_of(s, q, lens, 6, 1, 1, choices(s, q, lens, 6, 1, 1))


def test_refusals():
    s = Sessions([100], 4, 2, 64, "bf16", seed=17)
    q, lens = s.normal(1, 4, 64).cuda(), i32([100])
    p = s.pool
    with pytest.raises(kv.KVError):
        p.update_bounds(0, 1, lens)
    with pytest.raises(kv.KVError):
        p.select_pages(0, q, lens, 4)
    with pytest.raises(kv.KVError):
        p.key_bounds(0, 1, i32([0]))
    need = kv.kv_bounds_bytes(p.desc)
    buf = torch.zeros(need + 512, dtype=torch.uint8, device="cuda")
    for ptr, n in ((buf.data_ptr() + 16, need), (buf.data_ptr(), need - 1)):
        with pytest.raises(kv.KVError):
            kv.kv_pool_set_bounds(p.handle, ptr, n)
    p.set_bounds(True)
    for call in (lambda: p.update_bounds(0, 2, lens), lambda: p.update_bounds(-1, 1, lens),
                 lambda: p.update_bounds(0, 0, lens), lambda: p.key_bounds(1, 1, i32([0])),
                 lambda: p.select_pages(1, q, lens, 4), lambda: p.select_pages(0, q, lens, 2, first=1, recent=2),
                 lambda: p.select_pages(0, q, lens, 4, first=-1), lambda: p.select_pages(0, q, lens, 4, recent=-1),
                 lambda: p.select_pages(0, q, lens, 0, first=0, recent=0),
                 lambda: p.select_pages(0, torch.zeros(1, 3, 64, dtype=q.dtype, device="cuda"), lens, 4),
                 lambda: p.select_pages(0, torch.zeros(1, 34, 64, dtype=q.dtype, device="cuda"), lens, 4)):
        with pytest.raises(kv.KVError) as e:
            call()
        assert e.value.status == kv.KV_ERR_INVALID
    table, picks = p.page_table, torch.zeros(1, 2, 3, dtype=torch.int32, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    good = [p.handle, 0, q.data_ptr(), table.data_ptr(), table.shape[1], lens.data_ptr(), 1, 4, 3, 1, 1,
            picks.data_ptr(), picks.data_ptr(), ws.data_ptr(), ws.numel()]
    kv.paged_select_pages(*good)
    for i, bad in ((2, 0), (2, q.data_ptr() + 2), (3, 0), (4, 0), (4, 1 << 31), (5, 0), (6, -1), (6, 8193), (11, 0),
                   (12, 0), (13, 0), (13, ws.data_ptr() + 128), (14, 255)):
        args = list(good)
        args[i] = bad
        with pytest.raises(kv.KVError) as e:
            kv.paged_select_pages(*args)
        assert e.value.status == kv.KV_ERR_INVALID, i
    p.set_bounds(False)
    with pytest.raises(kv.KVError):
        p.update_bounds(0, 1, lens)


# -- bounds that are set while a page has a cold copy already ------------------


def clean_sessions(n, where="device", dtype="bf16", sessions=1, seed=20, room=None):
    """Sessions of n tokens each with valid cold copies of all pages, resident: set up before the pool
    keeps bounds, as a cache that was running already has them."""
    from paper_2609_25782_amd.pool import HotColdPool
    pages = pages_for(n)
    s = Sessions([n] * sessions, 4, 2, 64, dtype, seed=seed, layers=2, max_sessions=sessions + 4)
    if room is None:
        room = sessions * pages + pages
    p = s.pool = HotColdPool(2, 2, 64, dtype, room, 2 * sessions * pages + 8, sessions + 4, pages + 2, cold_location=where)
    for b in range(sessions):
        p.create_session(n)
        p.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    for b in range(sessions):
        p.evict(b)
    for b in range(sessions):
        p.resume(b)
    p.set_bounds(True)
    return s


def bounds_of(s, b, n):
    return np.stack([values(*page_bounds(s.k[b][layer], n)) for layer in range(2)])


def are(s, sid, want, cold=False):
    hot, copies = s.pool.info(sid)[2:]
    entries = [c | kv.KV_PAGE_COLD for c in copies] if cold else hot
    assert min(entries) >= 0
    got = s.pool.key_bounds(0, len(want), i32(entries)).cpu().double().numpy()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("where", ["device", "host"])
@pytest.mark.parametrize("pages", [5, 128, 129, 300])
@pytest.mark.parametrize("path", ["evict", "evict_pages", "victims"])
def test_bounds_of_pages_with_cold_copies_survive(path, pages, where):
    """An eviction that writes no page takes the bounds along all the same: of a session, of pages of a
    paused one, and of pages that make room for another session."""
    n = 16 * pages - 3
    s = clean_sessions(n, where, room=pages + 4)
    p, want = s.pool, bounds_of(s, 0, n)
    p.update_bounds(0, 2, i32([n]))
    are(s, 0, want)
    written = p.stats()["pages_to_cold"]
    if path == "evict":
        p.evict(0)
    else:
        p.pause(0)
        if path == "evict_pages":
            assert p.evict_pages(pages - 1) == pages - 1
            p.evict_pages(pages)
        else:
            p.destroy_session(p.create_session(16 * pages))
            assert p.stats()["lru_evicted_pages"] == pages - 4
            p.evict_pages(pages)
    assert p.stats()["pages_to_cold"] == written
    are(s, 0, want, cold=True)
    p.create_session(16)                      # a page that the resume then cannot have
    p.resume(0)
    are(s, 0, want)


def test_bounds_of_imported_pages_survive():
    n = 200
    s = clean_sessions(n)
    p, want = s.pool, bounds_of(s, 0, n)
    sid = p.import_cold(n, p.info(0)[3])
    p.destroy_session(0)
    p.resume(sid)
    lens = torch.zeros(p.max_sessions, dtype=torch.int32, device="cuda")
    lens[sid] = n
    p.update_bounds(0, 2, lens)
    for _ in range(2):
        p.evict(sid)
        p.resume(sid)
        are(s, sid, want)


def test_bounds_that_waited_for_a_resume_survive():
    """A page that was full before its bounds were renewed, evicted and resumed in between."""
    n = 16 * 6 + 9
    s = clean_sessions(n)
    p = s.pool
    p.update_bounds(0, 2, i32([n]))
    more = s.normal(2, 7, 2, 64), s.normal(2, 7, 2, 64)
    s.k[0] = torch.cat([s.k[0], more[0]], dim=1)
    p.extend(0, n + 7)
    p.write_tokens_layers(0, 0, n, more[0].cuda(), more[1].cuda())
    p.evict(0), p.resume(0)
    p.update_bounds(0, 2, i32([n + 7]), starts=i32([n]))
    want = bounds_of(s, 0, n + 7)
    are(s, 0, want)
    p.evict(0), p.resume(0)
    are(s, 0, want)


def test_bounds_of_promoted_pages_survive():
    n = 16 * 9
    s = clean_sessions(n)
    p, want = s.pool, bounds_of(s, 0, n)
    p.set_spill(True)
    p.evict(0)
    p.resume_lazy(0)
    assert p.promote(9) == 9
    p.update_bounds(0, 2, i32([n]))
    p.evict(0)
    p.resume_lazy(0)
    are(s, 0, want, cold=True)
    q = s.normal(1, 4, 64)
    picks_of(s, q, [n], 4, 1, 1, choices(s, q, [n], 4, 1, 1))
    assert p.promote(9) == 9
    are(s, 0, want)


def test_bounds_of_branches_that_share_cold_copies_survive():
    n = 16 * 5
    s = clean_sessions(n, room=20)
    p, want = s.pool, bounds_of(s, 0, n)
    p.update_bounds(0, 2, i32([n]))
    child = p.fork(0)
    assert p.info(child)[3] == p.info(0)[3]
    for order in ([child, 0], [0, child]):
        p.evict(order[0]), p.evict(order[1])
        p.resume(order)
        are(s, 0, want), are(s, child, want)
    p.evict([0, child])
    p.resume([child, 0])
    are(s, 0, want), are(s, child, want)
    twig = p.fork(child)                      # of pages whose records came back from the cold tier
    are(s, twig, want)


def test_a_branch_carries_renewed_bounds_to_the_shared_copies():
    """The branch alone is evicted after its parent is gone: what it took over is what comes back."""
    n = 16 * 5
    s = clean_sessions(n)
    p, want = s.pool, bounds_of(s, 0, n)
    p.update_bounds(0, 2, i32([n]))
    child = p.fork(0)
    p.destroy_session(0)
    p.evict(child), p.resume(child)
    are(s, child, want)


@pytest.mark.parametrize("together", [False, True])
@pytest.mark.parametrize("n", [80, 16 * 150])
def test_old_bounds_do_not_replace_renewed_ones(n, together):
    """Two sessions with the same cold pages, of which one had its bounds renewed: the other's eviction
    leaves the cold record as it is, before, after or in the same call."""
    s = clean_sessions(n, room=3 * pages_for(n))
    p, want = s.pool, bounds_of(s, 0, n)
    twin = p.import_cold(n, p.info(0)[3])
    p.resume(twin)
    p.update_bounds(0, 2, i32([n]))
    for order in ([0, twin], [twin, 0]):
        if together:
            p.evict(order)
        else:
            for sid in order:
                p.evict(sid)
        are(s, 0, want, cold=True)
        p.resume([0, twin])
        are(s, 0, want), are(s, twin, want)
        at = i32(p.info(twin)[2]).long()      # the twin's records grow old again
        record = 2 * 2 * 64 + 16
        flat = p.bounds[:2 * record * (p.num_hot_pages + p.num_cold_pages)].view(2, -1, record)
        flat[:, at] = 0
        p.update_bounds(0, 2, i32([n]))


def test_several_sessions_renew_the_same_cold_pages_at_once():
    n = 16 * 140
    s = clean_sessions(n, room=4 * 140)
    p, want = s.pool, bounds_of(s, 0, n)
    others = [p.import_cold(n, p.info(0)[3]) for _ in range(2)]
    p.resume(others)
    lens = torch.zeros(p.max_sessions, dtype=torch.int32, device="cuda")
    lens[[0] + others] = n
    p.update_bounds(0, 2, lens)
    p.evict([others[1], 0, others[0]])
    are(s, 0, want, cold=True)
    p.resume([0] + others)
    for sid in [0] + others:
        are(s, sid, want)


@pytest.mark.parametrize("pages", [6, 300])
def test_a_captured_eviction_of_clean_pages_takes_their_bounds(pages):
    """Replays after other calls have used the pool's copy lists."""
    n = 16 * pages
    s = clean_sessions(n, sessions=3, room=4 * pages)
    p = s.pool
    p.update_bounds(0, 2, i32([n] * 3))
    want = bounds_of(s, 1, n)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p.evict(1, stream=st)
    saved = p.bounds.clone()
    cold = i32(p.info(1)[3]).long() + p.num_hot_pages
    record = 2 * 2 * 64 + 16
    for turn in range(3):
        p.bounds.copy_(saved)               # the session's old pages are free: resumes below may take them
        p.bounds[:2 * record * (p.num_hot_pages + p.num_cold_pages)].view(2, -1, record)[:, cold] = 0
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        are(s, 1, want, cold=True)
        p.evict(0), p.resume(0)                 # eager calls between the replays
        p.evict(2), p.resume(2)
        torch.cuda.synchronize()


def test_evictions_without_bounds_leave_the_buffer_alone():
    n = 16 * 4
    s = clean_sessions(n)
    p = s.pool
    p.update_bounds(0, 2, i32([n]))
    buf = p.bounds
    p.set_bounds(False)
    before = buf.clone()
    p.evict(0), p.resume(0)
    torch.cuda.synchronize()
    assert torch.equal(buf, before)


# -- the choice of tables of more than 512 pages a row: scores and choice in kernels of their own -------


def wide(s, rows, stride=600):
    """The first rows of the pool's table in one of `stride` pages a row; entries past a row's end name
    page 0 of the pool, whose keys must not matter."""
    table = torch.zeros((rows, stride), dtype=torch.int32, device="cuda")
    own = s.pool.page_table[:rows]
    for b in range(rows):
        n = pages_for(s.lens[b])
        table[b, :n] = own[b, :n]
    return table


@pytest.mark.parametrize("width,first,recent", [(1, 0, 0), (5, 2, 3), (9, 1, 2), (40, 3, 1)])
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES + [(16, 8, 64, "bf16"), (32, 16, 128, "bf16"), (6, 6, 64, "f32"),
                                                     (16, 16, 128, "f32"), (32, 2, 128, "bf16")])
def test_picks_of_wide_tables_match_the_definition(hq, hkv, d, dtype, width, first, recent):
    """Every head layout and type, rows shorter than a block's turn and longer ones."""
    lens = [1, 0, 16, 150, 333, 16 * 40, 16 * 41, 1000, 16 * 130 + 5]
    s = spread(Sessions(lens, hq, hkv, d, dtype, seed=21), 22)
    q = s.normal(len(lens), hq, d)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32(lens))
    assert kv.paged_select_workspace_bytes(s.pool.handle, len(lens), 600, width) > 256
    picks_of(s, q, lens, width, first, recent, choices(s, q, lens, width, first, recent), page_table=wide(s, len(lens)))


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 4, 128, "bf16"), (2, 2, 64, "f32"), (3, 3, 64, "bf16")])
def test_wide_tables_of_many_rows(hq, hkv, d, dtype):
    """So many rows that a block goes on to further pages of its row, some rows far longer than others."""
    rng = np.random.default_rng(23)
    lens = [int(x) for x in rng.integers(0, 120, 520)]
    lens[7], lens[300], lens[519] = 16 * 700, 16 * 1000 + 3, 16 * 257
    s = Sessions(lens, hq, hkv, d, dtype, seed=23)
    q = s.normal(len(lens), hq, d)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32(lens))
    assert s.pool.stride > 512
    picks_of(s, q, lens, 5, 1, 1, choices(s, q, lens, 5, 1, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wide_tables_with_entries_that_name_no_page(dtype):
    s = Sessions([16 * 50, 16 * 200], 8, 2, 64, dtype, seed=24)
    q = s.normal(2, 8, 64)
    lens = [800, 3200]
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32(lens))
    table = wide(s, 2)
    bad = [[20, 33], [0, 64, 199]]
    sc = [scores(q[b], *page_bounds(s.k[b][0], n)) for b, n in enumerate(lens)]
    for b, pages in enumerate(bad):
        table[b, pages] = i32([-1, 1 << 25, (1 << 30) | 3][:len(pages)])
        sc[b][:, pages] = np.inf
    for width in (1, 2, 7):
        want = [[choose(list(sc[b][g]), width, 0, 0) for g in range(2)] for b in range(2)]
        picks_of(s, q, lens, width, 0, 0, want, page_table=table)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 2.0 ** 80, 2.0 ** -80])
@pytest.mark.parametrize("dtype,d", [("f32", 128), ("bf16", 64)])
def test_wide_tables_with_queries_of_any_size(dtype, d, value):
    s = Sessions([16 * 60], 4, 2, d, dtype, seed=25)
    q = s.normal(1, 4, d)
    if value == value and abs(value) != float("inf"):
        q = q * value
    else:
        q[0, 1, 17] = value
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([960]))
    picks_of(s, q, [960], 11, 1, 1, choices(s, q, [960], 11, 1, 1), page_table=wide(s, 1))


def test_ties_of_wide_tables_go_to_the_lowest_pages():
    s = Sessions([16 * 300], 4, 2, 128, "bf16", seed=26)
    s.k[0][0] = s.k[0][0, :1]
    s.k[0][0, 16 * 200:16 * 201] = s.normal(1, 2, 128)
    q = s.normal(1, 4, 128)
    s.pool.write_tokens_layers(0, 0, 0, s.k[0].cuda(), s.v[0].cuda())
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([4800]))
    for width, first, recent in ((1, 0, 0), (64, 0, 0), (65, 1, 1), (299, 0, 0)):
        picks_of(s, q, [4800], width, first, recent, choices(s, q, [4800], width, first, recent), page_table=wide(s, 1))


def test_wide_tables_with_lengths_that_do_not_fit():
    s = Sessions([200, 200, 200, 200], 4, 2, 64, "bf16", seed=27)
    q = s.normal(4, 4, 64)
    s.pool.set_bounds(True)
    s.pool.update_bounds(0, 1, i32([200] * 4))
    lens = [-1, 0, 16 * 600 + 1, 200]
    want = [[[], []]] * 3 + choices(s, q, [0, 0, 0, 200], 5, 1, 1)[3:]
    picks_of(s, q, lens, 5, 1, 1, want, page_table=wide(s, 4))
