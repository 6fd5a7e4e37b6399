"""Attention of prompt chunks over the paged cache (paged_prefill_attention) against its
float64 definition: packed chunks of any lengths, causal, over hot and spilled pages."""

import numpy as np
import pytest
import torch

from chunk_reference import PAGE, Sessions, attend, check, i32, prefill_reference
from paper_2609_25782_amd import hotcold_kv as kv

pytestmark = pytest.mark.gpu

SHAPES = [(8, 1, 128, "bf16"), (6, 2, 64, "bf16"), (16, 1, 64, "bf16"), (3, 3, 128, "bf16"), (10, 2, 128, "bf16"),
          (4, 1, 64, "f32"), (10, 2, 128, "f32"), (16, 16, 64, "f32")]
# (cached tokens, new tokens) of every row
ROWS = {
    "one": [(0, 1)],
    "short": [(0, 1), (0, 0), (5, 3), (15, 1), (16, 17), (0, 33), (31, 2), (100, 0), (63, 1), (64, 64), (1, 200)],
    "blocks": [(48, 16), (0, 64), (0, 65), (1, 63), (191, 130), (0, 300)],
    "deep": [(2500, 3), (1800, 40)],
}


def packed(rows, gap=0):
    starts = np.cumsum([gap] + [n for _, n in rows]).tolist()
    return starts, [c + n for c, n in rows]


def call(s, q, starts, lens, **kw):
    return s.pool.prefill(0, q.cuda(), i32(starts), i32(lens), **kw)


@pytest.mark.parametrize("rows", sorted(ROWS))
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_matches_definition(hq, hkv, d, dtype, rows):
    starts, lens = packed(ROWS[rows])
    s = Sessions(lens, hq, hkv, d, dtype, seed=len(rows))
    q = s.normal(starts[-1], hq, d)
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.7])
def test_scales(scale, dtype):
    rows = [(0, 40), (77, 9)]
    starts, lens = packed(rows)
    s = Sessions(lens, 4, 2, 64, dtype, seed=3)
    q = s.normal(starts[-1], 4, 64)
    check(call(s, q, starts, lens, scale=scale), *prefill_reference(s, q, starts, lens, scale=scale))


def test_queries_of_no_row_stay():
    """Queries before the first row's and after the last's are left as they were."""
    rows = [(3, 20), (0, 0), (40, 7)]
    starts, lens = packed(rows, gap=5)
    s = Sessions(lens, 8, 2, 128, "bf16", seed=4)
    q = s.normal(starts[-1] + 9, 8, 128)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    got = call(s, q, starts, lens, out=out)
    assert got is out
    ref, bound = prefill_reference(s, q, starts, lens)
    ref[:5] = 7.0
    ref[starts[-1]:] = 7.0
    check(got, ref, bound)


def test_lengths_that_do_not_fit():
    """NaN for a row whose length is below its chunk's or beyond its table row; a range of
    queries outside q writes nothing; the other rows are right."""
    rows = [(10, 12), (0, 6), (20, 5), (0, 4), (30, 8)]
    starts, lens = packed(rows)
    s = Sessions(lens, 4, 2, 64, "bf16", seed=5, stride=4)
    q = s.normal(starts[-1], 4, 64)
    ref, bound = prefill_reference(s, q, starts, lens)
    given = list(lens)
    given[0], given[1], given[2] = 11, -3, 16 * s.pool.stride + 1
    ref[:starts[3]] = np.nan
    check(call(s, q, starts, given), ref, bound)
    # row 4's range ends behind the last query, so row 4 is left out
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    wrong = starts[:5] + [starts[5] + 1]
    ref, bound = prefill_reference(s, q, starts, lens)
    ref[starts[4]:] = 7.0
    check(call(s, q, wrong, lens, out=out), ref, bound)
    # a descending range: that row and no other (row 2 now begins two queries earlier, on row 0's
    # last two, so those belong to two rows and are left out of the comparison)
    wrong = [starts[0], starts[1], starts[1] - 2] + starts[3:]
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    got = call(s, q, wrong, lens, out=out)
    ref, bound = prefill_reference(s, q, starts, lens)
    check(got[:starts[1] - 2], ref[:starts[1] - 2], bound[:starts[1] - 2])
    check(got[starts[3]:], ref[starts[3]:], bound[starts[3]:])


@pytest.mark.parametrize("bad", [-1, 1 << 20, (1 << 29) | 1, (1 << 30) | 3])
def test_bad_pages(bad):
    """Queries that attend to a token on a page outside the pools get NaN, earlier ones their value."""
    rows = [(100, 70), (0, 50)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 1, 128, "bf16", seed=6)
    q = s.normal(starts[-1], 8, 128)
    table = s.pool.page_table[:2].clone()
    table[0, 7] = bad                       # tokens 112 .. 127: queries 12 .. of row 0
    table[1, 0] = bad
    ref, bound = prefill_reference(s, q, starts, lens)
    ref[12:70] = np.nan
    ref[70:] = np.nan
    check(call(s, q, starts, lens, page_table=table), ref, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_later_tokens_do_not_matter(value, dtype):
    """K and V of a token that is not a number: queries before it see nothing of it, queries
    from it on get what the definition gives (V: the value itself)."""
    rows = [(0, 90), (37, 40)]
    starts, lens = packed(rows)
    s = Sessions(lens, 6, 2, 64, dtype, seed=7)
    s.v[0][0, 20, 1, 5] = value             # query 20 on
    s.v[0][0, 70, 0, 63] = value
    s.v[0][0, 71, 0, 63] = -value           # with the opposite infinity: NaN from 71 on
    s.v[1][0, 50] = value                   # query 13 on, every dim
    s.write(0, 0, 20)
    s.write(0, 0, 70)
    s.write(0, 0, 71)
    s.write(1, 0, 50)
    q = s.normal(starts[-1], 6, 64)
    with np.errstate(invalid="ignore"):
        ref, bound = prefill_reference(s, q, starts, lens)
    check(call(s, q, starts, lens), ref, bound)


def test_later_keys_do_not_matter():
    rows = [(0, 90)]
    starts, lens = packed(rows)
    s = Sessions(lens, 4, 1, 128, "bf16", seed=8)
    q = s.normal(90, 4, 128)
    ref, bound = prefill_reference(s, q, starts, lens)
    s.k[0][0, 33] = float("nan")
    s.write(0, 0, 33)
    ref[33:] = np.nan
    check(call(s, q, starts, lens), ref, bound)


def test_wide_scores():
    """Scores of several hundred: the running maximum keeps the exponentials in range."""
    rows = [(500, 60)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 2, 128, "f32", seed=9, value=30.0)
    q = s.normal(60, 8, 128, value=20.0)
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(dtype):
    """More rows than threads of a block, many without queries, all lengths small."""
    rng = np.random.default_rng(10)
    rows = [(int(c), int(n)) for c, n in zip(rng.integers(0, 40, 700), rng.integers(-4, 6, 700).clip(0))]
    rows[100:300] = [(3, 0)] * 200
    starts, lens = packed(rows)
    s = Sessions(lens, 2, 1, 64, dtype, seed=10)
    q = s.normal(starts[-1], 2, 64)
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


def test_long_context_split_over_the_gpu():
    """Few queries over long contexts: tiles cut between many workers."""
    rows = [(9000, 2), (0, 5), (5000, 130)]
    starts, lens = packed(rows)
    s = Sessions(lens, 4, 2, 128, "bf16", seed=11)
    q = s.normal(starts[-1], 4, 128)
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


@pytest.mark.parametrize("host", [False, True])
def test_spilled_pages_in_place(host):
    """Pages that a lazy resume left in the cold tier are read there."""
    rows = [(120, 50), (64, 30)]
    starts, lens = packed(rows)
    from paper_2609_25782_amd.pool import HotColdPool
    s = Sessions(lens, 8, 2, 128, "bf16", seed=12)
    pool = HotColdPool(1, 2, 128, "bf16", 40, 40, 2, 16, cold_location="host" if host else "device")
    for b, L in enumerate(lens):
        pool.create_session(L)
        pool.write_tokens(b, 0, 0, s.k[b][0].cuda(), s.v[b][0].cuda())
    pool.set_spill(True)
    pool.evict([0, 1])
    pool.resume_lazy([0, 1])
    pool.promote(5)
    s.pool = pool
    q = s.normal(starts[-1], 8, 128)
    assert bool(((pool.page_table[:2] >> 30) == 1).any()) and bool((pool.page_table[0] < 1 << 29).any())
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


def test_page_placement_does_not_matter():
    rows = [(300, 200), (10, 33)]
    starts, lens = packed(rows)
    outs = []
    for spare in (8, 100):
        s = Sessions(lens, 8, 2, 128, "bf16", seed=13, spare=spare)
        g = torch.Generator().manual_seed(99)
        k = [torch.randn((1, n, 2, 128), generator=g).bfloat16() for n in lens]
        for b, n in enumerate(lens):
            s.pool.write_tokens_layers(b, 0, 0, k[b].cuda(), (-k[b]).cuda())
        q = torch.randn((starts[-1], 8, 128), generator=g).bfloat16()
        outs.append(call(s, q, starts, lens))
    assert torch.equal(outs[0], outs[1])


def test_layers_and_decode_agree():
    """Each layer reads its own slice; the last query of a row is what decode gives."""
    rows = [(200, 30), (17, 5)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 2, 128, "bf16", seed=14, layers=3)
    q = s.normal(starts[-1], 8, 128)
    for layer in range(3):
        got = s.pool.prefill(layer, q.cuda(), i32(starts), i32(lens))
        ref, bound = prefill_reference(s, q, starts, lens, layer=layer)
        check(got, ref, bound)
        last = [e - 1 for e in starts[1:]]
        dec = s.pool.decode(layer, q[last].cuda().contiguous(), i32(lens), page_table=s.pool.page_table[:2])
        diff = (dec.float() - got[last].float()).abs().cpu().numpy()
        assert np.all(diff <= 2 * bound[last])   # both are within the bound of the definition


def test_graph_replays():
    """A captured call reads lengths, starts and pages when it is replayed; two graphs and the
    eager call do not disturb each other."""
    rows = [(700, 40), (90, 100), (0, 60)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 2, 128, "bf16", seed=15)
    q = [s.normal(starts[-1], 8, 128).cuda() for _ in range(2)]
    d_starts, d_lens = i32(starts), i32(lens)
    refs = [prefill_reference(s, x.cpu(), starts, lens) for x in q]
    outs = [torch.zeros_like(x) for x in q]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for i in range(2):
        s.pool.prefill(0, q[i], d_starts, d_lens, out=outs[i], stream=side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            s.pool.prefill(0, q[i], d_starts, d_lens, out=outs[i], stream=side)
        graphs.append(g)
    other = torch.cuda.Stream()
    for rep in range(4):
        for o in outs:
            o.fill_(7.0)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):      # beside the first
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            check(outs[i], *refs[i], what="replay %d graph %d" % (rep, i))
        eager = s.pool.prefill(0, q[0], d_starts, d_lens)
        torch.cuda.synchronize()
        assert torch.equal(eager, outs[0])
    new = [650, 130, 60]                    # other lengths, the same chunks
    d_lens.copy_(i32(new))
    new_starts = [0, 35, 140, 200]
    d_starts.copy_(i32(new_starts))
    ref = prefill_reference(s, q[1].cpu(), new_starts, [650, 130, 60])
    graphs[1].replay()
    torch.cuda.synchronize()
    check(outs[1], *ref, what="changed lengths")


def test_calls_on_two_streams():
    rows = [(1500, 60), (400, 33)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 2, 128, "bf16", seed=16)
    q = [s.normal(starts[-1], 8, 128) for _ in range(2)]
    refs = [prefill_reference(s, x, starts, lens) for x in q]
    dq, ds, dl = [x.cuda() for x in q], i32(starts), i32(lens)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        outs = [s.pool.prefill(0, dq[i], ds, dl, stream=streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for i in range(2):
            check(outs[i], *refs[i])


def test_profiling_counts_both_kernels():
    rows = [(64, 16)]
    starts, lens = packed(rows)
    s = Sessions(lens, 4, 1, 64, "bf16", seed=17)
    q = s.normal(16, 4, 64)
    kv.kv_pool_set_profiling(s.pool.handle, True)
    call(s, q, starts, lens)
    torch.cuda.synchronize()
    for k in (kv.KV_KERNEL_CHUNK, kv.KV_KERNEL_CHUNK_MERGE):
        n, ms = kv.kv_pool_profile_read(s.pool.handle, k)
        assert n == 1 and ms > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ["64", "65", "even", "uneven", "several tiles"])
def test_splits(rows, dtype):
    """Batches on both sides of a wave's lanes; tiles in equal parts, and where those would be
    uneven, in ranges; several tiles a row."""
    r = {"64": [(40 * b % 700, b % 4) for b in range(64)], "65": [(40 * b % 700, b % 4) for b in range(65)],
         "even": [(3000, 8), (3010, 7), (2900, 8), (2990, 1)], "uneven": [(5000, 8), (3, 7), (90, 8), (2500, 1)],
         "several tiles": [(3000, 120), (2900, 70), (3100, 33)]}[rows]
    starts, lens = packed(r)
    s = Sessions(lens, 8, 1, 128, dtype, seed=32)
    q = s.normal(starts[-1], 8, 128)
    check(call(s, q, starts, lens), *prefill_reference(s, q, starts, lens))


def test_a_captured_stream_that_is_not_current():
    """A call on a stream under capture, made while another stream is current, takes its workspace
    from its graph as well: the graph and eager calls on that stream do not share one."""
    rows = [(0, 40), (77, 9)]
    starts, lens = packed(rows)
    s = Sessions(lens, 8, 2, 64, "bf16", seed=31)
    q = s.normal(starts[-1], 8, 64)
    side, dq, dstarts, dlens = torch.cuda.Stream(), q.cuda(), i32(starts), i32(lens)
    out = torch.empty_like(dq)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    main = torch.cuda.current_stream()
    with torch.cuda.graph(graph, stream=side):
        with torch.cuda.stream(main):
            s.pool.prefill(0, dq, dstarts, dlens, out=out, stream=side)
    assert not s.pool._ws
    ref = prefill_reference(s, q, starts, lens)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        got = s.pool.prefill(0, dq, dstarts, dlens, stream=side)
        torch.cuda.synchronize()
        check(out, *ref)
        check(got, *ref)
    assert s.pool._ws


def test_a_length_past_2_30_is_nan():
    """Lengths of more than 2^30 tokens fit no row, however long its table claims to be: NaN, and
    nothing of the table or the pages is read (2^30 tokens of a table that is there would not fit
    into memory)."""
    s = Sessions([40], 4, 2, 64, "bf16", seed=30)
    q = s.normal(16, 4, 64).cuda()
    out = torch.zeros_like(q)
    ws = torch.empty(kv.paged_prefill_workspace_bytes(s.pool.handle, 1, 16, 4), dtype=torch.uint8, device="cuda")
    for length in ((1 << 30) + 1, 2**31 - 1):
        out.zero_()
        starts, lens = i32([0, 16]), i32([length])
        kv.paged_prefill_attention(s.pool.handle, 0, q.data_ptr(), starts.data_ptr(), 16, s.pool.page_table.data_ptr(),
                                   1 << 28, lens.data_ptr(), 1, 4, 0.1, out.data_ptr(), ws.data_ptr(), ws.numel())
        torch.cuda.synchronize()
        assert out.isnan().all()


def test_refusals():
    s = Sessions([40], 4, 2, 64, "bf16", seed=18, layers=2)
    q = s.normal(16, 4, 64).cuda()
    out = torch.zeros_like(q)
    starts, lens = i32([0, 16]), i32([40])
    need = kv.paged_prefill_workspace_bytes(s.pool.handle, 1, 16, 4)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    good = dict(pool=s.pool.handle, layer=1, q_ptr=q.data_ptr(), q_starts_ptr=starts.data_ptr(), total_q=16,
                page_table_ptr=s.pool.page_table.data_ptr(), pt_stride=s.pool.stride, seq_lens_ptr=lens.data_ptr(),
                batch=1, num_q_heads=4, scale=0.1, out_ptr=out.data_ptr(), workspace_ptr=ws.data_ptr(),
                ws_bytes=need)
    kv.paged_prefill_attention(**good)
    torch.cuda.synchronize()
    done = out.clone()
    bad = [dict(layer=2), dict(layer=-1), dict(q_ptr=0), dict(q_starts_ptr=0), dict(total_q=-1),
           dict(page_table_ptr=0), dict(pt_stride=0), dict(seq_lens_ptr=0), dict(batch=-1), dict(batch=8193),
           dict(pt_stride=1 << 31), dict(num_q_heads=0), dict(num_q_heads=5), dict(num_q_heads=34), dict(out_ptr=0),
           dict(out_ptr=out.data_ptr() + 8), dict(q_ptr=q.data_ptr() + 2), dict(workspace_ptr=0),
           dict(workspace_ptr=ws.data_ptr() + 128), dict(ws_bytes=need - 1), dict(pool=0)]
    for change in bad:
        with pytest.raises(kv.KVError) as e:
            kv.paged_prefill_attention(**{**good, **change})
        assert e.value.status == kv.KV_ERR_INVALID, change
    kv.paged_prefill_attention(**{**good, "batch": 0})        # nothing to do
    kv.paged_prefill_attention(**{**good, "total_q": 0})
    torch.cuda.synchronize()
    assert torch.equal(out, done)
    assert kv.paged_prefill_workspace_bytes(s.pool.handle, 1, 16, 5) == 0
    for wrong in (dict(q=q.float()), dict(q=q[:, :, :32].contiguous()), dict(q=q.transpose(0, 1)),
                  dict(q_starts=i32([0])), dict(seq_lens=lens.long()), dict(page_table=s.pool.page_table[:0]),
                  dict(out=out[:8])):
        args = dict(layer=0, q=q, q_starts=starts, seq_lens=lens)
        args.update(wrong)
        with pytest.raises(AssertionError):
            s.pool.prefill(**args)


@pytest.mark.parametrize("hkv", [1, 2])
def test_workspace_sizes_know_what_is_refused(hkv):
    """0 for the batches and heads that the calls refuse, and for no others."""
    pool = Sessions([40], 4 * hkv, hkv, 64, "bf16", seed=19).pool
    sizes = {"prefill": lambda batch, heads: kv.paged_prefill_workspace_bytes(pool.handle, batch, 16, heads),
             "tree": lambda batch, heads: kv.paged_tree_workspace_bytes(pool.handle, batch, 4, heads)}
    for name, size in sizes.items():
        for batch in (0, 1, 8192):
            for heads in (hkv, 3 * hkv, 16 * hkv):
                assert size(batch, heads) > 0, (name, batch, heads)
        for batch, heads in ((8193, hkv), (1 << 30, hkv), (-1, hkv), (1, 17 * hkv), (1, 32 * hkv), (1, 0), (1, -hkv),
                             (0, 17 * hkv)):
            assert size(batch, heads) == 0, (name, batch, heads)
    assert kv.paged_prefill_workspace_bytes(pool.handle, 1, -1, hkv) == 0
    for width in (0, -1, 65):
        assert kv.paged_tree_workspace_bytes(pool.handle, 1, width, hkv) == 0
