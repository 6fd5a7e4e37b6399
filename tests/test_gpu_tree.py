"""Attention of drafted tokens over the paged cache (paged_tree_attention), the write of the
accepted ones (kv_accept_drafts), and a serving run of prompt, draft, check and accept."""

import numpy as np
import pytest
import torch

from chunk_reference import (PAGE, TORCH, Sessions, check, i32, mask_tensor, prefill_reference, random_tree,
                             tree_reference)
from paper_2609_25782_amd import hotcold_kv as kv
from paper_2609_25782_amd.pool import HotColdPool

pytestmark = pytest.mark.gpu

SHAPES = [(8, 1, 128, "bf16"), (32, 4, 128, "bf16"), (6, 2, 64, "bf16"), (16, 1, 64, "bf16"), (3, 3, 128, "bf16"),
          (4, 1, 64, "f32"), (10, 2, 128, "f32")]
# width, (cached tokens, drafts) of every row
ROWS = {
    "one": (1, [(0, 1), (1, 1), (700, 1)]),
    "eight": (8, [(0, 8), (1, 3), (15, 0), (16, 8), (17, 1), (63, 8), (64, 7), (65, 8), (640, 5)]),
    "odd": (33, [(100, 33), (0, 20), (31, 32), (200, 1)]),
    "wide": (64, [(0, 64), (130, 64), (64, 49), (2000, 63)]),
}


def setup(rows, width, hq, hkv, d, dtype, seed, **kw):
    lens, drafts = [c for c, _ in rows], [n for _, n in rows]
    s = Sessions(lens, hq, hkv, d, dtype, seed=seed, **kw)
    rng = np.random.default_rng(seed)
    masks = [random_tree(rng, n, width) for n in drafts]
    B = len(rows)
    q, kd, vd = s.normal(B, width, hq, d), s.normal(B, width, hkv, d), s.normal(B, width, hkv, d)
    return s, lens, drafts, masks, q, kd, vd


def call(s, q, kd, vd, masks, lens, drafts, **kw):
    kw.setdefault("out", torch.zeros(q.shape, dtype=q.dtype, device="cuda"))
    return s.pool.tree_decode(0, q.cuda(), kd.cuda(), vd.cuda(), mask_tensor(masks), i32(lens),
                              draft_lens=None if drafts is None else i32(drafts), **kw)


@pytest.mark.parametrize("rows", sorted(ROWS))
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_matches_definition(hq, hkv, d, dtype, rows):
    width, r = ROWS[rows]
    s, lens, drafts, masks, q, kd, vd = setup(r, width, hq, hkv, d, dtype, seed=len(rows))
    check(call(s, q, kd, vd, masks, lens, drafts), *tree_reference(s, q, kd, vd, masks, lens, drafts))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_of_any_kind(dtype):
    """Empty masks (nothing but the context, or nothing at all: zeros), bits without the draft's
    own, bits past the row's drafts, drafts seeing later ones."""
    rows = [(0, 6), (40, 6), (0, 9), (5, 9)]
    s, lens, drafts, _, q, kd, vd = setup(rows, 9, 4, 2, 64, dtype, seed=1)
    full = (1 << 64) - 1
    masks = [[0, 1, 2, 0, full, 1 << 63] + [0] * 3, [0, 0, 32, full, 1 << 8, 63] + [0] * 3, [full] * 9, [0] * 9]
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    assert not ref[0, 0].any() and not ref[0, 5].any()
    check(call(s, q, kd, vd, masks, lens, drafts), ref, bound)


@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_scales(scale):
    s, lens, drafts, masks, q, kd, vd = setup([(33, 5), (0, 4)], 5, 4, 2, 64, "bf16", seed=2)
    check(call(s, q, kd, vd, masks, lens, drafts, scale=scale),
          *tree_reference(s, q, kd, vd, masks, lens, drafts, scale=scale))


def test_draft_counts():
    """Without counts every draft is live; counts outside [0, width] count as the nearer end;
    drafts past the count are neither read nor written."""
    s, lens, _, masks, q, kd, vd = setup([(20, 7), (3, 7), (50, 7)], 7, 8, 2, 128, "bf16", seed=3)
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, [7, 7, 7])
    check(call(s, q, kd, vd, masks, lens, None), ref, bound)
    q[1, 4:], kd[1, 4:], vd[1, 4:] = float("nan"), float("nan"), float("nan")
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, [7, 4, 0])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ref[1, 4:] = 7.0
    ref[2] = 7.0
    check(call(s, q, kd, vd, masks, lens, [99, 4, -2], out=out), ref, bound)


def test_lengths_that_do_not_fit():
    s, lens, drafts, masks, q, kd, vd = setup([(20, 3), (3, 2), (50, 4)], 4, 4, 2, 64, "f32", seed=4)
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    ref[0, :3] = np.nan
    ref[1, :2] = np.nan
    check(call(s, q, kd, vd, masks, [-1, 16 * s.pool.stride + 1, 50], drafts), ref, bound)


@pytest.mark.parametrize("bad", [-1, 1 << 20, (1 << 29) | 1, (1 << 30) | 3])
def test_bad_pages(bad):
    s, lens, drafts, masks, q, kd, vd = setup([(90, 5), (33, 5)], 5, 8, 1, 128, "bf16", seed=5)
    table = s.pool.page_table[:2].clone()
    table[0, 3] = bad
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    ref[0] = np.nan
    check(call(s, q, kd, vd, masks, lens, drafts, page_table=table), ref, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_other_branches_do_not_matter(value, dtype):
    """A draft whose K and V are not numbers changes its descendants only."""
    width = 40
    s, lens, drafts, _, q, kd, vd = setup([(70, 40), (0, 12)], width, 6, 2, 64, dtype, seed=6)
    masks = [[(1 << i) | (1 << (i % 2)) for i in range(width)], [1 << i for i in range(width)]]
    vd[0, 1, 0, 3] = value              # odd drafts of row 0
    kd[1, 4] = float("nan")             # draft 4 of row 1 alone
    vd[1, 7] = value
    with np.errstate(invalid="ignore"):
        ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    assert np.isnan(ref[1, 4]).all() and np.isfinite(ref[1, 5]).all() and np.isfinite(ref[0, 2]).all()
    check(call(s, q, kd, vd, masks, lens, drafts), ref, bound)


def test_many_rows():
    rng = np.random.default_rng(7)
    rows = [(int(c), int(n)) for c, n in zip(rng.integers(0, 200, 600), rng.integers(-2, 4, 600).clip(0))]
    rows[50:250] = [(9, 0)] * 200
    s, lens, drafts, masks, q, kd, vd = setup(rows, 3, 4, 1, 64, "bf16", seed=7)
    check(call(s, q, kd, vd, masks, lens, drafts), *tree_reference(s, q, kd, vd, masks, lens, drafts))


@pytest.mark.parametrize("width", [2, 20])
def test_long_context_split_over_the_gpu(width):
    s, lens, drafts, masks, q, kd, vd = setup([(12000, width), (3, 1)], width, 8, 1, 128, "bf16", seed=8)
    check(call(s, q, kd, vd, masks, lens, drafts), *tree_reference(s, q, kd, vd, masks, lens, drafts))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ["64", "65", "even", "uneven", "two tiles"])
def test_splits(rows, dtype):
    """Batches on both sides of a wave's lanes; tiles in equal parts, and where those would be
    uneven, in ranges; two tiles a row cut alike."""
    width, r = {"64": (3, [(40 * b % 700, b % 4) for b in range(64)]),
                "65": (3, [(40 * b % 700, b % 4) for b in range(65)]),
                "even": (8, [(3000, 8), (3010, 7), (2900, 8), (2990, 1)]),
                "uneven": (8, [(5000, 8), (3, 7), (90, 8), (2500, 1)]),
                "two tiles": (64, [(3000, 64), (2900, 40), (3100, 50)])}[rows]
    s, lens, drafts, masks, q, kd, vd = setup(r, width, 8, 1, 128, dtype, seed=21)
    check(call(s, q, kd, vd, masks, lens, drafts), *tree_reference(s, q, kd, vd, masks, lens, drafts))


def test_one_draft_is_a_decode_step():
    """A draft that sees itself, accepted, then decoded: decode over C + 1 tokens."""
    rows = [(100, 1), (31, 1), (640, 1)]
    s, lens, drafts, _, q, kd, vd = setup(rows, 1, 8, 2, 128, "bf16", seed=9, stride=48)
    masks = [[1]] * 3
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    got = call(s, q, kd, vd, masks, lens, drafts)
    check(got, ref, bound)
    for b, L in enumerate(lens):
        s.pool.extend(b, L + 1)
    s.pool.accept_drafts(0, s.pool.page_table[:3].contiguous(), i32(lens), torch.zeros((3, 1), dtype=torch.int32).cuda(),
                         i32([1, 1, 1]), kd.cuda()[None], vd.cuda()[None])
    dec = s.pool.decode(0, q[:, 0].cuda().contiguous(), i32([n + 1 for n in lens]))
    assert np.all((dec.float() - got[:, 0].float()).abs().cpu().numpy() <= 2 * bound[:, 0])


def test_graph_replays():
    s, lens, drafts, masks, q, kd, vd = setup([(900, 6), (100, 3), (40, 6)], 6, 8, 2, 128, "bf16", seed=10)
    args = [q.cuda(), kd.cuda(), vd.cuda(), mask_tensor(masks), i32(lens)]
    dl = i32(drafts)
    out = torch.zeros_like(args[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.pool.tree_decode(0, *args, draft_lens=dl, out=out, stream=side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        s.pool.tree_decode(0, *args, draft_lens=dl, out=out, stream=side)
    ref, bound = tree_reference(s, q, kd, vd, masks, lens, drafts)
    for rep in range(4):
        out.fill_(0.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(out, ref, bound, what="replay %d" % rep)
        eager = s.pool.tree_decode(0, *args, draft_lens=dl, out=torch.zeros_like(out))
        torch.cuda.synchronize()
        assert torch.equal(eager, out)
    lens2, drafts2 = [500, 99, 0], [2, 6, 5]
    args[4].copy_(i32(lens2))
    dl.copy_(i32(drafts2))
    masks2 = [random_tree(np.random.default_rng(1), n, 6) for n in drafts2]
    args[3].copy_(mask_tensor(masks2))
    out.fill_(0.0)
    g.replay()
    torch.cuda.synchronize()
    check(out, *tree_reference(s, q, kd, vd, masks2, lens2, drafts2))


def test_tree_refusals():
    s, lens, drafts, masks, q, kd, vd = setup([(40, 4)], 4, 4, 2, 64, "bf16", seed=11)
    q, kd, vd, mk, ln = q.cuda(), kd.cuda(), vd.cuda(), mask_tensor(masks), i32(lens)
    out = torch.zeros_like(q)
    need = kv.paged_tree_workspace_bytes(s.pool.handle, 1, 4, 4)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    good = dict(pool=s.pool.handle, layer=0, q_ptr=q.data_ptr(), k_draft_ptr=kd.data_ptr(),
                v_draft_ptr=vd.data_ptr(), masks_ptr=mk.data_ptr(), draft_lens_ptr=0, width=4,
                page_table_ptr=s.pool.page_table.data_ptr(), pt_stride=s.pool.stride, seq_lens_ptr=ln.data_ptr(),
                batch=1, num_q_heads=4, scale=0.1, out_ptr=out.data_ptr(), workspace_ptr=ws.data_ptr(), ws_bytes=need)
    kv.paged_tree_attention(**good)
    torch.cuda.synchronize()
    done = out.clone()
    bad = [dict(layer=1), dict(layer=-1), dict(q_ptr=0), dict(k_draft_ptr=0), dict(v_draft_ptr=0), dict(masks_ptr=0),
           dict(masks_ptr=mk.data_ptr() + 4), dict(width=0), dict(width=65), dict(page_table_ptr=0),
           dict(pt_stride=0), dict(pt_stride=1 << 31), dict(seq_lens_ptr=0), dict(batch=-1), dict(batch=8193),
           dict(num_q_heads=3), dict(num_q_heads=34), dict(out_ptr=0), dict(out_ptr=out.data_ptr() + 8),
           dict(k_draft_ptr=kd.data_ptr() + 8), dict(v_draft_ptr=vd.data_ptr() + 2), dict(workspace_ptr=0),
           dict(workspace_ptr=ws.data_ptr() + 16), dict(ws_bytes=need - 1), dict(pool=0)]
    for change in bad:
        with pytest.raises(kv.KVError) as e:
            kv.paged_tree_attention(**{**good, **change})
        assert e.value.status == kv.KV_ERR_INVALID, change
    kv.paged_tree_attention(**{**good, "batch": 0})
    torch.cuda.synchronize()
    assert torch.equal(out, done)
    assert kv.paged_tree_workspace_bytes(s.pool.handle, 1, 65, 4) == 0
    for wrong in (dict(q=q.float()), dict(k_draft=kd[:, :3].contiguous()), dict(masks=mk.int()), dict(masks=mk[:, :2]),
                  dict(seq_lens=ln.long()), dict(draft_lens=i32([1, 2])), dict(out=out[:, :2])):
        args = dict(layer=0, q=q, k_draft=kd, v_draft=vd, masks=mk, seq_lens=ln)
        args.update(wrong)
        with pytest.raises(AssertionError):
            s.pool.tree_decode(**args)


# -- accepted drafts -----------------------------------------------------------

def tokens_of(pool, page_bytes, dtype, hkv, d):
    """Pages as [pages][layers][K, V][16 tokens][kv_heads][d]."""
    x = 8 if dtype == "bf16" else 4
    t = page_bytes.view(TORCH[dtype]).view(-1, pool.num_layers, hkv, 2, d * PAGE)
    k = t[:, :, :, 0].reshape(-1, pool.num_layers, hkv, d // x, PAGE, x).permute(0, 1, 4, 2, 3, 5).reshape(
        -1, pool.num_layers, PAGE, hkv, d)
    v = t[:, :, :, 1].reshape(-1, pool.num_layers, hkv, d, PAGE).permute(0, 1, 4, 2, 3)
    return torch.stack([k, v], dim=2)


@pytest.mark.parametrize("layers,first,hkv,d,dtype", [(1, 0, 4, 128, "bf16"), (5, 2, 2, 64, "bf16"), (3, 0, 1, 64, "bf16"),
                                                      (2, 1, 16, 128, "f32"), (4, 0, 3, 64, "f32")])
@pytest.mark.parametrize("width", [1, 7, 64])
def test_accept_writes_the_path_and_nothing_else(layers, first, hkv, d, dtype, width):
    rng = np.random.default_rng(width)
    lens = [0, 1, 15, 16, 30, 100, 7]
    B = len(lens)
    s = Sessions(lens, hkv, hkv, d, dtype, seed=20, layers=layers, spare=60, poison=False)
    pool = HotColdPool(layers, hkv, d, dtype, 200, 0, B, 12)
    for b, L in enumerate(lens):
        pool.create_session(L + width)
    pool.hot.random_(0, 250)
    before = pool.hot_page_bytes().clone()
    counts = [int(x) for x in rng.integers(0, width, size=B, endpoint=True)]
    counts[0], counts[1], counts[2] = width, 0, width + 5
    path = np.stack([rng.integers(0, width, size=width) for _ in lens]).astype(np.int32)   # the same draft twice, too
    path[4, 0] = -1
    path[5, width - 1] = width
    n = layers - first
    kd, vd = s.normal(n, B, width, hkv, d), s.normal(n, B, width, hkv, d)
    table = pool.page_table.clone()
    pool.accept_drafts(first, table, i32(lens), torch.from_numpy(path).cuda(), i32(counts), kd.cuda(), vd.cuda())
    torch.cuda.synchronize()
    want = tokens_of(pool, before.cpu(), dtype, hkv, d).clone()
    got = tokens_of(pool, pool.hot_page_bytes().cpu(), dtype, hkv, d)
    t = table.cpu().numpy()
    for b, L in enumerate(lens):
        for j in range(max(0, min(counts[b], width))):
            src = int(path[b, j])
            if not 0 <= src < width:
                continue
            p, slot = int(t[b, (L + j) // PAGE]), (L + j) % PAGE
            want[p, first:, 0, slot] = kd[:, b, src]
            want[p, first:, 1, slot] = vd[:, b, src]
    as_bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(got.contiguous().view(as_bits), want.contiguous().view(as_bits))


def test_accept_past_the_table_and_bad_entries():
    """Positions past the row's table and entries that name no page write nothing; spilled pages are
    written in place."""
    pool = HotColdPool(1, 2, 64, "bf16", 4, 4, 3, 2)
    pool.set_spill(True)
    pool.hot.zero_()
    pool.cold.zero_()
    table = torch.tensor([[0, 1], [-1, 2], [(1 << 30) | 1, (1 << 30) | 9]], dtype=torch.int32).cuda()
    kd = torch.ones((1, 3, 8, 2, 64), dtype=torch.bfloat16).cuda()
    path = torch.arange(8, dtype=torch.int32).repeat(3, 1).cuda()
    pool.accept_drafts(0, table, i32([28, 12, 14]), path, i32([8, 8, 8]), kd, kd)
    torch.cuda.synchronize()
    hot = tokens_of(pool, pool.hot_page_bytes().cpu(), "bf16", 2, 64)[:, 0, :, :, 0, 0].float().sum(dim=(1, 2)).tolist()
    cold = tokens_of(pool, pool.cold.cpu(), "bf16", 2, 64)[:, 0, :, :, 0, 0].float().sum(dim=(1, 2)).tolist()
    assert hot == [0.0, 8.0, 8.0, 0.0]      # K and V of 4 tokens each: 28 .. 31, and 16 .. 19 of row 1
    assert cold == [0.0, 4.0, 0.0, 0.0]     # tokens 14 and 15 of row 2; page 9 does not exist
    # lengths that name no token
    pool.accept_drafts(0, table, i32([-5, 32, 1 << 30]), path, i32([8, 8, 8]), kd, kd)
    torch.cuda.synchronize()
    again = tokens_of(pool, pool.hot_page_bytes().cpu(), "bf16", 2, 64)[:, 0, :, :, 0, 0].float().sum(dim=(1, 2)).tolist()
    assert again == hot


def test_accept_refusals():
    pool = HotColdPool(2, 2, 64, "bf16", 4, 0, 1, 4)
    pool.hot.zero_()
    kd = torch.ones((2, 1, 8, 2, 64), dtype=torch.bfloat16).cuda()
    ln, path, cnt = i32([0]), torch.zeros((1, 8), dtype=torch.int32).cuda(), i32([8])
    good = dict(pool=pool.handle, layer_begin=0, num_layers=2, table_ptr=pool.page_table.data_ptr(), pt_stride=4,
                seq_lens_ptr=ln.data_ptr(), path_ptr=path.data_ptr(), counts_ptr=cnt.data_ptr(), batch=1, width=8,
                k_ptr=kd.data_ptr(), v_ptr=kd.data_ptr())
    bad = [dict(pool=0), dict(layer_begin=-1), dict(layer_begin=1), dict(num_layers=0), dict(num_layers=3),
           dict(num_layers=2 ** 31 - 1, layer_begin=1), dict(table_ptr=0), dict(pt_stride=0), dict(pt_stride=1 << 31),
           dict(seq_lens_ptr=0), dict(path_ptr=0), dict(counts_ptr=0), dict(batch=-1), dict(batch=8193), dict(width=0),
           dict(width=65), dict(k_ptr=0), dict(v_ptr=0), dict(k_ptr=kd.data_ptr() + 8), dict(v_ptr=kd.data_ptr() + 2)]
    for change in bad:
        with pytest.raises(kv.KVError) as e:
            kv.kv_accept_drafts(**{**good, **change})
        assert e.value.status == kv.KV_ERR_INVALID, change
    kv.kv_accept_drafts(**{**good, "batch": 0})
    for wrong in (dict(k=kd[0]), dict(path=path[:, :4]), dict(counts=cnt.long()), dict(table=pool.page_table[:0])):
        args = dict(layer_begin=0, table=pool.page_table, seq_lens=ln, path=path, counts=cnt, k=kd, v=kd)
        args.update(wrong)
        with pytest.raises(AssertionError):
            pool.accept_drafts(**args)
    torch.cuda.synchronize()
    assert not pool.hot.any()               # an unused page table names no page either


# -- together ------------------------------------------------------------------

def test_prompt_draft_check_accept():
    """A serving run: prompts are taken in, sessions pause and come back, then every step drafts
    a tree, checks it, accepts a path on the device (inside a replayed graph) and goes on."""
    layers, hq, hkv, d, T, dtype = 3, 8, 2, 128, 6, "bf16"
    g = torch.Generator().manual_seed(30)

    def normal(*shape):
        return torch.randn(shape, generator=g).bfloat16()

    prompts = [150, 33, 400]
    B = len(prompts)
    pool = HotColdPool(layers, hkv, d, dtype, 200, 200, B, 64)
    pool.hot.view(torch.bfloat16).fill_(float("nan"))
    s = Sessions([], hq, hkv, d, dtype)
    s.k = [normal(layers, n, hkv, d) for n in prompts]
    s.v = [normal(layers, n, hkv, d) for n in prompts]
    s.pool = pool
    starts = np.cumsum([0] + prompts).tolist()
    for b, n in enumerate(prompts):
        assert pool.create_session(n) == b
        pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    for layer in range(layers):
        q = normal(starts[-1], hq, d)
        check(pool.prefill(layer, q.cuda(), i32(starts), i32(prompts)), *prefill_reference(s, q, starts, prompts, layer))
    pool.evict([0, 1, 2])
    pool.resume([2, 0, 1])
    lens = list(prompts)
    q = torch.zeros((layers, B, T, hq, d), dtype=torch.bfloat16, device="cuda")
    kd = torch.zeros((layers, B, T, hkv, d), dtype=torch.bfloat16, device="cuda")
    vd, out = torch.zeros_like(kd), torch.zeros_like(q)
    d_lens, d_mask = i32(lens), torch.zeros((B, T), dtype=torch.int64, device="cuda")
    path, counts = torch.zeros((B, T), dtype=torch.int32, device="cuda"), i32([0] * B)
    table = torch.zeros((B, pool.stride), dtype=torch.int32, device="cuda")

    def step():
        table.copy_(pool.page_table)
        for layer in range(layers):
            pool.tree_decode(layer, q[layer], kd[layer], vd[layer], d_mask, d_lens, page_table=table, out=out[layer],
                             stream=side)
        pool.accept_drafts(0, table, d_lens, path, counts, kd, vd, stream=side)
        d_lens.add_(counts)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    rng = np.random.default_rng(31)
    for turn in range(5):
        for b in range(B):
            pool.extend(b, lens[b] + T)
        hq_, hk, hv = normal(layers, B, T, hq, d), normal(layers, B, T, hkv, d), normal(layers, B, T, hkv, d)
        masks = [random_tree(rng, T, T) for _ in range(B)]
        paths, n = np.zeros((B, T), np.int32), [int(x) for x in rng.integers(0, T, size=B, endpoint=True)]
        for b in range(B):
            paths[b, :n[b]] = np.sort(rng.permutation(T)[:n[b]])
        q.copy_(hq_)
        kd.copy_(hk)
        vd.copy_(hv)
        d_mask.copy_(mask_tensor(masks))
        path.copy_(torch.from_numpy(paths))
        counts.copy_(i32(n))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for layer in range(layers):
            check(out[layer], *tree_reference(s, hq_[layer], hk[layer], hv[layer], masks, lens, [T] * B, layer),
                  what="turn %d layer %d" % (turn, layer))
        for b in range(B):
            s.k[b] = torch.cat([s.k[b], hk[:, b, paths[b, :n[b]]]], dim=1)
            s.v[b] = torch.cat([s.v[b], hv[:, b, paths[b, :n[b]]]], dim=1)
            lens[b] += n[b]
        assert d_lens.tolist() == lens
    # the accepted tokens survive an eviction, and a tool's output joins them
    pool.evict([1])
    pool.resume([1])
    new = [9, 0, 21]
    rows = i32([0] * 9 + [2] * 21)
    pos = i32([lens[0] + i for i in range(9)] + [lens[2] + i for i in range(21)])
    k, v = normal(layers, 30, hkv, d), normal(layers, 30, hkv, d)
    for b in range(B):
        if new[b]:
            pool.extend(b, max(pool.info(b)[1], lens[b] + new[b]))
    pool.append_tokens_table(0, pool.page_table, rows, pos, k.cuda(), v.cuda())
    at = 0
    for b in range(B):
        s.k[b] = torch.cat([s.k[b], k[:, at:at + new[b]]], dim=1)
        s.v[b] = torch.cat([s.v[b], v[:, at:at + new[b]]], dim=1)
        at += new[b]
        lens[b] += new[b]
    starts = [0, 9, 9, 30]
    for layer in range(layers):
        q1 = normal(30, hq, d)
        check(pool.prefill(layer, q1.cuda(), i32(starts), i32(lens)), *prefill_reference(s, q1, starts, lens, layer))
