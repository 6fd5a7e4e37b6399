"""Measured calls of the attention over several new tokens of a session, and of the
write that follows a verified draft.

  prefill  causal attention of packed prompt chunks over their sessions' pages: row b
           brings the last n_b of its L_b tokens as queries (a whole prompt when
           n_b = L_b, an agent turn's tool output when most of L_b is cached)
  tree     attention of a tree of drafted tokens: every draft attends to its session's
           cached context and to the drafts its mask names (itself and its ancestors)
  accept   the drafts that the target model accepted get their K and V written to the
           sessions' pages, all layers at once

Context and chunk lengths, draft trees' sizes and accepted counts belong to the case
(drawn from its `length_seed`); values, page placement and the trees' shapes come from
the seed.  Values are N(0, 1): scores then spread as a trained model's do.
"""

import numpy as np
import torch

own = False

PAGE = 16
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
# (query heads, KV heads, head dim): the model's attention shape, and the grouped,
# multi-query and multi-head shapes that the tests cover
SHAPES = [(32, 4, 128), (32, 4, 128), (32, 8, 128), (16, 1, 128), (8, 2, 64), (16, 16, 64), (6, 2, 64), (4, 1, 64)]
MODEL = {"hq": 32, "hkv": 4, "d": 128, "dtype": "bf16"}


def _case(name, op, batch, ctx, new, layers=1, width=0, length_seed=0, **shape):
    """`ctx` and `new` are (lowest, highest) counts per session: tokens cached before the
    call, and tokens (or drafts, or accepted drafts) it brings."""
    c = {"op": op, "batch": batch, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0], "new_hi": new[1],
         "layers": layers, "width": width, "length_seed": length_seed}
    c.update(MODEL)
    c.update(shape)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The smallest call: four short float32 chunks, where launches and latency count.
        _case("prefill_tiny_f32", "prefill", 4, (0, 300), (1, 40), hq=4, hkv=1, d=64, dtype="f32"),
        # Chunks of odd lengths with three query heads per KV head, a few new tokens to
        # many, over contexts from nothing on.
        _case("prefill_odd_group", "prefill", 7, (0, 3001), (1, 701), hq=6, hkv=2, d=64),
        # An ordinary agent step: eight resumed sessions of 8K to 32K tokens each take in
        # a tool's output.
        _case("prefill_turns", "prefill", 8, (8192, 32768), (64, 1024)),
        # New sessions' prompts of very different lengths, packed.
        _case("prefill_prompts", "prefill", 12, (0, 0), (200, 6000)),
        # One long prompt.
        _case("prefill_long", "prefill", 1, (0, 0), (24576, 24576)),
        # The smallest draft: two short float32 sessions, five drafts each.
        _case("tree_tiny_f32", "tree", 2, (100, 500), (5, 5), width=5, hq=4, hkv=1, d=64, dtype="f32"),
        # A small interactive batch, eight drafts per session.
        _case("tree_8x2k", "tree", 8, (1500, 2600), (8, 8), width=8),
        # One layer of an agentic batch: 32 sessions of 8K to 32K tokens, 4 to 16 drafts.
        _case("tree_layer", "tree", 32, (8192, 32768), (4, 16), width=16),
        # Few sessions with wide trees, where the products count as much as the reads.
        _case("tree_wide", "tree", 4, (16384, 65536), (49, 64), width=64),
        # The end of a verified step of a 48-layer model, a small batch.
        _case("accept_8x8", "accept", 8, (1000, 2600), (0, 8), layers=48, width=8),
        # The same for a large batch with wider drafts.
        _case("accept_64x16", "accept", 64, (8192, 32768), (0, 16), layers=48, width=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(float(np.exp(rng.uniform(np.log(lo), np.log(hi))))))


def draw(rng):
    op = rng.choice(["prefill", "prefill", "tree", "tree", "accept"])
    length_seed = rng.randrange(1 << 30)
    hq, hkv, d = rng.choice(SHAPES)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    shape = {"hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "length_seed": length_seed}
    slow = 8 if dtype == "f32" else 1
    if op == "prefill":
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 16384)
        ctx = rng.choice([0, _log_int(rng, 1, 32768)])
        # at most a quarter of the long prompt's products, and 2 GB of K and V
        while batch * hi * (ctx + hi / 2) * hq * d * slow > 2.5e11 * 4 or \
                batch * (ctx + hi) * hkv * d * BYTES[dtype] > 1e9:
            batch, hi, ctx = max(1, batch // 2), max(1, hi * 3 // 4), ctx * 3 // 4
        return _case("", "prefill", batch, (rng.randint(0, ctx), ctx), (rng.randint(1, hi), hi), **shape)
    width = rng.choice([1, 64, rng.randint(2, 63), rng.randint(2, 16), rng.randint(2, 16)])
    least = rng.choice([0, 1])       # some sessions may bring nothing, of a large enough batch
    if op == "tree":
        batch = _log_int(rng, 1, 256)
        ctx = _log_int(rng, 1, 65536)
        while batch * ctx * hkv * d * BYTES[dtype] > 6e8 or batch * width * ctx * hq * d * slow > 1e11:
            batch, ctx = max(1, batch * 2 // 3), ctx * 4 // 5
        least = least if batch > 4 else 1
        return _case("", "tree", batch, (rng.randint(0, ctx), ctx), (rng.randint(least, width), width),
                     width=width, **shape)
    layers = rng.choice([1, 4, 24, 48])
    batch = _log_int(rng, 1, 256)
    while batch * width * layers * hkv * d * BYTES[dtype] > 48 * 64 * 16 * 4 * 128 * 2:
        batch, layers, width = max(1, batch // 2), max(1, layers * 3 // 4), max(1, width * 3 // 4)
    ctx = _log_int(rng, 1, 32768)
    return _case("", "accept", batch, (rng.randint(0, ctx), ctx), (least if batch > 4 else 1, width), layers=layers,
                 width=width, **shape)


# -- what a case consists of ---------------------------------------------------

def _counts(c):
    """(context tokens, new tokens) of every session."""
    r = np.random.Generator(np.random.PCG64(c["length_seed"]))
    ctx = r.integers(c["ctx_lo"], c["ctx_hi"], size=c["batch"], endpoint=True)
    new = r.integers(c["new_lo"], c["new_hi"], size=c["batch"], endpoint=True)
    return [int(x) for x in ctx], [int(x) for x in new]


def _pages(n):
    return -(-n // PAGE)


def _generator(seed, *coordinates):
    words = np.random.SeedSequence([int(seed), *[int(x) for x in coordinates]]).generate_state(2)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(words[0]) * (1 << 31) + int(words[1]))
    return g


def _numbers(seed, *coordinates):
    return np.random.Generator(np.random.PCG64(np.random.SeedSequence([int(seed), *coordinates])))


def _normal(c, shape, *key):
    return torch.randn(shape, generator=_generator(*key), device="cuda", dtype=torch.float32).to(TORCH[c["dtype"]])


def _cached(c, seed, lens):
    """K and V of every session's cached tokens, [tokens][KV heads][head dim] each."""
    return [tuple(_normal(c, (n, c["hkv"], c["d"]), seed, 1, i, kind) for kind in (0, 1))
            for i, n in enumerate(lens)]


def _trees(c, seed, new):
    """Attention masks [batch][width] of random trees: draft i's parent is an earlier draft
    or the context; bit j of mask i is set for i itself and its ancestors."""
    r = _numbers(seed, 2)
    masks = np.zeros((c["batch"], c["width"]), np.uint64)
    for b, n in enumerate(new):
        for i in range(n):
            parent = int(r.integers(-1, i)) if i else -1
            up = masks[b, parent] if parent >= 0 else np.uint64(0)
            masks[b, i] = up | (np.uint64(1) << np.uint64(i))
    return masks.view(np.int64)


def _paths(c, seed, new):
    """Accepted draft indices [batch][width]: ascending, a path down the tree."""
    r = _numbers(seed, 3)
    acc = np.zeros((c["batch"], c["width"]), np.int32)
    for b, n in enumerate(new):
        acc[b, :n] = np.sort(r.permutation(c["width"])[:n])
    return acc


def _i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")


def _inputs(c, seed):
    """The call's device inputs, without the cache."""
    ctx, new = _counts(c)
    s = {"case": c, "ctx": ctx, "new": new}
    hq, hkv, d, B, T = c["hq"], c["hkv"], c["d"], c["batch"], c["width"]
    if c["op"] == "prefill":
        starts = np.concatenate([[0], np.cumsum(new)])
        s["starts_host"] = [int(x) for x in starts]
        s["starts"] = _i32(starts)
        s["lens_host"] = [a + n for a, n in zip(ctx, new)]
        s["lens"] = _i32(s["lens_host"])
        s["q"] = _normal(c, (s["starts_host"][-1], hq, d), seed, 4)
        s["out"] = torch.zeros_like(s["q"])
    elif c["op"] == "tree":
        s["lens_host"] = ctx
        s["lens"] = _i32(ctx)
        s["drafts"] = _i32(new)
        s["masks"] = torch.from_numpy(_trees(c, seed, new)).cuda()
        s["q"] = _normal(c, (B, T, hq, d), seed, 4)
        s["kd"] = _normal(c, (B, T, hkv, d), seed, 5)
        s["vd"] = _normal(c, (B, T, hkv, d), seed, 6)
        s["out"] = torch.zeros_like(s["q"])
    else:
        s["lens"] = _i32(ctx)
        s["count"] = _i32(new)
        s["path"] = torch.from_numpy(_paths(c, seed, new)).cuda()
        s["kd"] = _normal(c, (c["layers"], B, T, hkv, d), seed, 5)
        s["vd"] = _normal(c, (c["layers"], B, T, hkv, d), seed, 6)
    return s


def _accept_table(c, seed, ctx):
    """Page table of an accept case: only the pages that drafts can reach exist (the pages
    before them are named by id 0 and not touched), in shuffled order."""
    spans = [(n // PAGE, _pages(n + c["width"])) for n in ctx]
    total = sum(hi - lo for lo, hi in spans)
    ids = _numbers(seed, 7).permutation(total).astype(np.int32)
    table = np.zeros((c["batch"], max(hi for _, hi in spans)), np.int32)
    at = 0
    for b, (lo, hi) in enumerate(spans):
        table[b, lo:hi] = ids[at:at + hi - lo]
        at += hi - lo
    return torch.from_numpy(table).cuda(), total


def _accept_pages(c, seed, pages):
    """What those pages hold before: [layers][pages][KV heads][K, V][head dim * 16]."""
    return _normal(c, (c["layers"], pages, c["hkv"], 2, c["d"] * PAGE), seed, 8)


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    if c["op"] == "accept":
        s["table"], pages = _accept_table(c, seed, s["ctx"])
        s["hot"] = _accept_pages(c, seed, pages)
        if own:
            from paper_2609_25782_amd.pool import HotColdPool
            s["pool"] = HotColdPool(c["layers"], c["hkv"], c["d"], c["dtype"], pages, 0, c["batch"],
                                    s["table"].shape[1])
            s["pool"].hot.copy_(s["hot"].reshape(-1).view(torch.uint8))
            s["hot"] = s["pool"].hot.view(TORCH[c["dtype"]]).view(s["hot"].shape)
        return s
    cached = _cached(c, seed, s["lens_host"])
    if not own:
        s["cached"] = cached
        return s
    from paper_2609_25782_amd.pool import HotColdPool
    need = [_pages(n) for n in s["lens_host"]]
    ids = _numbers(seed, 7).permutation(sum(need) + 16)
    pool = HotColdPool(1, c["hkv"], c["d"], c["dtype"], len(ids), 0, c["batch"], max(max(need), 1))
    at = 0
    for i, (n, p) in enumerate(zip(s["lens_host"], need)):
        sid = pool.create_session(n, [int(x) for x in ids[at:at + p]])
        at += p
        if n:
            pool.write_tokens(sid, 0, 0, *cached[i])
    torch.cuda.synchronize()
    s["pool"], s["table"] = pool, pool.page_table
    return s


# -- one pass ------------------------------------------------------------------

ROOM = 1 << 28   # scores held at once by the plain form


def _attend(q, k, v, allowed, scale):
    """Softmax attention of queries [n][G][d] over one KV head's k and v [m][d], float32;
    allowed(i0, i1) gives the [i1 - i0][m] table of who sees what, or None."""
    n, G, d = q.shape
    out = torch.empty((n, G, d), dtype=torch.float32, device=q.device)
    step = max(1, ROOM // max(1, G * k.shape[0]))
    for i in range(0, n, step):
        j = min(n, i + step)
        sc = torch.mm(q[i:j].reshape(-1, d), k.t()).view(j - i, G, -1) * scale
        sc.masked_fill_(~allowed(i, j)[:, None, :], float("-inf"))
        top = sc.amax(dim=-1, keepdim=True)
        top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
        w = sc.sub_(top).exp_()
        total = w.sum(dim=-1, keepdim=True)
        o = torch.mm(w.view((j - i) * G, -1), v).view(j - i, G, d)
        out[i:j] = torch.where(total > 0, o / total, torch.zeros_like(o))
    return out


def _plain_prefill(s):
    c = s["case"]
    G, scale = c["hq"] // c["hkv"], c["d"] ** -0.5
    for b, (k, v) in enumerate(s["cached"]):
        a, e, L = s["starts_host"][b], s["starts_host"][b + 1], s["lens_host"][b]
        q, k, v = s["q"][a:e].float(), k.float(), v.float()
        pos = torch.arange(L - (e - a), L, device=q.device)
        key = torch.arange(L, device=q.device)
        for h in range(c["hkv"]):
            o = _attend(q[:, h * G:(h + 1) * G], k[:, h].contiguous(), v[:, h].contiguous(),
                        lambda i, j: key[None, :] <= pos[i:j, None], scale)
            s["out"][a:e, h * G:(h + 1) * G] = o.to(s["out"].dtype)
    return s["out"]


def _plain_tree(s):
    c = s["case"]
    G, scale = c["hq"] // c["hkv"], c["d"] ** -0.5
    for b, (k, v) in enumerate(s["cached"]):
        n = s["new"][b]
        if n == 0:
            continue
        q = s["q"][b, :n].float()
        k = torch.cat([k.float(), s["kd"][b, :n].float()])
        v = torch.cat([v.float(), s["vd"][b, :n].float()])
        bit = torch.arange(n, device=q.device)
        tree = ((s["masks"][b, :n, None] >> bit[None, :]) & 1) != 0
        table = torch.cat([torch.ones((n, s["lens_host"][b]), dtype=torch.bool, device=q.device), tree], dim=1)
        for h in range(c["hkv"]):
            o = _attend(q[:, h * G:(h + 1) * G], k[:, h].contiguous(), v[:, h].contiguous(),
                        lambda i, j: table[i:j], scale)
            s["out"][b, :n, h * G:(h + 1) * G] = o.to(s["out"].dtype)
    return s["out"]


def _plain_accept(s):
    c = s["case"]
    B, T, d, x = c["batch"], c["width"], c["d"], 16 // BYTES[c["dtype"]]
    j = torch.arange(T, device="cuda")
    live = j[None, :] < s["count"][:, None]
    row = torch.arange(B, device="cuda")[:, None].expand(B, T)[live]
    pos = (s["lens"][:, None].long() + j[None, :])[live]
    src = s["path"].long()[live]
    page, slot = s["table"].long()[row, pos // PAGE], pos % PAGE
    hot = s["hot"]
    k = hot[:, :, :, 0].view(c["layers"], -1, c["hkv"], d // x, PAGE, x)
    v = hot[:, :, :, 1].view(c["layers"], -1, c["hkv"], d, PAGE)
    # the two index tensors stand apart in the subscript, so their dimension leads
    k[:, page, :, :, slot] = s["kd"][:, row, src].view(c["layers"], -1, c["hkv"], d // x, x).transpose(0, 1)
    v[:, page, :, :, slot] = s["vd"][:, row, src].transpose(0, 1)
    return hot


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"prefill": _plain_prefill, "tree": _plain_tree, "accept": _plain_accept}[op](s)
    if op == "prefill":
        return s["pool"].prefill(0, s["q"], s["starts"], s["lens"], page_table=s["table"], out=s["out"])
    if op == "tree":
        return s["pool"].tree_decode(0, s["q"], s["kd"], s["vd"], s["masks"], s["lens"], draft_lens=s["drafts"],
                                     page_table=s["table"], out=s["out"])
    s["pool"].accept_drafts(0, s["table"], s["lens"], s["path"], s["count"], s["kd"], s["vd"])
    return s["hot"]


def work(case):
    c = case
    ctx, new = _counts(c)
    e = BYTES[c["dtype"]]
    token = 2 * c["hkv"] * c["d"] * e          # K and V of one token of one layer
    query = 2 * c["hq"] * c["d"] * e           # a query and its output
    if c["op"] == "accept":
        n = sum(new)
        return {"bytes": 2 * n * c["layers"] * token + 4 * n, "flops": 0}
    read = sum(a + n for a, n in zip(ctx, new) if n) * token + sum(new) * query
    if c["op"] == "prefill":
        pairs = sum(n * a + n * (n + 1) // 2 for a, n in zip(ctx, new))
    else:
        pairs = sum(n * (a + 1) for a, n in zip(ctx, new))
    return {"bytes": read, "flops": 4 * c["hq"] * c["d"] * pairs}


# -- the definition, in 64 bits ------------------------------------------------

def _softmax_average(q, k, v, seen):
    """One query head: q [n][d], k and v [m][d], seen [n][m]; all float64."""
    weights = torch.matmul(k, q.t().contiguous()).t() / (q.shape[1] ** 0.5)
    weights = torch.where(seen, weights, torch.full_like(weights, -float("inf")))
    norm = torch.logsumexp(weights, dim=1, keepdim=True)
    weights = torch.exp(weights - torch.where(torch.isinf(norm), torch.zeros_like(norm), norm))
    return torch.matmul(weights, v)


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "accept":
        table, pages = _accept_table(c, seed, s["ctx"])
        hot = _accept_pages(c, seed, pages).double()
        x = 16 // BYTES[c["dtype"]]
        dim = torch.arange(c["d"], device="cuda")
        entries, path = table.cpu().numpy(), s["path"].cpu().numpy()
        for b, n in enumerate(s["new"]):
            for j in range(n):
                at = s["ctx"][b] + j
                p, t = int(entries[b, at // PAGE]), at % PAGE
                hot[:, p, :, 0, ((dim // x) * PAGE + t) * x + dim % x] = s["kd"][:, b, int(path[b, j])].double()
                hot[:, p, :, 1, dim * PAGE + t] = s["vd"][:, b, int(path[b, j])].double()
        return hot
    G = c["hq"] // c["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    masks = s["masks"].cpu().numpy().view(np.uint64) if c["op"] == "tree" else None
    cached = _cached(c, seed, s["lens_host"])
    for b in range(c["batch"]):
        n, total = s["new"][b], s["lens_host"][b]
        if n == 0:
            continue
        k, v = (x.double() for x in cached[b])
        if c["op"] == "tree":
            k, v = torch.cat([k, s["kd"][b, :n].double()]), torch.cat([v, s["vd"][b, :n].double()])
            q, o = s["q"][b, :n], out[b, :n]
            bits = [[bool((int(m) >> j) & 1) for j in range(n)] for m in masks[b, :n]]
            tail = torch.tensor(bits, dtype=torch.bool, device="cuda")
        else:
            a = s["starts_host"][b]
            q, o = s["q"][a:a + n], out[a:a + n]
            tail = None
        for i in range(0, n, 4096):
            m = min(n, i + 4096)
            if tail is None:
                rows = torch.arange(i, m, device="cuda")[:, None] + (total - n)
                seen = torch.arange(total, device="cuda")[None, :] <= rows
            else:
                seen = torch.ones((m - i, total + n), dtype=torch.bool, device="cuda")
                seen[:, total:] = tail[i:m]
            for h in range(c["hq"]):
                o[i:m, h] = _softmax_average(q[i:m, h].double(), k[:, h // G].contiguous(),
                                             v[:, h // G].contiguous(), seen)
    return out
