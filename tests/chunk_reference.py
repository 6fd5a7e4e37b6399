"""Float64 definition of prompt and tree attention, with error bounds, and pools to compare
them with.

Error bounds, per output element, derived from the number formats (u = half a step:
2^-8 for bf16, 2^-24 for float32), with A = sum w |v| / sum w the average magnitude:
  scores   a float32 product of `d` terms is off by at most (d + 2) 2^-24 sum |q_i k_i|, its
           exponent by that times the scale, plus the rounding of s c - m c and of the
           exponential itself: a relative error of a weight of
           e = |scale| (d + 2) 2^-24 max sum |q_i k_i| + 2^-22 (2 + |scale| max |s|)
  weights  bf16 pools round each to bf16: u_w = 2^-8 (float32: 0)
  sums     T terms in float32, in numerator and denominator: (T + 64) 2^-24 each; the
           64 covers rescales and joins of partial results
  output   one rounding, u |out|
so |got - out| <= (2 e + u_w + 2 (T + 64) 2^-24) A + u |out|, with 1 % on top for products
of these errors.
"""

import numpy as np
import torch

from paper_2609_25782_amd.pool import HotColdPool

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
PAGE = 16


def pages_for(n):
    return -(-n // PAGE)


def attend(q, k, v, seen, scale, dtype):
    """q [n][Hq][d], k, v [m][Hkv][d] (CPU tensors of the pool dtype), seen bool [n][m].
    Returns (out, bound) float64 [n][Hq][d]: only attended tokens enter, whatever the others hold."""
    n, hq, d = q.shape
    hkv, G = k.shape[1], hq // k.shape[1]
    out = np.zeros((n, hq, d))
    bound = np.zeros((n, hq, d))
    q, k, v = (t.double().numpy() for t in (q, k, v))
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    uw = 2.0 ** -8 if dtype == "bf16" else 0.0
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if len(at) == 0:
            continue
        T = len(at)
        for g in range(hkv):
            kk, vv, qq = k[at, g], v[at, g], q[i, g * G:(g + 1) * G]
            s = qq @ kk.T                              # [G][T]
            mag = np.abs(qq) @ np.abs(kk).T
            z = s * scale
            w = np.exp(z - z.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            o = w @ vv
            A = w @ np.abs(vv)
            e = abs(scale) * (d + 2) * 2.0 ** -24 * mag.max(axis=1) + \
                2.0 ** -22 * (2 + abs(scale) * np.abs(s).max(axis=1))
            out[i, g * G:(g + 1) * G] = o
            bound[i, g * G:(g + 1) * G] = 1.01 * ((2 * e[:, None] + uw + 2 * (T + 64) * 2.0 ** -24) * A +
                                                  u * np.abs(o))
    return out, bound


def check(got, out, bound, what=""):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    assert got.shape == out.shape
    nan = np.isnan(out)
    assert np.array_equal(np.isnan(got), nan), "%s: NaN in other places" % what
    inf = np.isinf(out)
    assert np.array_equal(got[inf], out[inf]), "%s: infinities differ" % what
    ok = ~(nan | inf)
    err = np.abs(got[ok] - out[ok])
    worst = float((err - bound[ok]).max()) if err.size else -1.0
    assert worst <= 0, "%s: off by %g beyond the bound (largest error %g)" % (what, worst, err.max())


class Sessions:
    """A pool with sessions of given lengths on shuffled pages, and their K and V on the CPU."""

    def __init__(self, lens, hq, hkv, d, dtype, seed=0, layers=1, spare=8, stride=0, cold=0, poison=True,
                 value=1.0, max_sessions=0):
        self.lens, self.hq, self.hkv, self.d, self.dtype = list(lens), hq, hkv, d, dtype
        self.g = torch.Generator().manual_seed(seed)
        need = [pages_for(n) for n in lens]
        self.pool = HotColdPool(layers, hkv, d, dtype, sum(need) + spare, cold, max(len(lens), max_sessions, 1),
                                max(max(need + [1]), stride))
        if poison:     # slots that no token was written to hold NaN
            self.pool.hot.view(TORCH[dtype]).fill_(float("nan"))
        order = torch.randperm(sum(need) + spare, generator=self.g).tolist()
        self.k, self.v, self.pages, at = [], [], [], 0
        for n, p in zip(lens, need):
            self.pages.append(order[at:at + p])
            sid = self.pool.create_session(n, order[at:at + p])
            at += p
            k, v = self.normal(layers, n, hkv, d, value=value), self.normal(layers, n, hkv, d)
            self.k.append(k)
            self.v.append(v)
            if n:
                self.pool.write_tokens_layers(sid, 0, 0, k.cuda(), v.cuda())

    def normal(self, *shape, value=1.0):
        return (torch.randn(shape, generator=self.g) * value).to(TORCH[self.dtype])

    def write(self, b, layer, tok):
        """Write token `tok` of session b again, from self.k and self.v."""
        self.pool.write_tokens(b, layer, tok, self.k[b][layer, tok:tok + 1].cuda().contiguous(),
                               self.v[b][layer, tok:tok + 1].cuda().contiguous())


def i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def prefill_reference(s, q, starts, lens, layer=0, scale=None):
    """(out, bound) of a prompt call over sessions 0.. of `s`; queries of no row stay 0."""
    out, bound = np.zeros(tuple(q.shape)), np.zeros(tuple(q.shape))
    scale = s.d ** -0.5 if scale is None else scale
    for b, L in enumerate(lens):
        a, e = starts[b], starts[b + 1]
        if e <= a:
            continue
        n = e - a
        seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
        out[a:e], bound[a:e] = attend(q[a:e], s.k[b][layer][:L], s.v[b][layer][:L], seen, scale, s.dtype)
    return out, bound


def tree_reference(s, q, kd, vd, masks, lens, drafts, layer=0, scale=None):
    out, bound = np.zeros(tuple(q.shape)), np.zeros(tuple(q.shape))
    scale = s.d ** -0.5 if scale is None else scale
    for b, (C, n) in enumerate(zip(lens, drafts)):
        if n == 0:
            continue
        bits = np.array([[(int(m) >> j) & 1 for j in range(n)] for m in masks[b][:n]], bool)
        seen = np.concatenate([np.ones((n, C), bool), bits], axis=1)
        k, v = torch.cat([s.k[b][layer][:C], kd[b, :n]]), torch.cat([s.v[b][layer][:C], vd[b, :n]])
        out[b, :n], bound[b, :n] = attend(q[b, :n], k, v, seen, scale, s.dtype)
    return out, bound


def random_tree(rng, n, width):
    """Masks of a random tree of n drafts: itself and its ancestors."""
    masks = [0] * width
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        masks[i] = (masks[parent] if parent >= 0 else 0) | (1 << i)
    return masks


def mask_tensor(masks):
    return torch.from_numpy(np.array(masks, np.uint64).view(np.int64)).cuda()
