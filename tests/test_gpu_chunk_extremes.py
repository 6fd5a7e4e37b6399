"""Prompt and tree attention where numbers reach the ends of their range: weights that underflow
beside values near the largest, and scores of minus infinity."""

import numpy as np
import pytest
import torch

from chunk_reference import Sessions, attend, check, i32, mask_tensor

pytestmark = pytest.mark.gpu

HUGE = 2.0 ** 127     # of both types
LOW = -200.0          # a score whose weight beside a score of 0 is 2^-288: no float32


def scored(s, b, scores, heads, n):
    """Session b's keys score `scores` under n queries of ones in the first dim (scale 1)."""
    k = torch.zeros_like(s.k[b])
    k[0, :, :, 0] = torch.tensor(scores)[:, None]
    s.k[b] = k
    s.pool.write_tokens_layers(b, 0, 0, s.k[b].cuda(), s.v[b].cuda())
    q = torch.zeros((n, heads, s.d), dtype=s.k[b].dtype)
    q[:, :, 0] = 1
    return q


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("tokens", [300, 9000])     # inside one tile's blocks, and cut between workers
@pytest.mark.parametrize("high", [0, 70])           # the tokens that count stand first, or in the middle
def test_underflowing_weights_add_nothing(tokens, high, dtype, d):
    """Sixteen tokens score 0, the others so low that their weights are 0; some of those hold values
    near the largest number.  Their share of the output is below the smallest number there is."""
    s = Sessions([tokens], 4, 1, d, dtype, seed=50)
    scores = [0.0 if high <= t < high + 16 else LOW for t in range(tokens)]
    s.v[0][0, tokens - 1, 0, 3] = HUGE
    s.v[0][0, tokens // 2, 0, 5] = -HUGE
    s.v[0][0, high + 20, 0, 9] = HUGE
    q = scored(s, 0, scores, 4, 1)
    ref, bound = attend(q, s.k[0][0], s.v[0][0], np.ones((1, tokens), bool), 1.0, dtype)
    assert np.abs(ref).max() < 4
    check(s.pool.prefill(0, q.cuda(), i32([0, 1]), i32([tokens]), scale=1.0), ref, bound, what="prefill")
    # the same as a draft that sees the context alone, and as one that sees drafts like that as well
    kd, vd = torch.zeros((1, 2, 1, d), dtype=q.dtype), s.normal(1, 2, 1, d)
    kd[0, :, 0, 0] = LOW
    vd[0, 1, 0, 7] = HUGE
    got = s.pool.tree_decode(0, q.expand(2, 4, d)[None].contiguous().cuda(), kd.cuda(), vd.cuda(), mask_tensor([[0, 3]]),
                             i32([tokens]), scale=1.0)
    for i in range(2):
        check(got[0, i:i + 1], ref, bound, what="draft %d" % i)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_scores_of_minus_infinity_in_prompts(dtype, d):
    """A query all of whose scores are minus infinity has no softmax: NaN, as from decode; beside any
    other score such a token has no weight."""
    first, n = 70, 150
    s = Sessions([n, 9000, 9000], 4, 1, d, dtype, seed=51)
    qs, refs, bounds = [], [], []
    for b, (tokens, new, low) in enumerate(((n, n, range(first)), (9000, 2, range(9000)), (9000, 2, range(16, 9000)))):
        scores = s.normal(tokens).float().tolist()
        for t in low:
            scores[t] = float("-inf")
        q = scored(s, b, scores, 4, new)
        q[:, :, 1:] = 0.5          # against zeros
        seen = np.arange(tokens)[None, :] <= (tokens - new + np.arange(new))[:, None]
        seen[:, list(low)] = False
        ref, bound = attend(q, s.k[b][0], s.v[b][0], seen, 1.0, dtype)
        ref[~seen.any(axis=1)] = np.nan
        qs.append(q), refs.append(ref), bounds.append(bound)
    q, ref, bound = torch.cat(qs), np.concatenate(refs), np.concatenate(bounds)
    assert np.isnan(ref).any(axis=(1, 2)).tolist() == [True] * first + [False] * (n - first) + [True] * 2 + [False] * 2
    starts = [0, n, n + 2, n + 4]
    got = s.pool.prefill(0, q.cuda(), i32(starts), i32([n, 9000, 9000]), scale=1.0)
    check(got, ref, bound)
    alone = s.pool.prefill(0, q[n:n + 2].contiguous().cuda(), i32([0, 2]), i32([9000]),
                           page_table=s.pool.page_table[1:2].contiguous(), scale=1.0)
    assert alone.isnan().all()
    dec = s.pool.decode(0, q[[0, n + 1]].contiguous().cuda(), i32([1, 9000]),
                        page_table=s.pool.page_table[:2].contiguous(), scale=1.0)
    assert dec.isnan().all()


@pytest.mark.parametrize("width", [6, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [0, 30, 9000])
def test_scores_of_minus_infinity_in_trees(ctx, dtype, width):
    """The same for drafts: NaN where everything that a draft sees scores minus infinity, zeros
    where it sees nothing, and no weight beside other scores."""
    d, hq = 64, 4
    s = Sessions([ctx], hq, 1, d, dtype, seed=52)
    q = torch.zeros((1, width, hq, d), dtype=s.k[0].dtype)
    q[..., 0] = 1
    if ctx:
        scored(s, 0, [float("-inf")] * ctx, hq, 1)
    kd, vd = torch.zeros((1, width, 1, d), dtype=q.dtype), s.normal(1, width, 1, d)
    kd[0, :, 0, 0] = float("-inf")
    kd[0, 1, 0, 0] = 2.0
    last = 1 << (width - 1)
    masks = [1, 2, 3, 0, last, last | 2] + [last | 1] * (width - 6)
    got = s.pool.tree_decode(0, q.cuda(), kd.cuda(), vd.cuda(), mask_tensor([masks]), i32([ctx]), scale=1.0)
    ref, bound = np.zeros(tuple(q.shape)), np.zeros(tuple(q.shape))
    for i, m in enumerate(masks):
        if m & 2:                        # draft 1 alone counts
            ref[0, i], bound[0, i] = (x[0] for x in attend(q[0, i:i + 1], kd[0, 1:2], vd[0, 1:2], np.ones((1, 1), bool), 1.0, dtype))
        elif m or ctx:
            ref[0, i] = np.nan
    check(got, ref, bound)
