"""Prompt and tree attention where numbers reach the ends of their range: weights that underflow
beside values near the largest."""

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
