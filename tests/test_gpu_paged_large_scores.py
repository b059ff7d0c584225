"""Paged attention of scores so large that one key takes all the weight: the output is that key's V.

Bounds, derived before the first run.  A score's fp32 sum of head_dim exact products and its product with the scale are off by up to
d = (head_dim + 2) 2^-24 of the largest sum |q k| times the scale (as in test_gpu_paged).  Where the oracle's largest score leads the next
by more than 2 d + 20 the same key leads in the kernel, by more than 20: the others' weights are below e^-20 each, which moves the output
by less than len e^-20 2 max|V| < 1e-5 (len < 400, |V| < 5).  The leading key's weight is rounded to bf16 once while the sum is not, a
factor within 2^-8 of 1; the output is rounded to bf16, half a step within 2^-8 of its value."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O
from test_gpu_paged import U, _setup


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [3, 45, 90])
@pytest.mark.parametrize("scale", [3e4, -3e4])
@pytest.mark.parametrize("size", [1.0, 30.0])
def test_the_leading_key_takes_all(size, scale, new, D, columns):
    rng = np.random.default_rng(31)
    H, KV = 4, 2
    lens, counts = [333, 94], [new, new]
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, H, KV, D, 16, scale=size, columns=columns)
    lse = torch.empty(2 * new, H, device="cuda")
    out = cache.attention(0, b, q, lse=lse, scale=scale, right=0).float().cpu().numpy()
    lse = lse.cpu().numpy()
    assert cache.status() == 0
    led = 0
    for s in range(len(lens)):
        for i in range(counts[s]):
            ok = O.visible(lens[s], firsts[s] + i, right=0)
            for h in range(H):
                k, v = keys[s][ok, h * KV // H].astype(np.float64), values[s][ok, h * KV // H]
                x = qf[start[s] + i, h].astype(np.float64)
                scores = k @ x * scale
                d = (D + 2) * 2.0 ** -24 * (np.abs(k) @ np.abs(x)).max() * abs(scale)
                best = int(scores.argmax())
                if len(scores) > 1 and scores[best] - np.delete(scores, best).max() <= 2 * d + 20:
                    continue
                led += 1
                got = out[start[s] + i, h]
                assert (np.abs(got - v[best]) <= (2 * U + U * U) * np.abs(v[best]) + 1e-5).all(), (s, i, h)
                assert abs(lse[start[s] + i, h] - scores[best]) <= d + 2.0 ** -21 * (1 + abs(scores[best])), (s, i, h)
    assert led >= 0.9 * len(qf) * H, led
    cache.close()
