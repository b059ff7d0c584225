"""The paged operators together, as a server loop uses them (paged_run): at every layer of every forward the keys and values that the
tables lead to are the projection's rows, normed and turned, and the attention is that of each request alone, by the 64-bit oracle.
Bounds: those of test_gpu_paged.py."""
import numpy as np
import pytest

from gpu_common import requires_gpu
from oracle import paged_oracle as O

U = 2.0 ** -8


@requires_gpu
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 64, 16), (4, 4, 128, 64)])
def test_server_loop_against_the_oracle(heads, kv, dim, page):
    from paper_2511_21759_b200 import paged_run as R
    layers = R.Layers(2, heads, kv, dim, seed=3)
    freq, mag = O.frequencies(dim)
    looked = []
    stale = {}            # (layer, request, position) -> K and V the oracle expects there, as stored

    def seen(server, batch, first, count, layer, qkv, q, out):
        f = lambda t: t.float().cpu().numpy()
        x = f(qkv).reshape(-1, heads + 2 * kv, dim)
        pool, table = f(server.cache.kv)[layer], batch.table.cpu().numpy()
        qs, o = f(q), f(out)
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(first, count)])
        norm = lambda part, gain: O.norm_rope(part, gain.cpu().numpy(), 1e-6, pos, freq, mag, False)
        wq, wk = norm(x[:, :heads], layers.q_gain[layer]), norm(x[:, heads:heads + kv], layers.k_gain[layer])
        # rounded once; the few fp32 roundings in front of it are 2^-20 of a pair's two terms, each below sqrt(2) of the largest result
        slack = lambda w: U * np.abs(w) + 2.0 ** -20 * 2 * 2 ** 0.5 * np.abs(w).max()
        assert (np.abs(qs - wq) <= slack(wq)).all()
        r = 0
        for s, (a, n, total) in enumerate(zip(first, count, server.total)):
            at = lambda i: pool[i, table[s, np.arange(total) // page], :, np.arange(total) % page] if total else np.zeros((0, kv, dim), np.float32)
            k, v = at(0), at(1)
            assert (np.abs(k[a:a + n] - wk[r:r + n]) <= slack(wk)[r:r + n]).all() and np.array_equal(v[a:a + n], x[r:r + n, heads + kv:])
            for p in range(total):                           # positions outside the rows keep what an earlier forward stored
                if a <= p < a + n:
                    stale[layer, s, p] = (k[p].copy(), v[p].copy())
                else:
                    assert np.array_equal(stale[layer, s, p][0], k[p]) and np.array_equal(stale[layer, s, p][1], v[p]), (layer, s, p)
            want, _, m, size = O.attention(qs[r:r + n], k, v, pos[r:r + n])
            d = (dim * 2.0 ** -24 * size)[..., None]
            tol = U * np.abs(want) + (U + 2.2 * d + 2.0 ** -20) * m * 1.01
            assert (np.abs(o[r:r + n] - want) <= tol).all(), (layer, s)
            r += n
        held = [p for s, total in enumerate(server.total) for p in table[s, :O.pages_of(total, page)]]
        assert len(set(held)) == len(held)
        looked.append((layer, sum(count)))

    server = R.run(layers, requests=3, blocks=2, block=16, page_size=page, steps=1, seen=seen, say=lambda *_: None)
    assert len(looked) == 2 * 2 * 2 and server.length == server.total
    # everything given back: all pages are free again
    server.total = [0] * len(server.total)
    server.forward("refresh")
    assert sorted(server.free.cpu().tolist()) == list(range(server.cache.n_pages))
