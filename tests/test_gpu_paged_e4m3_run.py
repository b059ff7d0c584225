"""The operators of a cache in 8 bits together, as a server loop uses them (paged_run): at every layer of every forward the codes and scales
that the tables lead to are the projection's rows, normed, turned and quantised, those of earlier forwards are what they were (or are rounded
once more where their block's scale has grown), rows read back are what the codes stand for, and the attention is that of each request alone,
by the 64-bit oracle.  Bounds: those of test_gpu_paged_e4m3.py and, for q, of test_gpu_paged.py."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O
from test_gpu_paged_e4m3 import E4M3, U, VALUES, check, codes_of


@requires_gpu
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 64, 16), (4, 4, 128, 64)])
def test_server_loop_against_the_oracle(heads, kv, dim, page):
    from paper_2511_21759_b200 import paged_run as R
    layers = R.Layers(2, heads, kv, dim, seed=3)
    freq, mag = O.frequencies(dim)
    looked = []
    before = {}           # (layer, request) -> values of K and V at its positions, exponents of its blocks, after the layer's last forward

    def seen(server, batch, first, count, layer, qkv, q, out):
        f = lambda t: t.float().cpu().numpy()
        cache = server.cache
        x = f(qkv).reshape(-1, heads + 2 * kv, dim).astype(np.float64)
        codes, scales, table = codes_of(cache.kv[layer]), f(cache.scales)[layer].astype(np.float64), batch.table.cpu().numpy()
        qs = f(q)
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(first, count)])
        norm = lambda part, gain: O.norm_rope(part, gain.cpu().numpy(), 1e-6, pos, freq, mag, False)
        wq, wk = norm(x[:, :heads], layers.q_gain[layer]), norm(x[:, heads:heads + kv], layers.k_gain[layer])
        slack = lambda w: 2.0 ** -20 * 2 * 2 ** 0.5 * np.abs(w).max()
        assert (np.abs(qs - wq) <= U * np.abs(wq) + slack(wq)).all()
        back_k, back_v = (f(t) for t in cache.load(layer, batch))
        want = [wk, x[:, heads + kv:]]
        keys, values, vscale = [], [], []
        r = 0
        for s, (a, n, total) in enumerate(zip(first, count, server.total)):
            j = np.arange(total)
            pg, off = table[s, j // page], j % page
            got = [(VALUES[codes[i, pg, :, off]] * scales[i, pg, :, off // O.BLOCK][..., None]).reshape(total, kv, dim) for i in range(2)]
            exps = [np.log2(scales[i, pg, :, off // O.BLOCK]).reshape(total, kv)[::O.BLOCK] for i in range(2)]
            for i in range(2):
                e = np.repeat(exps[i], O.BLOCK, 0)[:total][..., None]
                assert np.array_equal(e, np.round(e))
                w = want[i][r:r + n]
                lost = slack(wk) * 1.1 if i == 0 else 0.0
                assert (np.abs(got[i][a:a + n] - w) <= np.maximum(2.0 ** -4 * np.abs(w), 2.0 ** (e[a:a + n] - 10)) + lost).all(), (layer, s, i)
                if (layer, s) in before:                     # positions outside the rows, under the scale of now
                    old = before[layer, s][0][i]
                    keep = [p for p in range(min(total, len(old))) if not a <= p < a + n]
                    assert np.array_equal(got[i][keep], O.e4m3_round(old[keep] / 2.0 ** e[keep]) * 2.0 ** e[keep]), (layer, s, i)
                for b in range(O.pages_of(total, O.BLOCK) if i else 0):       # V's exponents: of what is written, and of what is kept
                    p0, p1 = b * O.BLOCK, min(total, (b + 1) * O.BLOCK)
                    rows = [p for p in range(p0, p1) if a <= p < a + n]
                    for h in range(kv if rows else 0):
                        e1 = O.exponent_for(np.abs(x[[r + p - a for p in rows], heads + kv + h]).max())
                        if len(rows) < p1 - p0:
                            e1 = max(e1, before[layer, s][1][i][b, h])
                        assert exps[i][b, h] == e1, (layer, s, b, h)
            assert np.array_equal(back_k[r:r + n], got[0][a:a + n]) and np.array_equal(back_v[r:r + n], got[1][a:a + n])
            before[layer, s] = (got, exps)
            keys.append(got[0]), values.append(got[1]), vscale.append(2.0 ** np.repeat(exps[1], O.BLOCK, 0)[:total])
            r += n
        start = np.concatenate([[0], np.cumsum(count)])
        check(out.view(-1, heads, dim), None, qs, keys, values, vscale, start, first, dim)
        held = [p for s, total in enumerate(server.total) for p in table[s, :O.pages_of(total, page)]]
        assert len(set(held)) == len(held)
        looked.append((layer, sum(count)))

    server = R.run(layers, requests=3, blocks=2, block=16, page_size=page, steps=1, seen=seen, say=lambda *_: None, dtype=E4M3)
    assert len(looked) == 2 * 2 * 2 and server.length == server.total and server.cache.kv.dtype is torch.float8_e4m3fn
    # everything given back: all pages are free again
    server.total = [0] * len(server.total)
    server.forward("refresh")
    assert sorted(server.free.cpu().tolist()) == list(range(server.cache.n_pages))
