"""The paged K/V cache's operators against the 64-bit oracle: block tables and slot maps (whole numbers, equal), norm +
rotation + store, attention over pages.

Bounds, derived before the first run.
  norm_rope_store: the result is rounded once to bf16, half a step = 2^-8 of its value; in front of it a handful of fp32
  roundings of the pair's two terms (norm, two products, a sum, sine and cosine of an angle exact to 2^-32 of a turn), taken
  together below 2^-20 of |a| + |b| (after the norm).
  attention: the output's rounding is 2^-8 of its value; P rounded to bf16 is off by up to 2^-8 of itself, the weighted
  values by up to 2^-8 sum w|v|; a score's fp32 sum of head_dim exact products is off by up to head_dim 2^-24 sum|q k| scale
  =: d, which moves numerator and denominator by a factor e^d each; log-sum-exp by d and a rounding of fp32."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O

U = 2.0 ** -8


def paged():
    from paper_2511_21759_b200 import paged as P
    return P


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(rng, *shape, scale=1.0):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(scale)).to(torch.bfloat16)
    return t, t.float().numpy()


# ---- layout -----------------------------------------------------------------------------------------------------------

def _check_layout(rng, page, before, after, first, count, spare=3, pad=4):
    P = paged()
    before, after, first, count = (np.asarray(v, np.int32) for v in (before, after, first, count))
    held = [O.pages_of(int(n), page) for n in before]
    need = [O.pages_of(int(n), page) for n in after]
    n_pages = max(sum(held), sum(need)) + spare
    n_pages = max(n_pages, 1)
    width = max(held + need + [1])
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(before), width), -7, np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    free = np.full(n_pages, -9, np.int32)
    free[: n_pages - at] = order[at:]
    rows = int(count.sum()) + pad
    want = O.layout(table, free, before, after, first, count, page, rows)
    cache = P.PagedCache(1, 1, 1, 64, page, n_pages)
    b = P.Batch(cache, table=dev(table), free_pages=dev(free), len_before=dev(before), len_after=dev(after), first=dev(first),
                count=dev(count), max_rows=rows)
    for _ in range(2):                       # a call that is repeated gives the same: its inputs are still there
        cache.layout(b)
        assert cache.status() == 0
        for got, w, name in zip((b.table, b.free_pages, b.row_start, b.row_seq, b.row_pos, b.row_slot), want,
                                ("table", "free", "row_start", "row_seq", "row_pos", "row_slot")):
            assert np.array_equal(got.cpu().numpy(), w), name
    # no page twice
    held_now = [p for s, n in enumerate(need) for p in want[0][s, :n]]
    assert sorted(held_now + list(want[1][: n_pages - sum(need)])) == list(range(n_pages))
    cache.close()


@requires_gpu
@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("seqs", [1, 2, 31, 257, 1024])
def test_layout_of_random_forwards(seqs, page):
    rng = np.random.default_rng(seqs * 7 + page)
    hi = 5 * page if seqs < 100 else 2 * page
    before = rng.integers(0, hi + 1, seqs)
    after = rng.integers(0, hi + 1, seqs)
    keep = rng.random(seqs) < 0.4
    after[keep] = before[keep]
    count = np.minimum(after, rng.integers(0, 40, seqs))
    first = (after - count) * rng.integers(0, 2, seqs)
    _check_layout(rng, page, before, after, first, count)


@requires_gpu
@pytest.mark.parametrize("before,after", [([0], [0]), ([0], [1]), ([1], [0]), ([16], [17]), ([17], [16]), ([0, 0, 0], [0, 33, 0]),
                                          ([100, 0], [0, 100]), ([0, 100], [100, 0]), ([48, 48, 48], [0, 0, 0]), ([0], [16 * 1200])])
def test_layout_at_its_edges(before, after):
    n = len(before)
    for full in (False, True):
        count = after if full else [min(a, 3) for a in after]
        first = [a - c for a, c in zip(after, count)]
        _check_layout(np.random.default_rng(3), 16, before, after, first, count, spare=0, pad=0 if full else 300)


@requires_gpu
def test_layout_refuses_what_does_not_fit_and_changes_nothing():
    P = paged()
    from paper_2511_21759_b200 import binding as B
    cases = [  # before, after, first, count -> status
        ([16, 16], [16, 200], [0, 0], [1, 1], B.ODB_ERR_ARG),            # longer than a table row
        ([16, -1], [16, 16], [0, 0], [1, 1], B.ODB_ERR_ARG),
        ([16, 16], [16, -5], [0, 0], [1, 1], B.ODB_ERR_ARG),
        ([16, 16], [16, 16], [0, 10], [1, 7], B.ODB_ERR_ARG),            # rows behind the length
        ([16, 16], [16, 16], [-1, 0], [1, 1], B.ODB_ERR_ARG),
        ([16, 16], [16, 16], [0, 0], [1, -1], B.ODB_ERR_ARG),
        ([16, 16], [64, 64], [0, 0], [1, 1], B.ODB_ERR_WORKSPACE),       # eight pages of five
        ([64, 64], [0, 0], [0, 0], [0, 0], B.ODB_ERR_WORKSPACE),         # held more than there are
        ([16, 16], [32, 32], [0, 0], [16, 17], B.ODB_ERR_SHAPE),         # more rows than the maps have
        ([2 ** 31 - 1, 0], [0, 0], [0, 0], [0, 0], B.ODB_ERR_ARG),
        ([16, 16], [16, 16], [2 ** 31 - 1, 0], [2 ** 31 - 1, 0], B.ODB_ERR_ARG),
    ]
    cache = P.PagedCache(1, 1, 1, 64, 16, 5)
    for before, after, first, count, status in cases:
        table = np.array([[0, -1, -1, -1], [1, -1, -1, -1]], np.int32)
        free = np.array([2, 3, 4, -1, -1], np.int32)
        i32 = lambda v: dev(np.asarray(v, np.int32))
        b = P.Batch(cache, table=dev(table), free_pages=dev(free), len_before=i32(before), len_after=i32(after), first=i32(first),
                    count=i32(count), max_rows=32)
        cache.layout(b)
        assert cache.status() == status, (before, after, first, count)
        assert cache.status() == 0
        assert np.array_equal(b.table.cpu().numpy(), table) and np.array_equal(b.free_pages.cpu().numpy(), free)
        assert (b.row_start == 0).all() and (b.row_seq == -1).all() and (b.row_pos == -1).all() and (b.row_slot == -1).all()
    # a table with a page that is none: its rows have no slot
    b = P.Batch(cache, table=i32([[0, 77, -1, -1], [1, -1, -1, -1]]), free_pages=i32([2, 3, 4, -1, -1]), len_before=i32([32, 16]),
                len_after=i32([32, 16]), first=i32([15, 0]), count=i32([2, 1]), max_rows=4)
    cache.layout(b)
    assert cache.status() == B.ODB_ERR_STATE
    assert b.row_slot.cpu().tolist() == [15, -1, 16, -1]
    cache.close()


# ---- norm, rotation, store --------------------------------------------------------------------------------------------

STORE = [  # rows, heads, kv heads, head dim, page, rot, interleaved, norm, scaling, factor, farthest position
    (1, 1, 1, 64, 16, 64, False, True, "none", 1.0, 10),
    (1, 32, 8, 128, 64, 128, False, True, "none", 1.0, 131072),
    (7, 6, 2, 128, 16, 64, True, True, "yarn", 8.0, 60000),
    (33, 5, 5, 64, 32, 24, True, False, "linear", 4.0, 9000),
    (130, 8, 1, 128, 128, 96, False, True, "ntk", 4.0, 1 << 20),
    (65, 3, 3, 64, 1024, 0, False, True, "none", 1.0, 100),
    (40, 71, 1, 64, 16, 8, False, False, "none", 1.0, 2 ** 31 - 1),
    (257, 16, 4, 128, 64, 128, True, False, "yarn", 32.0, 200000),
    (1118, 4, 4, 64, 64, 64, False, True, "none", 1.0, 2048),
]


@requires_gpu
@pytest.mark.parametrize("case", STORE)
@pytest.mark.parametrize("packed", [True, False])
def test_norm_rope_store(case, packed):
    rows, H, KV, D, page, rot, inter, norm, scaling, factor, far = case
    P = paged()
    rng = np.random.default_rng(rows + H + rot)
    n_pages = O.pages_of(rows, page) + 2
    layer, layers = 1, 2
    qkv, qkv_f = bf16(rng, rows, (H + 2 * KV) * D, scale=2.0)
    kv0, _ = bf16(rng, layers, 2, n_pages, KV, page, D)
    cache = P.PagedCache(layers, H, KV, D, page, n_pages, kv=kv0.cuda())
    pos = rng.integers(0, far, rows).astype(np.int32)
    slot = rng.permutation(n_pages * page)[:rows].astype(np.int32)
    if rows > 5:
        slot[3] = -1                                          # K and V of this row are not stored
        pos[rows - 1], slot[rows - 1] = -1, -1                # a row behind the last
        slot[4] = n_pages * page                              # no slot
    qg, kg = (rng.standard_normal(D).astype(np.float32) * 0.2 + 1 for _ in range(2))
    b = P.Batch(cache, row_pos=dev(pos), row_slot=dev(slot))
    rope = P.Rope(rot, interleaved=inter, scaling=scaling, factor=factor, original_len=4096)
    x = qkv.cuda()
    a, c = H * D, (H + KV) * D
    parts = (x[:, :a], x[:, a:c], x[:, c:]) if packed else \
        (x[:, :a].reshape(rows, H, D).contiguous(), x[:, a:c].reshape(rows, KV, D).contiguous(), x[:, c:].contiguous())
    q_out = torch.full((rows, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cache.norm_rope_store(layer, b, *parts, rope, q_gain=dev(qg) if norm else None, k_gain=dev(kg) if norm else None, q_out=q_out)
    assert got is q_out and cache.status() == 0
    freq, mag = O.frequencies(rot, scaling=scaling, factor=factor, original_len=4096)
    xf = qkv_f.reshape(rows, H + 2 * KV, D)
    q_got = q_out.float().cpu().numpy()
    live = pos >= 0
    want_q = O.norm_rope(xf[:, :H], qg if norm else None, 1e-6, pos, freq, mag, inter)
    want_k = O.norm_rope(xf[:, H:H + KV], kg if norm else None, 1e-6, pos, freq, mag, inter)

    def tol(want, raw, gain):
        n = O.norm_rope(raw, gain, 1e-6, pos, np.zeros(0), 1.0, inter)     # the values that are turned
        half = rot // 2
        pair = np.abs(n).copy()
        i0, i1 = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if inter else (np.arange(half), np.arange(half, rot))
        pair[..., i0] = pair[..., i1] = np.abs(n[..., i0]) + np.abs(n[..., i1])
        return U * np.abs(want) + 2.0 ** -20 * mag * pair

    assert (np.abs(q_got - want_q) <= tol(want_q, xf[:, :H], qg if norm else None))[live].all()
    assert (q_got[~live] == 7.0).all()
    pool, before = cache.kv.float().cpu().numpy(), kv0.float().numpy()
    ok = (slot >= 0) & (slot < n_pages * page)
    t = tol(want_k, xf[:, H:H + KV], kg if norm else None)
    written = np.zeros((n_pages, page), bool)
    for r in np.flatnonzero(ok):
        p, o = slot[r] // page, slot[r] % page
        written[p, o] = True
        assert (np.abs(pool[layer, 0, p, :, o] - want_k[r]) <= t[r]).all(), r
        assert np.array_equal(pool[layer, 1, p, :, o], xf[r, H + KV:]), r
    assert np.array_equal(pool[0], before[0])                 # the other layer
    rest = ~written
    assert np.array_equal(pool[layer].transpose(1, 3, 0, 2, 4)[rest], before[layer].transpose(1, 3, 0, 2, 4)[rest])
    cache.close()


@requires_gpu
def test_norm_rope_store_in_place_and_without_anything_to_do():
    P = paged()
    rng = np.random.default_rng(5)
    cache = P.PagedCache(1, 4, 2, 64, 16, 4, kv=torch.zeros(1, 2, 4, 2, 16, 64, dtype=torch.bfloat16, device="cuda"))
    q, _ = bf16(rng, 20, 4, 64)
    kv, _ = bf16(rng, 20, 2, 64)
    pos = np.arange(20, dtype=np.int32) * 50
    b = P.Batch(cache, row_pos=dev(pos), row_slot=dev(np.arange(20, dtype=np.int32)))
    rope = P.Rope(64)
    out = cache.norm_rope_store(0, b, q.cuda(), kv.cuda(), kv.cuda(), rope)
    x = q.cuda()
    assert cache.norm_rope_store(0, b, x, kv.cuda(), kv.cuda(), rope, q_out=x) is x
    assert torch.equal(x, out)
    same = cache.norm_rope_store(0, b, q.cuda(), kv.cuda(), kv.cuda(), P.Rope(0))     # neither norm nor rotation: the values
    assert torch.equal(same.cpu(), q) and torch.equal(cache.kv[0, 0, 0].permute(1, 0, 2).cpu(), kv[:16])
    empty = P.Batch(cache, max_rows=0)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    nkv = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert cache.norm_rope_store(0, empty, none, nkv, nkv, rope).shape == (0, 4, 64)
    cache.close()


# The table's width is what the host knows of the keys, and with few of them every number of rows takes the kernel of few rows: the
# same requests in a wide table take the tensor cores'.
@pytest.fixture(params=["narrow", "wide"])
def columns(request):
    return {"narrow": 1, "wide": 5000}[request.param]


# ---- attention --------------------------------------------------------------------------------------------------------

def _setup(rng, lens, counts, firsts, H, KV, D, page, layers=1, layer=0, poison=True, scale=1.0, spare=2, columns=1):
    """A pool of shuffled pages; everything that is no key of a request is NaN, and so are pages nobody holds."""
    P = paged()
    held = [O.pages_of(n, page) for n in lens]
    n_pages = sum(held) + spare
    pool = torch.full((layers, 2, n_pages, KV, page, D), float("nan") if poison else 0.0, dtype=torch.bfloat16)
    order = rng.permutation(n_pages)
    width = max(held + [1]) + columns
    table = np.full((len(lens), width), 10 ** 6, np.int32)
    keys, values = [], []
    at = 0
    for s, n in enumerate(lens):
        mine = order[at:at + held[s]]
        at += held[s]
        table[s, :held[s]] = mine
        k, kf = bf16(rng, n, KV, D, scale=scale)
        v, vf = bf16(rng, n, KV, D)
        for j in range(n):
            pool[layer, 0, mine[j // page], :, j % page] = k[j]
            pool[layer, 1, mine[j // page], :, j % page] = v[j]
        keys.append(kf)
        values.append(vf)
    rows = sum(counts)
    q, qf = bf16(rng, rows, H, D, scale=scale)
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    cache = P.PagedCache(layers, H, KV, D, page, n_pages, kv=pool.cuda())
    i32 = lambda v: dev(np.asarray(v, np.int32))
    batch = P.Batch(cache, table=dev(table), len_after=i32(lens), first=i32(firsts), row_start=dev(start), max_rows=rows,
                    max_new=max(counts))
    return cache, batch, q.cuda(), qf, keys, values, start


def _check(out, lse, qf, keys, values, start, firsts, D, scale=None, **mask):
    out, lse = out.float().cpu().numpy(), None if lse is None else lse.cpu().numpy()
    for s in range(len(keys)):
        rows = slice(start[s], start[s + 1])
        pos = firsts[s] + np.arange(start[s + 1] - start[s])
        want, wl, mag, size = O.attention(qf[rows], keys[s], values[s], pos, scale, **mask)
        d = (D * 2.0 ** -24 * size)[..., None]
        tol = U * np.abs(want) + (U + 2.2 * d + 2.0 ** -20) * mag * 1.01
        assert (np.abs(out[rows] - want) <= tol).all(), (s, np.abs(out[rows] - want).max(), (np.abs(out[rows] - want) / np.maximum(tol, 1e-30)).max())
        if lse is not None:
            gone = np.isinf(wl)
            assert np.array_equal(np.isinf(lse[rows]), gone) and (lse[rows][gone] == -np.inf).all()
            err = np.abs(lse[rows] - wl)[~gone]
            assert (err <= (d[..., 0] + 2.0 ** -21 * (1 + np.abs(wl)))[~gone]).all(), (s, err.max())


def _check_scaled(out, lse, qf, keys, values, start, firsts, D, scale, **mask):
    """As _check where the scores' own error d is not small: the weights are off by up to e^(2 d) - 1 each, the output at most by
    the largest value; log-sum-exp in relative terms of the scores it comes from."""
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    for s in range(len(keys)):
        rows = slice(start[s], start[s + 1])
        pos = firsts[s] + np.arange(start[s + 1] - start[s])
        want, wl, mag, size = O.attention(qf[rows], keys[s], values[s], pos, scale, **mask)
        d = D * 2.0 ** -24 * size + 2.0 ** -23 * size              # the sum of products, and its own rounding after the scale
        grow = np.minimum(np.expm1(np.minimum(2 * d, 50.0)), 1e6)[..., None]
        top = max(np.abs(v).max() for v in values)
        tol = U * np.abs(want) + np.minimum((U + grow + 2.0 ** -20) * mag * 1.01, 2.02 * top)
        assert (np.abs(out[rows] - want) <= tol).all(), (s, np.abs(out[rows] - want).max())
        assert (np.abs(lse[rows] - wl) <= d + 2.0 ** -21 * (1 + np.abs(wl))).all(), (s, np.abs(lse[rows] - wl).max())


ATT = [  # lens, rows (0: all), H, KV, D, page, mask
    ([1], 1, 1, 1, 64, 16, {}),
    ([577], 1, 32, 8, 128, 16, {}),
    ([5, 64, 65, 1, 200], 1, 8, 2, 128, 64, dict(right=0)),
    ([63, 128, 129, 1000], 1, 16, 16, 64, 32, dict(right=0)),
    ([3000], 1, 6, 2, 128, 128, {}),
    ([2500, 17], 1, 71, 1, 64, 16, dict(right=0)),
    ([300, 40, 77], 1, 8, 2, 64, 16, dict(left=31, right=0, sinks=4)),
    ([900, 64], 1, 4, 4, 128, 64, dict(left=0, right=0)),
    ([900], 1, 8, 2, 128, 32, dict(left=127, right=0, sinks=100)),
    ([500, 33, 90], 7, 8, 4, 128, 16, dict(right=0)),
    ([500, 33, 90], 4, 8, 2, 64, 64, dict(left=10, right=0, sinks=3)),
    ([200, 130], 16, 6, 2, 128, 16, dict(left=20, right=5)),
    ([257, 96, 64], 32, 8, 2, 128, 64, {}),
    ([400, 33], 33, 4, 1, 64, 128, dict(right=0)),
    ([150, 70, 1], 0, 4, 4, 128, 64, {}),
    ([130, 65, 64], 0, 6, 2, 64, 16, dict(right=0)),
    ([300], 0, 8, 2, 128, 256, dict(left=50, right=0, sinks=2)),
    ([210], 0, 3, 1, 128, 16, dict(left=40, right=40)),
    ([1000, 33, 200], 32, 8, 2, 128, 32, {}),                      # 128 packed rows
    ([700, 100], 25, 10, 2, 64, 16, dict(right=0)),                # 125 packed rows, groups of five
    ([900, 64, 129], 20, 8, 2, 64, 128, dict(left=100, right=3, sinks=70)),
    ([520], 0, 10, 2, 128, 64, dict(right=0)),
    ([2000], 40, 4, 1, 64, 64, dict(left=300, right=0, sinks=130)),
    ([300, 290], 0, 1, 1, 64, 32, dict(right=0)),
    ([40], 0, 71, 1, 64, 16, dict(right=0)),
    ([30], 0, 130, 1, 64, 16, dict(right=0)),                      # more heads in a group than a Q tile has rows
]


@requires_gpu
@pytest.mark.parametrize("case", ATT)
def test_attention(case, columns):
    lens, new, H, KV, D, page, mask = case
    rng = np.random.default_rng(len(lens) * 31 + H + D + page)
    counts = [min(n, new) if new else n for n in lens]
    firsts = [n - c for n, c in zip(lens, counts)]
    if not mask and new > 1:
        firsts = [max(0, f // 2) for f in firsts]                 # a block in the middle
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, H, KV, D, page, columns=columns)
    lse = torch.empty(sum(counts), H, device="cuda")
    out = cache.attention(0, b, q, lse=lse, **mask)
    assert cache.status() == 0
    _check(out, lse, qf, keys, values, start, firsts, D, **mask)
    again = cache.attention(0, b, q, **mask)                      # without lse; the same bits
    assert torch.equal(again, out)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,G", [(1, 4), (30, 4), (60, 4)])
def test_attention_of_many_requests_of_a_tile_or_two(new, G, D, columns):
    """More items than CTAs, each of one to three key tiles: shares of many items, and items cut in two."""
    rng = np.random.default_rng(new + D)
    seqs = 230
    lens = [int(n) for n in rng.integers(1, 150, seqs)]
    counts = [min(n, new) for n in lens]
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 2 * G, 2, D, 16, columns=columns)
    lse = torch.empty(sum(counts), 2 * G, device="cuda")
    out = cache.attention(0, b, q, right=0, lse=lse)
    assert cache.status() == 0
    got, gl = out.float().cpu().numpy(), lse.cpu().numpy()
    for s in range(0, seqs, 1 if new == 1 else 9):                 # the oracle takes its time
        rows = slice(start[s], start[s + 1])
        _check(torch.from_numpy(got[rows]), torch.from_numpy(gl[rows]), qf[rows], keys[s:s + 1], values[s:s + 1],
               np.array([0, counts[s]]), firsts[s:s + 1], D, right=0)
    assert np.isfinite(got).all() and torch.equal(cache.attention(0, b, q, right=0), out)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("max_new", [1, 8, 16, 20, 64, 5000])
def test_the_hint_decides_no_result(max_new, columns):
    rng = np.random.default_rng(9)
    lens, counts = [90, 300, 20], [1, 37, 5]
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 8, 2, 128, 32, columns=columns)
    b._c.max_new = max_new
    lse = torch.empty(sum(counts), 8, device="cuda")
    out = cache.attention(0, b, q, right=0, lse=lse)
    assert cache.status() == 0
    _check(out, lse, qf, keys, values, start, firsts, 128, right=0)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new", [1, 3, 20, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_rows_that_see_nothing_and_requests_without_rows_or_keys(new, D, columns):
    rng = np.random.default_rng(new + D)
    lens, counts = [0, 70, 0, 12, 33], [new, 0, 0, new, new]
    firsts = [0, 3, 0, 40, 60]                                     # 40 - left > 12: the window lies behind the keys
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 4, 2, D, 16, columns=columns)
    for mask in (dict(), dict(right=0), dict(left=5, right=0), dict(left=5, right=0, sinks=3), dict(left=0, sinks=1)):
        lse = torch.full((sum(counts), 4), 3.0, device="cuda")
        out = torch.full((sum(counts), 4, D), 3.0, dtype=torch.bfloat16, device="cuda")
        cache.attention(0, b, q, lse=lse, out=out, **mask)
        assert cache.status() == 0
        _check(out, lse, qf, keys, values, start, firsts, D, **mask)
    assert bool((out[:new] == 0).all())
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new,G", [(1, 4), (5, 2), (20, 1), (9, 4), (16, 4), (20, 4), (70, 1), (70, 2), (100, 3)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_infinities_and_nan_reach_only_the_rows_that_see_them(new, G, D, columns):
    rng = np.random.default_rng(new + D)
    n = 150
    first = n - new
    cache, b, q, qf, keys, values, start = _setup(rng, [n], [new], [first], 2 * G, 2, D, 16, columns=columns)
    table = b.table.cpu().numpy()[0]
    mask = dict(left=60, right=0, sinks=2)
    clean = cache.attention(0, b, q, **mask).float().cpu().numpy()
    bad = {3: float("nan"), 60: float("inf"), n - 70: float("nan"), n - new: float("inf"), n - 1: float("nan")}
    for j, x in bad.items():
        cache.kv[0, 1, table[j // 16], 1, j % 16, 5] = x           # V of the second K/V head, one dim
    got = cache.attention(0, b, q, **mask).float().cpu().numpy()
    assert cache.status() == 0
    assert np.array_equal(got[:, :G], clean[:, :G])                # the first K/V head's group
    for r in range(new):
        ok = O.visible(n, first + r, **mask)
        seen = [x for j, x in bad.items() if ok[j]]
        col = got[r, G:, 5]
        if not seen:
            assert np.isfinite(got[r]).all() and np.array_equal(got[r], clean[r]), r
        else:
            want_nan = any(np.isnan(x) for x in seen)
            assert (np.isnan(col) if want_nan else np.isposinf(col)).all(), (r, seen, col)
            other = np.delete(got[r, G:], 5, axis=1)
            assert np.array_equal(other, np.delete(clean[r, G:], 5, axis=1)), r
    # a NaN in K outside every window changes nothing either
    for j, x in bad.items():
        cache.kv[0, 1, table[j // 16], 1, j % 16, 5] = 0.0
    base = cache.attention(0, b, q, **mask)
    j = first - 61 - 1
    if j > 2:
        cache.kv[0, 0, table[j // 16], 1, j % 16, 7] = float("nan")
        assert torch.equal(cache.attention(0, b, q, **mask), base)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [3, 45, 90])
def test_attention_of_large_scores_and_another_scale(new, D, columns):
    rng = np.random.default_rng(21)
    lens, counts = [333, 94], [new, new]
    firsts = [n - c for n, c in zip(lens, counts)]
    for scale in (0.0, 0.25, 1e-4, -0.05, 3e4):
        for size in (1.0, 30.0):
            cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 4, 2, D, 16, scale=size, columns=columns)
            lse = torch.empty(2 * new, 4, device="cuda")
            out = cache.attention(0, b, q, lse=lse, scale=scale, right=0)
            _check_scaled(out, lse, qf, keys, values, start, firsts, D, scale or None, right=0)
            cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,new,G", [([1500], 1500, 4), ([700, 90], 90, 1), ([2600], 30, 4), ([3000], 1, 4)])
def test_attention_of_scores_far_below_zero_in_parts(lens, new, G, D, columns):
    """Rows whose scores all lie hundreds below zero, some of whose item's parts hold no key that they see."""
    rng = np.random.default_rng(22)
    counts = [new] * len(lens)
    firsts = [n - new for n in lens]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 2 * G, 2, D, 16, columns=columns)
    cache.kv[:, 0].abs_()
    for mask in (dict(right=0), dict(left=70, right=0)):
        lse = torch.empty(len(qf), 2 * G, device="cuda")
        out = cache.attention(0, b, q.abs(), lse=lse, scale=-8.0, **mask)
        _check_scaled(out, lse, np.abs(qf), [np.abs(k) for k in keys], values, start, firsts, D, -8.0, **mask)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4])
def test_attention_of_prompts_blocks_and_single_tokens_in_one_forward(G, D, columns):
    """Requests of one, a few and many row tiles by turns, so that shares begin and end in each kind."""
    rng = np.random.default_rng(23)
    lens = [700, 577, 90, 1, 2000, 64, 300, 1500, 129, 520]
    counts = [300, 1, 1, 1, 33, 64, 300, 1, 129, 2]
    firsts = [n - c for n, c in zip(lens, counts)]
    for mask in (dict(right=0), dict(left=200, right=0, sinks=5), dict()):
        cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 2 * G, 2, D, 32, columns=columns)
        lse = torch.empty(len(qf), 2 * G, device="cuda")
        out = cache.attention(0, b, q, lse=lse, **mask)
        _check(out, lse, qf, keys, values, start, firsts, D, **mask)
        again = cache.attention(0, b, q, **mask)
        assert torch.equal(out, again)
        cache.close()


@requires_gpu
def test_attention_reads_strided_rows_and_other_layers_and_leaves_rows_behind_the_last():
    rng = np.random.default_rng(4)
    lens, counts, firsts = [50, 90], [2, 5], [48, 85]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 8, 4, 64, 16, layers=3, layer=2)
    wide = torch.full((7, 8 * 64 + 72), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 512] = q.view(7, 512)
    res = torch.full((9, 8 * 64 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    out = cache.attention(2, b, wide[:, 8:520], right=0, out=res[:7, :512])
    _check(out.view(7, 8, 64) if out.is_contiguous() else out.reshape(7, 8, 64), None, qf, keys, values, start, firsts, 64, right=0)
    assert bool((res[7:] == 3.0).all()) and bool((res[:, 512:] == 3.0).all())
    # fewer rows than the maps have
    P = paged()
    big = torch.full((12, 8, 64), 1.0, dtype=torch.bfloat16, device="cuda")
    big[:7] = q
    b2 = P.Batch(cache, table=b.table, len_after=b.len_after, first=b.first, row_start=b.row_start, max_rows=12, max_new=5)
    o2 = torch.full((12, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    cache.attention(2, b2, big, right=0, out=o2)
    assert torch.equal(o2[:7].reshape(7, 512), res[:7, :512]) and bool((o2[7:] == 3.0).all())
    cache.close()


@requires_gpu
def test_a_table_of_nonsense_stays_inside_the_pool():
    """Page ids that are none read as zeros, lengths beyond the table are cut: defined results, nothing out of bounds."""
    rng = np.random.default_rng(8)
    cache, b, q, qf, keys, values, start = _setup(rng, [40, 40], [1, 1], [39, 39], 2, 1, 64, 16)
    b.table.fill_(-5)
    b.table[1] = 2 ** 31 - 1
    out = cache.attention(0, b, q)
    assert bool((out == 0).all())
    b.len_after.fill_(2 ** 31 - 1)
    b.first.fill_(-2 ** 31)
    assert bool((cache.attention(0, b, q, right=0) == 0).all())
    b.row_start.copy_(torch.tensor([0, 1, 2 ** 31 - 1], dtype=torch.int32))
    cache.attention(0, b, q)
    b.row_start.copy_(torch.tensor([-9, -3, -1], dtype=torch.int32))
    cache.attention(0, b, q)
    torch.cuda.synchronize()
    cache.close()


@requires_gpu
def test_streams_and_graphs():
    rng = np.random.default_rng(12)
    lens, counts, firsts = [700, 90], [4, 4], [696, 86]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 8, 2, 128, 64)
    want = cache.attention(0, b, q, right=0)
    side = torch.cuda.Stream()
    outs = []
    for i in range(6):                                              # by turns on two streams: the workspace is shared
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            outs.append(cache.attention(0, b, q, right=0))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    out = torch.zeros_like(want)
    with torch.cuda.stream(side):
        cache.attention(0, b, q, right=0, out=out)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            cache.attention(0, b, q, right=0, out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    cache.close()


# ---- refusals ---------------------------------------------------------------------------------------------------------

@requires_gpu
def test_calls_that_are_refused():
    P = paged()
    from paper_2511_21759_b200 import binding as B
    for bad in (dict(head_dim=96), dict(n_heads=6, n_kv_heads=4), dict(page_size=24), dict(page_size=8), dict(n_pages=0), dict(n_layers=0),
                dict(n_pages=1 << 28)):
        cfg = dict(n_layers=1, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=4) | bad
        with pytest.raises(B.OdbError) as e:
            P.PagedCache(**cfg)
        assert e.value.status == B.ODB_ERR_SHAPE
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 2, 64, 16, 4, kv=torch.zeros(1, 2, 4, 2, 16, 64, device="cuda"))
    cache = P.PagedCache(1, 4, 2, 64, 16, 4)
    i32 = lambda v: dev(np.asarray(v, np.int32))
    b = P.Batch(cache, table=i32([[0]]), len_after=i32([10]), first=i32([9]), row_start=i32([0, 1]), row_pos=i32([9]), row_slot=i32([9]))
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    for wrong in (q.float(), q.cpu(), q[:, :2], torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"),
                  torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            cache.attention(0, b, wrong)
    for kw in (dict(left=-2), dict(right=-3), dict(sinks=-1), dict(scale=float("nan"))):
        with pytest.raises(B.OdbError) as e:
            cache.attention(0, b, q, **kw)
        assert e.value.status == B.ODB_ERR_ARG
    for layer in (-1, 1):
        with pytest.raises(B.OdbError) as e:
            cache.attention(layer, b, q)
        assert e.value.status == B.ODB_ERR_ARG
    with pytest.raises(B.OdbError):                                  # an address off its boundary
        flat = torch.zeros(4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
        cache.attention(0, b, flat[1:257].view(1, 4, 64))
    with pytest.raises(B.OdbError):                                  # no lengths
        cache.layout(P.Batch(cache, table=i32([[0]]), row_start=i32([0, 0])))
    with pytest.raises(ValueError):
        P.Batch(cache, table=i32([[0]]), len_after=i32([1, 2]))
    with pytest.raises(ValueError):
        P.Batch(cache, table=torch.zeros(1, 1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        P.Rope(64, scaling="other")
    for bad in (dict(rot_dim=12), dict(rot_dim=136), dict(rot_dim=-8)):
        with pytest.raises(B.OdbError):
            P.Rope(**bad)
    for bad in (dict(theta=0.5), dict(scaling="yarn", factor=0.5), dict(scaling="linear", factor=float("inf"))):
        with pytest.raises(B.OdbError):
            P.Rope(64, **bad)
    with pytest.raises(B.OdbError):                                  # more values turned than a head has
        cache.norm_rope_store(0, b, q, kv, kv, P.Rope(128))
    with pytest.raises(ValueError):
        cache.norm_rope_store(0, b, q, kv, kv, P.Rope(64), q_gain=torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(B.OdbError):
        cache.norm_rope_store(0, b, q, kv, kv, P.Rope(64), eps=-1.0)
    assert cache.status() == 0
    cache.close()
