"""The paged cache in 8 bits against the 64-bit oracle: what is written and under which scales, rows read back, attention over the codes.

Bounds, derived before the first run.
  store: V comes in as bf16 and meets no arithmetic but its rounding: codes and scales are the oracle's.  K is rounded once: half a step of
  e4m3, 2^-4 of its value or 2^-10 of the scale, in front of it the fp32 roundings of norm and rotation, below 2^-20 of the pair's terms;
  its exponent is the oracle's unless the largest value lies within those 2^-20 of a border.  What is kept is rounded from the codes before:
  the oracle's, under the exponent that the block got.
  load: exact.
  attention, over the values that the codes stand for: the output's rounding to bf16, 2^-8 of its value (half a step is 2^-9; the double is
  kept for the sums in front of it); a weight's rounding, 2^-8 (bf16, over a copy) or 2^-11 (f16) of itself, and in f16 no less
  than 2^-24 of the row's largest product of weight and scale (half a step of 2^-24 where that is rounded up to a power of two): at most
  the weight itself; a score's fp32 sum of head_dim exact products, head_dim 2^-24 sum|q k|
  scale, and Q in f16 under a power of two, 2^-25 of its largest value per dim: together d, which moves numerator and denominator by a
  factor e^d each; log-sum-exp by d and a rounding of fp32."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O
from test_gpu_paged import ATT, bf16, dev, paged

U = 2.0 ** -8
VALUES = O.e4m3_values()
E4M3 = torch.float8_e4m3fn


def i32(v):
    return dev(np.asarray(v, np.int32))


def codes_of(t):
    """The codes of a float8 tensor as numpy."""
    return t.view(torch.uint8).cpu().numpy()


def pool_values(cache):
    """[layers][2][pages][kv][page][hd] in 64 bits."""
    return VALUES[codes_of(cache.kv)] * np.repeat(cache.scales.cpu().numpy().astype(np.float64), O.BLOCK, -1)[..., None]


def random_pool(rng, layers, n_pages, KV, page, D, low=-3, high=4, poison=False):
    """Codes and scales on the CPU; poison: NaN everywhere."""
    shape = (layers, 2, n_pages, KV, page, D)
    if poison:
        return torch.full(shape, 0x7f, dtype=torch.uint8), torch.full(shape[:4] + (page // O.BLOCK,), float("nan"))
    c = rng.integers(0, 256, shape).astype(np.uint8)
    c[(c & 127) == 127] = 3
    s = 2.0 ** rng.integers(low, high, shape[:4] + (page // O.BLOCK,))
    return torch.from_numpy(c), torch.from_numpy(s.astype(np.float32))


def make(layers, H, KV, D, page, n_pages, pool, room=True):
    return paged().PagedCache(layers, H, KV, D, page, n_pages, kv=pool[0].cuda().view(E4M3), scales=pool[1].cuda(), room=room)


# ---- store ------------------------------------------------------------------------------------------------------------

STORE = [  # requests (first, rows, length), H, KV, D, page, rot, interleaved, norm, scaling, factor
    ([(0, 1, 1)], 1, 1, 64, 16, 64, False, True, "none", 1.0),
    ([(130, 1, 131)], 32, 8, 128, 64, 128, False, True, "none", 1.0),
    ([(0, 40, 40)], 4, 2, 128, 64, 128, False, True, "none", 1.0),
    ([(7, 20, 60), (0, 5, 5), (33, 1, 34), (64, 16, 80)], 6, 2, 128, 16, 64, True, True, "yarn", 8.0),
    ([(3, 1, 4), (15, 1, 16), (16, 1, 17), (31, 2, 40), (40, 1, 41)], 5, 5, 64, 32, 24, True, False, "linear", 4.0),
    ([(5, 100, 130), (16, 32, 48)], 8, 1, 128, 128, 96, False, True, "ntk", 4.0),
    ([(200, 65, 300)], 3, 3, 64, 1024, 0, False, True, "none", 1.0),
    ([(0, 33, 33), (90, 3, 95), (10, 1, 11)], 71, 1, 64, 16, 8, False, False, "none", 1.0),
    ([(100000, 47, 100100), (0, 16, 16)], 16, 4, 128, 64, 128, True, False, "yarn", 32.0),
    ([(0, 700, 700), (300, 418, 718)], 4, 4, 64, 64, 64, False, True, "none", 1.0),
    ([(i * 3, 1, i * 3 + 1) for i in range(70)], 4, 2, 64, 16, 64, False, True, "none", 1.0),
    # enough work for units of 4, of 8 and of 2 heads, the last of fewer; rows of two and more blocks in a window
    ([(i * 3, 1, i * 3 + 1) for i in range(90)], 26, 26, 64, 32, 64, False, True, "none", 1.0),
    ([(5, 1000, 1005)], 70, 70, 64, 64, 64, True, True, "none", 1.0),
    ([(i * 7 + 3, 9, i * 7 + 12) for i in range(60)], 31, 31, 128, 16, 128, False, False, "none", 1.0),
]


def _norm_slack(raw, gain, pos, rot, mag, inter):
    """2^-20 of |a| + |b| of every pair after the norm."""
    n = np.abs(O.norm_rope(raw, gain, 1e-6, pos, np.zeros(0), 1.0, inter))
    half = rot // 2
    pair = n.copy()
    a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if inter else (np.arange(half), np.arange(half, rot))
    pair[..., a] = pair[..., b] = n[..., a] + n[..., b]
    return 2.0 ** -20 * mag * pair


def _check_store(case, seed, layers=2, layer=1, size=1.0):
    req, H, KV, D, page, rot, inter, norm, scaling, factor = case
    P = paged()
    rng = np.random.default_rng(seed)
    held = [O.pages_of(n, page) for _, _, n in req]
    n_pages = sum(held) + 2
    order = rng.permutation(n_pages)
    pool = random_pool(rng, layers, n_pages, KV, page, D)
    cache = make(layers, H, KV, D, page, n_pages, pool)
    before = pool_values(cache)
    before_exp = np.log2(pool[1].numpy().astype(np.float64)).round().astype(int)
    seq, pos, slot, tables, at = [], [], [], [], 0
    for s, (first, n, length) in enumerate(req):
        tables.append(order[at:at + held[s]])
        at += held[s]
        for p in range(first, first + n):
            seq.append(s), pos.append(p), slot.append(tables[s][p // page] * page + p % page)
    seq, pos, slot = (np.asarray(v, np.int32) for v in (seq, pos, slot))
    rows = len(seq) + 3                                        # rows behind the last
    pad = lambda v: np.concatenate([v, np.full(3, -1, np.int32)])
    qkv, qkv_f = bf16(rng, rows, (H + 2 * KV) * D, scale=2.0)
    grow = (2.0 ** rng.integers(-6, 7, (rows, 1))).astype(np.float32) * np.float32(size)
    qkv_f = qkv_f * grow
    qkv = torch.from_numpy(qkv_f).to(torch.bfloat16)
    assert np.array_equal(qkv.float().numpy(), qkv_f)
    qg, kg = (rng.standard_normal(D).astype(np.float32) * 0.2 + 1 for _ in range(2))
    b = P.Batch(cache, len_after=i32([r[2] for r in req]), row_seq=dev(pad(seq)), row_pos=dev(pad(pos)), row_slot=dev(pad(slot)))
    rope = P.Rope(rot, interleaved=inter, scaling=scaling, factor=factor, original_len=4096)
    x = qkv.cuda()
    a, c = H * D, (H + KV) * D
    q_out = torch.full((rows, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    cache.norm_rope_store(layer, b, x[:, :a], x[:, a:c], x[:, c:], rope, q_gain=dev(qg) if norm else None, k_gain=dev(kg) if norm else None, q_out=q_out)
    assert cache.status() == 0
    freq, mag = O.frequencies(rot, scaling=scaling, factor=factor, original_len=4096)
    xf = qkv_f.reshape(rows, H + 2 * KV, D)[: rows - 3]
    args = lambda g: (g if norm else None, 1e-6, pos, freq, mag, inter)
    want_q, want_k, v = O.norm_rope(xf[:, :H], *args(qg)), O.norm_rope(xf[:, H:H + KV], *args(kg)), xf[:, H + KV:].astype(np.float64)
    slack_q, slack_k = (_norm_slack(t, g if norm else None, pos, rot, mag, inter) for t, g in ((xf[:, :H], qg), (xf[:, H:H + KV], kg)))
    got_q = q_out.float().cpu().numpy()
    assert (np.abs(got_q[: rows - 3] - want_q) <= U * np.abs(want_q) + slack_q).all() and (got_q[rows - 3:] == 7.0).all()
    after, scales = pool_values(cache), cache.scales.cpu().numpy().astype(np.float64)
    exps = np.log2(scales).round().astype(int)
    assert np.array_equal(2.0 ** exps, scales)
    want_pool, want_exps = before.copy(), before_exp.copy()
    codes_before, codes_after = pool[0].numpy(), codes_of(cache.kv)
    blocks = {}
    for r in range(len(seq)):
        blocks.setdefault((seq[r], pos[r] // O.BLOCK), []).append(r)
    for (s, blk), rr in blocks.items():
        at0 = slot[rr[0]] - pos[rr[0]] % O.BLOCK
        pg, o0 = at0 // page, at0 % page
        live = req[s][2] - blk * O.BLOCK
        offs = [int(pos[r]) % O.BLOCK for r in rr]
        kept = [o for o in range(min(live, O.BLOCK)) if o not in offs]
        for h in range(KV):
            place = (layer, slice(None), pg, h, slice(o0, o0 + O.BLOCK))
            b0 = before[place]
            e0 = before_exp[layer, :, pg, h, o0 // O.BLOCK]
            got, ge = after[place], exps[layer, :, pg, h, o0 // O.BLOCK]
            wv, we = O.quantise_block(b0[1], e0[1], v[rr, h], offs, live)
            assert ge[1] == we and np.array_equal(got[1][offs + kept], wv[offs + kept]), (s, blk, h)
            # K: the exponent by the largest value, give or take the roundings in front of it
            top, sl = np.abs(want_k[rr, h]).max(), slack_k[rr, h].max()
            lo, hi = O.exponent_for(max(top - sl, 0.0)), O.exponent_for(top + sl)
            if kept:
                lo, hi = max(lo, e0[0]), max(hi, e0[0])
            assert lo <= ge[0] <= hi, (s, blk, h)
            k = want_k[rr, h]
            tol = np.maximum(2.0 ** -4 * np.abs(k), 2.0 ** (ge[0] - 10)) + slack_k[rr, h] * 1.1
            assert (np.abs(got[0][offs] - k) <= tol).all(), (s, blk, h)
            assert np.array_equal(got[0][kept], O.e4m3_round(b0[0][kept] / 2.0 ** ge[0]) * 2.0 ** ge[0]), (s, blk, h)
            want_pool[place], want_exps[layer, :, pg, h, o0 // O.BLOCK] = got, ge
            for i in range(2):                                 # positions that are neither written nor kept: their codes stay
                rest = [o for o in range(O.BLOCK) if o not in offs + kept]
                old = codes_before[layer, i, pg, h, o0:o0 + O.BLOCK]
                now = codes_after[layer, i, pg, h, o0:o0 + O.BLOCK] if rest else old
                assert np.array_equal(now[rest], old[rest])
    assert np.array_equal(after, want_pool) and np.array_equal(exps, want_exps)     # nothing else has changed
    # the same call again finds its own scales and changes nothing
    cache.norm_rope_store(layer, b, x[:, :a], x[:, a:c], x[:, c:], rope, q_gain=dev(qg) if norm else None, k_gain=dev(kg) if norm else None, q_out=q_out)
    assert np.array_equal(pool_values(cache), after) and np.array_equal(cache.scales.cpu().numpy(), scales)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("case", STORE)
def test_store(case):
    _check_store(case, 11 + len(case[0]) + case[1])


@requires_gpu
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 60])
def test_store_of_small_and_large_values(size):
    _check_store(([(7, 20, 60), (0, 5, 5)], 4, 2, 128, 16, 64, False, False, "none", 1.0), 5, size=size)


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
def test_store_token_by_token_grows_the_scale_and_keeps_the_rows(D):
    """Sixteen calls of a row each, every one larger than those before: what is kept is rounded again each time; then all rows at once."""
    P = paged()
    rng = np.random.default_rng(D)
    cache = make(1, 2, 1, D, 16, 2, random_pool(rng, 1, 2, 1, 16, D, poison=True))
    rope = P.Rope(0)
    x = rng.standard_normal((16, D)).astype(np.float32) * (1.7 ** np.arange(16, dtype=np.float32))[:, None]
    xb = torch.from_numpy(x).to(torch.bfloat16)
    x = xb.double().numpy()
    want, e = np.zeros((16, D)), O.LOW_EXP
    for n in range(16):
        b = P.Batch(cache, len_after=i32([n + 1]), row_seq=i32([0]), row_pos=i32([n]), row_slot=i32([16 + n]))
        row = xb[n:n + 1].cuda()
        cache.norm_rope_store(0, b, row.repeat(1, 2), row, row, rope)
        want, e = O.quantise_block(want, e, x[n:n + 1], [n], n + 1)
        for i in range(2):
            assert cache.scales[0, i, 1, 0, 0].item() == 2.0 ** e
            assert np.array_equal(pool_values(cache)[0, i, 1, 0, :n + 1], want[:n + 1])
    first = O.quantise_block(np.zeros((16, D)), 0, x, list(range(16)), 16)[0]
    b = P.Batch(cache, len_after=i32([16]), row_seq=i32([0] * 16), row_pos=i32(range(16)), row_slot=i32(range(16)))
    cache.norm_rope_store(0, b, xb.cuda().repeat(1, 2), xb.cuda(), xb.cuda(), rope)
    assert np.array_equal(pool_values(cache)[0, 0, 0, 0], first)
    # a smaller block over it takes its scale down again: nothing is kept
    cache.norm_rope_store(0, b, xb.cuda().repeat(1, 2), xb.cuda() / 64, xb.cuda() / 64, rope)
    assert np.array_equal(pool_values(cache)[0, 1, 0, 0], first / 64)
    cache.close()


@requires_gpu
def test_store_of_values_that_are_not_finite():
    """They become NaN and take no part in the scale; a block of nothing else, or of zeros, has the smallest one."""
    P = paged()
    rng = np.random.default_rng(2)
    D = 64
    cache = make(1, 1, 1, D, 16, 4, random_pool(rng, 1, 4, 1, 16, D))
    x = torch.from_numpy(rng.standard_normal((48, D)).astype(np.float32)).to(torch.bfloat16)
    x[3, 5], x[4, 6], x[5, 7] = float("nan"), float("inf"), float("-inf")
    x[16:32] = 0.0
    x[32:48] = float("inf")
    b = P.Batch(cache, len_after=i32([48]), row_seq=i32([0] * 48), row_pos=i32(range(48)), row_slot=i32(range(48)))
    cache.norm_rope_store(0, b, x.cuda(), x.cuda(), x.cuda(), P.Rope(0))
    got = pool_values(cache)[0, :, :3, 0].reshape(2, 48, D)
    want = np.concatenate([O.quantise_block(np.zeros((16, D)), 0, x[i:i + 16].double().numpy(), list(range(16)), 16)[0] for i in (0, 16, 32)])
    for i in range(2):
        assert np.array_equal(got[i], want, equal_nan=True)
    assert np.isnan(want).sum() == 3 + 16 * D
    assert cache.scales[0, 0, :3, 0, 0].tolist() == [2.0 ** O.exponent_for(x[:16].double().abs()[torch.isfinite(x[:16])].max().item()), 2.0 ** -100, 2.0 ** -100]
    # the largest numbers of bf16, and the smallest
    x = torch.full((16, D), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16)
    x[1] = torch.finfo(torch.bfloat16).tiny
    b = P.Batch(cache, len_after=i32([16]), row_seq=i32([0] * 16), row_pos=i32(range(16)), row_slot=i32(range(16)))
    cache.norm_rope_store(0, b, x.cuda(), x.cuda(), x.cuda(), P.Rope(0))
    got = pool_values(cache)[0, 1, 0, 0]
    assert (got[0] == 448 * 2.0 ** 119).all() and (got[1] == 0).all() and cache.scales[0, 1, 0, 0, 0].item() == 2.0 ** 119
    k, v = cache.load(0, b)
    assert bool(torch.isfinite(k).all()) and (v[0, 0].double().cpu().numpy() == got[0]).all()
    cache.close()


@requires_gpu
def test_store_rounds_every_border_as_the_oracle():
    """All values of bf16 between two codes of an octave, ties among them, under a block whose largest value is 448."""
    P = paged()
    D = 128
    bits = np.arange(0x3b00, 0x43e1, dtype=np.uint32)             # from 2^-9 to 448
    n = -(-len(bits) // D) * D
    x = np.full(n, 448.0, np.float32)
    x[:len(bits)] = (bits << 16).view(np.float32)
    x = x.reshape(-1, D) * np.where(np.arange(n).reshape(-1, D) % 3 == 0, -1, 1).astype(np.float32)
    rows = len(x)
    x[:, 0] = 448.0
    length = -(-rows // 16) * 16
    cache = make(1, 1, 1, D, 16, length // 16, random_pool(np.random.default_rng(0), 1, length // 16, 1, 16, D))
    xb = torch.from_numpy(x).to(torch.bfloat16).cuda()
    b = P.Batch(cache, len_after=i32([rows]), row_seq=i32([0] * rows), row_pos=i32(range(rows)), row_slot=i32(range(rows)))
    cache.norm_rope_store(0, b, xb, xb, xb, P.Rope(0))
    got = pool_values(cache)[0, :, :, 0].reshape(2, -1, D)[:, :rows]
    assert np.array_equal(got[0], O.e4m3_round(x)) and np.array_equal(got[1], O.e4m3_round(x))
    cache.close()


@requires_gpu
def test_store_of_rows_without_a_place():
    """Rows without a position, a request or a slot, slots that are none or in another place than the position, and a row_seq or a length
    of nonsense: what has a place is stored, nothing else is written."""
    P = paged()
    rng = np.random.default_rng(4)
    D, KV = 64, 2
    pool = random_pool(rng, 1, 5, KV, 32, D)
    cache = make(1, 2, KV, D, 32, 5, pool)
    before = pool_values(cache)
    seq = [0, 0, 0, 0, -1, 7, 2 ** 31 - 1, 1, 1, 1, -2 ** 31]
    pos = [14, 15, 16, -1, 3, 3, 3, 5, 6, 2 ** 31 - 1, 4]
    slot = [14, -1, 16, 17, 100, 101, 102, 5 * 32 + 5, 40 + 3, 2 ** 31 - 1, 104]
    rows = len(seq)
    x = torch.from_numpy(rng.standard_normal((rows, 2 * D)).astype(np.float32)).to(torch.bfloat16).cuda()
    b = P.Batch(cache, len_after=i32([20, 2 ** 31 - 1, -5]), row_seq=i32(seq), row_pos=i32(pos), row_slot=i32(slot))
    q = cache.norm_rope_store(0, b, x, x, x, P.Rope(0), q_out=torch.full((rows, 2, D), 7.0, dtype=torch.bfloat16, device="cuda"))
    assert cache.status() == 0
    live = np.asarray(pos) >= 0
    assert torch.equal(q.view(rows, -1)[torch.from_numpy(live).cuda()], x[torch.from_numpy(live).cuda()]) and bool((q[3] == 7.0).all())
    after = pool_values(cache)
    xv = x.double().cpu().numpy().reshape(rows, KV, D)
    e0 = np.log2(pool[1].numpy().astype(np.float64)).astype(int)
    want = before.copy()
    for i in range(2):
        for h in range(KV):
            want[0, i, 0, h, :16], _ = O.quantise_block(before[0, i, 0, h, :16], e0[0, i, 0, h, 0], xv[0:1, h], [14], 20)
            w, _ = O.quantise_block(before[0, i, 0, h, 16:], e0[0, i, 0, h, 1], xv[2:3, h], [0], 4)
            want[0, i, 0, h, 16:20] = w[:4]
    # codes behind the length of a block whose scale has changed stand for something else now: nobody asked for them
    keep = np.ones((5, 32), bool)
    keep[0, 20:] = False
    assert np.array_equal(after.transpose(0, 1, 3, 5, 2, 4)[..., keep], want.transpose(0, 1, 3, 5, 2, 4)[..., keep])
    cache.close()


# ---- load -------------------------------------------------------------------------------------------------------------

@requires_gpu
@pytest.mark.parametrize("rows,KV,D,page", [(1, 1, 64, 16), (7, 3, 128, 32), (130, 8, 128, 64), (1000, 5, 64, 128), (3, 40, 128, 16)])
@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_load(rows, KV, D, page, kind):
    P = paged()
    rng = np.random.default_rng(rows)
    n_pages = O.pages_of(rows, page) + 2
    if kind == "e4m3":
        cache = make(2, KV, KV, D, page, n_pages, random_pool(rng, 2, n_pages, KV, page, D, low=-100, high=120))
        pool = pool_values(cache)
    else:
        kv, kvf = bf16(rng, 2, 2, n_pages, KV, page, D)
        cache = P.PagedCache(2, KV, KV, D, page, n_pages, kv=kv.cuda())
        pool = kvf.astype(np.float64)
    slot = rng.integers(0, n_pages * page, rows).astype(np.int32)      # the same row twice is no matter
    if rows > 5:
        slot[3], slot[5] = -1, n_pages * page
    ok = (slot >= 0) & (slot < n_pages * page)
    b = P.Batch(cache, row_slot=dev(slot))
    for layer in range(2):
        want = pool[layer][:, np.clip(slot, 0, n_pages * page - 1) // page, :, slot % page]
        both = torch.full((rows + 1, 2 * KV * D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
        k, v = cache.load(layer, b, k_out=both[:rows, : KV * D], v_out=both[:rows, KV * D: 2 * KV * D])
        got = both.double().cpu().numpy()
        w = want                                                      # [rows][2][kv][hd]: the two index arrays come first
        assert np.array_equal(got[:rows, : KV * D][ok], w[:, 0].reshape(rows, -1)[ok])
        assert np.array_equal(got[:rows, KV * D: 2 * KV * D][ok], w[:, 1].reshape(rows, -1)[ok])
        assert (got[:rows][~ok][:, : 2 * KV * D] == 3.0).all() and (got[rows] == 3.0).all() and (got[:, 2 * KV * D:] == 3.0).all()
        k2, v2 = cache.load(layer, b)
        good = torch.from_numpy(ok).cuda()
        assert torch.equal(k2.view(rows, -1)[good], k[good]) and torch.equal(v2.view(rows, -1)[good], v[good])
    assert cache.status() == 0
    empty = P.Batch(cache, max_rows=0)
    assert cache.load(0, empty)[0].shape == (0, KV, D)
    cache.close()


@requires_gpu
def test_load_of_every_code_under_every_scale():
    """All finite codes are exact in bf16 under all scales there are, and NaN stays one."""
    P = paged()
    exps = np.arange(O.LOW_EXP, O.HIGH_EXP + 1)
    n = len(exps)
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(4, 64), (4, 1))
    pool = torch.from_numpy(np.broadcast_to(codes, (1, 2, n, 1, 16, 64)).copy()), torch.from_numpy(np.broadcast_to((2.0 ** exps).astype(np.float32)[:, None, None], (1, 2, n, 1, 1)).copy())
    cache = make(1, 1, 1, 64, 16, n, pool)
    b = P.Batch(cache, row_slot=dev(np.arange(n * 16, dtype=np.int32)))
    k, v = cache.load(0, b)
    want = pool_values(cache)[0, 0].transpose(0, 2, 1, 3).reshape(n * 16, 64)
    assert np.array_equal(k[:, 0].double().cpu().numpy(), want, equal_nan=True) and np.array_equal(v[:, 0].double().cpu().numpy(), want, equal_nan=True)
    cache.close()


# ---- attention --------------------------------------------------------------------------------------------------------

# As for the pool of bf16, the table's width picks the kernel; in a wide one prompts are read from a copy in bf16 where there is room for it.
@pytest.fixture(params=["narrow", "wide", "wide without room"])
def columns(request):
    return {"narrow": 1, "wide": 5000, "wide without room": -5000}[request.param]


def setup(rng, lens, counts, firsts, H, KV, D, page, layers=1, layer=0, scale=1.0, spare=2, columns=1, spread=2, hidden=None):
    """A pool of shuffled pages; everything that is no key of a request is NaN, scales too.  hidden(s, block): the scale of a block that
    no row sees is NaN as well.  Returns cache, batch, q, its values, keys, values, scales of V by position, row starts."""
    P = paged()
    held = [O.pages_of(n, page) for n in lens]
    n_pages = sum(held) + spare
    codes, scales = random_pool(rng, layers, n_pages, KV, page, D, poison=True)
    codes, scales = codes.numpy(), scales.numpy()
    order = rng.permutation(n_pages)
    width = max(held + [1]) + abs(columns)
    table = np.full((len(lens), width), 10 ** 6, np.int32)
    keys, values, vscale = [], [], []
    at = 0
    for s, n in enumerate(lens):
        mine = order[at:at + held[s]]
        at += held[s]
        table[s, :held[s]] = mine
        both, sv = [], np.zeros((n, KV))
        for i in range(2):
            got = np.zeros((n, KV, D))
            for blk in range(O.pages_of(n, O.BLOCK)):
                j0, j1 = blk * O.BLOCK, min(n, (blk + 1) * O.BLOCK)
                x = rng.standard_normal((KV, j1 - j0, D)) * scale * 2.0 ** rng.uniform(-spread, spread, (KV, 1, 1))
                for h in range(KV):
                    e = O.exponent_for(np.abs(x[h]).max())
                    y = O.e4m3_round(x[h] / 2.0 ** e)
                    c = _codes(y)
                    pg, o = mine[j0 // page], j0 % page
                    codes[layer, i, pg, h, o:o + j1 - j0] = c
                    scales[layer, i, pg, h, o // O.BLOCK] = 2.0 ** e if not (hidden and hidden(s, blk)) else np.nan
                    got[j0:j1, h] = y * 2.0 ** e
                    if i:
                        sv[j0:j1, h] = 2.0 ** e
            both.append(got)
        keys.append(both[0]), values.append(both[1]), vscale.append(sv)
    rows = sum(counts)
    q, qf = bf16(rng, rows, H, D, scale=scale)
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    cache = make(layers, H, KV, D, page, n_pages, (torch.from_numpy(codes), torch.from_numpy(scales)), room=columns > 0)
    batch = P.Batch(cache, table=dev(table), len_after=i32(lens), first=i32(firsts), row_start=dev(start), max_rows=rows, max_new=max(counts))
    return cache, batch, q.cuda(), qf, keys, values, vscale, start


def _codes(y):
    """Codes of values that are values of codes."""
    c = np.searchsorted(VALUES[:127], np.abs(y)).astype(np.uint8)
    assert np.array_equal(VALUES[c], np.abs(y))
    return c | np.where(np.signbit(y), 128, 0).astype(np.uint8)


def check(out, lse, qf, keys, values, vscale, start, firsts, D, scale=None, scaled=False, **mask):
    out, lse = out.float().cpu().numpy(), None if lse is None else lse.cpu().numpy()
    sc = 1 / np.sqrt(D) if scale is None else scale
    for s in range(len(keys)):
        rows = slice(start[s], start[s + 1])
        n, H, KV = start[s + 1] - start[s], out.shape[1], keys[s].shape[1]
        pos = firsts[s] + np.arange(n)
        for r in range(n):
            ok = O.visible(len(keys[s]), int(pos[r]), **mask)
            if not ok.any():
                assert (out[rows][r] == 0).all() and (lse is None or (lse[rows][r] == -np.inf).all())
                continue
            for kv in range(KV):
                k, v, vs = keys[s][ok, kv], values[s][ok, kv], vscale[s][ok, kv]
                G = H // KV
                q = qf[rows][r, kv * G:(kv + 1) * G].astype(np.float64)
                x = q @ k.T * sc                                                    # [G][keys]
                m = x.max(1, keepdims=True)
                w = np.exp(x - m)
                total = w.sum(1, keepdims=True)
                w /= total
                want, mag = w @ v, w @ np.abs(v)
                size = (np.abs(q) @ np.abs(k).T).max(1) * abs(sc)
                d = D * 2.0 ** -24 * size + 2.0 ** -25 * np.abs(q).max(1) * np.abs(k).sum(1).max() * abs(sc)
                # f16: no less than 2^-24 of the row's largest product of weight and scale
                least = np.minimum(w * vs, 2.0 ** -24 * (w * vs).max(1, keepdims=True)) @ (np.abs(v) / vs[:, None])
                if scaled:
                    d = d + 2.0 ** -23 * size
                    grow = np.minimum(np.expm1(np.minimum(2 * d, 50.0)), 1e6)[:, None]
                    tol = U * np.abs(want) + least + np.minimum((U + grow + 2.0 ** -20) * mag * 1.01, 2.02 * np.abs(v).max())
                else:
                    tol = U * np.abs(want) + least + (U + 2.2 * d[:, None] + 2.0 ** -20) * mag * 1.01
                got = out[rows][r, kv * G:(kv + 1) * G]
                assert (np.abs(got - want) <= tol).all(), (s, r, kv, np.abs(got - want).max(), (np.abs(got - want) / np.maximum(tol, 1e-300)).max())
                if lse is not None:
                    wl = (m + np.log(total))[:, 0]
                    err = np.abs(lse[rows][r, kv * G:(kv + 1) * G] - wl)
                    assert (err <= d + 2.0 ** -21 * (1 + np.abs(wl))).all(), (s, r, err.max())


@requires_gpu
@pytest.mark.parametrize("case", ATT)
def test_attention(case, columns):
    lens, new, H, KV, D, page, mask = case
    rng = np.random.default_rng(len(lens) * 31 + H + D + page)
    counts = [min(n, new) if new else n for n in lens]
    firsts = [n - c for n, c in zip(lens, counts)]
    if not mask and new > 1:
        firsts = [max(0, f // 2) for f in firsts]                 # a block in the middle
    cache, b, q, *rest = setup(rng, lens, counts, firsts, H, KV, D, page, columns=columns)
    lse = torch.empty(sum(counts), H, device="cuda")
    out = cache.attention(0, b, q, lse=lse, **mask)
    assert cache.status() == 0
    check(out, lse, *rest, firsts, D, **mask)
    again = cache.attention(0, b, q, **mask)                      # without lse; the same bits
    assert torch.equal(again, out)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,G", [(1, 4), (30, 4)])
def test_attention_of_many_requests_of_a_tile_or_two(new, G, D, columns):
    """More items than CTAs, each of one to three key tiles: shares of many items, and items cut in two."""
    rng = np.random.default_rng(new + D)
    seqs = 230
    lens = [int(n) for n in rng.integers(1, 150, seqs)]
    counts = [min(n, new) for n in lens]
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, qf, keys, values, vscale, start = setup(rng, lens, counts, firsts, 2 * G, 2, D, 16, columns=columns)
    lse = torch.empty(sum(counts), 2 * G, device="cuda")
    out = cache.attention(0, b, q, right=0, lse=lse)
    assert cache.status() == 0
    for s in range(0, seqs, 1 if new == 1 else 9):                 # the oracle takes its time
        rows = slice(start[s], start[s + 1])
        check(out[rows], lse[rows], qf[rows], keys[s:s + 1], values[s:s + 1], vscale[s:s + 1], np.array([0, counts[s]]), firsts[s:s + 1], D, right=0)
    assert bool(torch.isfinite(out).all()) and torch.equal(cache.attention(0, b, q, right=0), out)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new", [1, 3, 10, 20, 40, 250])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_rows_that_see_nothing_and_requests_without_rows_or_keys(new, D, columns):
    rng = np.random.default_rng(new + D)
    lens, counts = [0, 70, 0, 12, 33], [new, 0, 0, new, new]
    firsts = [0, 3, 0, 40, 60]                                     # 40 - left > 12: the window lies behind the keys
    cache, b, q, *rest = setup(rng, lens, counts, firsts, 4, 2, D, 16, columns=columns)
    for mask in (dict(), dict(right=0), dict(left=5, right=0), dict(left=5, right=0, sinks=3), dict(left=0, sinks=1)):
        lse = torch.full((sum(counts), 4), 3.0, device="cuda")
        out = torch.full((sum(counts), 4, D), 3.0, dtype=torch.bfloat16, device="cuda")
        cache.attention(0, b, q, lse=lse, out=out, **mask)
        assert cache.status() == 0
        check(out, lse, *rest, firsts, D, **mask)
    assert bool((out[:new] == 0).all())
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new,G", [(1, 4), (5, 2), (5, 4), (20, 1), (9, 4), (20, 4), (70, 1), (100, 3), (130, 3)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_nan_codes_reach_only_the_rows_that_see_them(new, G, D, columns):
    rng = np.random.default_rng(new + D)
    n = 150
    first = n - new
    mask = dict(left=60, right=0, sinks=2)
    seen_by_some = lambda s, blk: not any(O.visible(n, p, **mask)[blk * 16:blk * 16 + 16].any() for p in range(first, n))
    cache, b, q, qf, keys, values, vscale, start = setup(rng, [n], [new], [first], 2 * G, 2, D, 16, columns=columns, hidden=seen_by_some)
    table = b.table.cpu().numpy()[0]
    clean = cache.attention(0, b, q, **mask)
    check(clean, None, qf, keys, values, vscale, start, [first], D, **mask)
    clean = clean.float().cpu().numpy()
    bad = [3, 60, n - 70, n - new, n - 1]
    raw = cache.kv.view(torch.uint8)
    for j in bad:
        raw[0, 1, table[j // 16], 1, j % 16, 5] = 0x7f if j % 2 else 0xff
    got = cache.attention(0, b, q, **mask).float().cpu().numpy()
    assert cache.status() == 0
    assert np.array_equal(got[:, :G], clean[:, :G])                # the first K/V head's group
    for r in range(new):
        ok = O.visible(n, first + r, **mask)
        if any(ok[j] for j in bad):
            assert np.isnan(got[r, G:, 5]).all(), r
            assert np.array_equal(np.delete(got[r, G:], 5, axis=1), np.delete(clean[r, G:], 5, axis=1)), r
        else:
            assert np.array_equal(got[r], clean[r]), r
    # a NaN in K reaches the rows that see it, all of their dims, and no other
    for j in bad:
        raw[0, 1, table[j // 16], 1, j % 16, 5] = 0
    base = cache.attention(0, b, q, **mask).float().cpu().numpy()
    for j in bad:
        raw[0, 0, table[j // 16], 1, j % 16, 7] = 0x7f
        got = cache.attention(0, b, q, **mask).float().cpu().numpy()
        for r in range(new):
            if O.visible(n, first + r, **mask)[j]:
                assert np.isnan(got[r, G:]).all() and np.array_equal(got[r, :G], base[r, :G])
            else:
                assert np.array_equal(got[r], base[r])
        raw[0, 0, table[j // 16], 1, j % 16, 7] = 0
        base = cache.attention(0, b, q, **mask).float().cpu().numpy()
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [3, 5, 45, 90, 240])
def test_attention_of_large_scores_and_another_scale(new, D, columns):
    rng = np.random.default_rng(21)
    lens, counts = [333, 94], [new, new]
    firsts = [n - c for n, c in zip(lens, counts)]
    for scale in (0.0, 0.25, 1e-4, -0.05, 3e4):
        for size in (1.0, 30.0):
            cache, b, q, *rest = setup(rng, lens, counts, firsts, 4, 2, D, 16, scale=size, columns=columns)
            lse = torch.empty(2 * new, 4, device="cuda")
            out = cache.attention(0, b, q, lse=lse, scale=scale, right=0)
            check(out, lse, *rest, firsts, D, scale or None, scaled=True, right=0)
            cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,new,G", [([1500], 300, 4), ([700, 90], 90, 1), ([2600], 30, 4), ([3000], 1, 4)])
@pytest.mark.parametrize("spread", [12, 40])
def test_attention_of_blocks_of_very_different_size(lens, new, G, D, spread, columns):
    """Blocks whose scales of K and V lie up to 2^24 and 2^80 apart: the weights of rows that see large values lightly."""
    rng = np.random.default_rng(22)
    counts = [new] * len(lens)
    firsts = [n - new for n in lens]
    cache, b, q, *rest = setup(rng, lens, counts, firsts, 2 * G, 2, D, 16, columns=columns, spread=spread)
    for scale in (0.0, 1e-6):
        lse = torch.empty(new * len(lens), 2 * G, device="cuda")
        out = cache.attention(0, b, q, lse=lse, right=0, scale=scale)
        assert cache.status() == 0
        check(out, lse, *rest, firsts, D, scale or None, scaled=True, right=0)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 4])
def test_attention_of_prompts_blocks_and_single_tokens_in_one_forward(G, D, columns):
    """Requests of one, a few and many row tiles by turns, so that shares begin and end in each kind."""
    rng = np.random.default_rng(23)
    lens = [700, 577, 90, 1, 2000, 64, 300, 1500, 129, 520]
    counts = [150, 1, 1, 1, 33, 64, 300, 1, 129, 2]
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, *rest = setup(rng, lens, counts, firsts, 2 * G, 2, D, 32, columns=columns)
    for mask in (dict(right=0), dict(left=200, right=0, sinks=5), dict()):
        lse = torch.empty(sum(counts), 2 * G, device="cuda")
        out = cache.attention(0, b, q, lse=lse, **mask)
        check(out, lse, *rest, firsts, D, **mask)
        assert torch.equal(out, cache.attention(0, b, q, **mask))
    cache.close()


@requires_gpu
def test_attention_of_queries_that_are_large_small_zero_or_not_finite():
    """A row's queries are its own matter: others keep their bits."""
    rng = np.random.default_rng(24)
    for new in (4, 40):
        cache, b, q, qf, *rest = setup(rng, [200], [new], [200 - new], 4, 2, 64, 16)
        base = cache.attention(0, b, q, right=0)
        x = q.clone()
        x[0] *= 2.0 ** 100
        x[1] *= 2.0 ** -120
        x[2] = 0.0
        x[3, 1, 5] = float("inf")
        x[3, 2, 6] = float("nan")
        out = cache.attention(0, b, x, right=0)
        assert torch.equal(out[4:], base[4:]) and torch.equal(out[3, 0], base[3, 0]) and torch.equal(out[3, 3], base[3, 3])
        assert bool(torch.isnan(out[3, 2]).all()) and bool(torch.isfinite(out[:3]).all())
        check(out[1:3], None, x[1:3].float().cpu().numpy(), *rest[:3], np.array([0, 2]), [200 - new + 1], 64, right=0)
        cache.close()


@requires_gpu
def test_attention_reads_strided_rows_and_other_layers_and_leaves_rows_behind_the_last():
    rng = np.random.default_rng(4)
    lens, counts, firsts = [50, 90], [2, 5], [48, 85]
    cache, b, q, qf, keys, values, vscale, start = setup(rng, lens, counts, firsts, 8, 4, 64, 16, layers=3, layer=2)
    wide = torch.full((7, 8 * 64 + 72), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 512] = q.view(7, 512)
    res = torch.full((9, 8 * 64 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    out = cache.attention(2, b, wide[:, 8:520], right=0, out=res[:7, :512])
    check(out.reshape(7, 8, 64), None, qf, keys, values, vscale, start, firsts, 64, right=0)
    assert bool((res[7:] == 3.0).all()) and bool((res[:, 512:] == 3.0).all())
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
    from paper_2511_21759_b200 import binding as B
    rng = np.random.default_rng(8)
    for new in (1, 30):
        cache, b, q, *_ = setup(rng, [40, 40], [new, new], [40 - new] * 2, 2, 1, 64, 16, columns=5000 if new > 1 else 1)
        b.table.fill_(-5)
        b.table[1] = 2 ** 31 - 1
        assert bool((cache.attention(0, b, q) == 0).all()) and cache.status() == B.ODB_ERR_STATE
        b.len_after.fill_(2 ** 31 - 1)
        b.first.fill_(-2 ** 31)
        assert bool((cache.attention(0, b, q, right=0) == 0).all()) and cache.status() == B.ODB_ERR_ARG
        for bad in ([0, 1, 2 ** 31 - 1], [-9, -3, -1], [1, 0, 2]):
            b.row_start.copy_(torch.tensor(bad, dtype=torch.int32))
            cache.attention(0, b, q)
            assert cache.status() == B.ODB_ERR_ARG
        cache.close()


@requires_gpu
def test_streams_and_graphs():
    """By turns on two streams, and a store, an attention and a load captured and replayed with other inputs in place."""
    P = paged()
    rng = np.random.default_rng(12)
    lens, counts, firsts = [700, 90], [4, 4], [696, 86]
    cache, b, q, *_ = setup(rng, lens, counts, firsts, 8, 2, 128, 64)
    want = cache.attention(0, b, q, right=0)
    side = torch.cuda.Stream()
    outs = []
    for i in range(6):
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            outs.append(cache.attention(0, b, q, right=0))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    table = b.table.cpu().numpy()
    pos = [696 + i for i in range(4)] + [86 + i for i in range(4)]
    seq = [0] * 4 + [1] * 4
    full = P.Batch(cache, table=b.table, len_after=b.len_after, first=b.first, row_start=b.row_start, row_seq=i32(seq), row_pos=i32(pos),
                   row_slot=i32([table[s][p // 64] * 64 + p % 64 for s, p in zip(seq, pos)]), max_new=4)
    x = torch.empty(8, 12 * 128, dtype=torch.bfloat16, device="cuda")
    rope = P.Rope(128)
    res = [torch.zeros(8, n, 128, dtype=torch.bfloat16, device="cuda") for n in (8, 8, 2, 2)]

    def forward():
        cache.norm_rope_store(0, full, x[:, :1024], x[:, 1024:1280], x[:, 1280:], rope, q_out=res[0])
        cache.attention(0, full, res[0], right=0, out=res[1])
        cache.load(0, full, k_out=res[2], v_out=res[3])

    inputs = [torch.from_numpy(rng.standard_normal((8, 12 * 128)).astype(np.float32)).to(torch.bfloat16).cuda() for _ in range(3)]
    first = cache.kv.view(torch.uint8).clone(), cache.scales.clone()

    def reset(y):
        cache.kv.view(torch.uint8).copy_(first[0])
        cache.scales.copy_(first[1])
        x.copy_(y)

    eager = []
    for y in inputs:
        reset(y)
        forward()
        eager.append([t.clone() for t in res])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        forward()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            forward()
    for y, e in zip(inputs, eager):
        torch.cuda.synchronize()
        reset(y)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(res, e))
    cache.close()


@requires_gpu
def test_prompts_copies_are_made_in_every_call():
    """Layers after one another through one copy's place, eagerly and replayed, with the pool changed in between."""
    rng = np.random.default_rng(31)
    cache, b, q, *_ = setup(rng, [300, 260], [250, 250], [50, 10], 4, 2, 64, 32, layers=2, layer=0, columns=5000)
    raw = cache.kv.view(torch.uint8)
    raw[1].copy_(raw[0].flip(-1))
    cache.scales[1].copy_(cache.scales[0])
    run = lambda: [cache.attention(i, b, q, right=0) for i in (0, 1, 0)]
    want = run()
    assert cache.status() == 0 and bool(torch.isfinite(want[0]).all()) and not torch.equal(want[0], want[1]) and torch.equal(want[0], want[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    raw[0, 1] ^= 0x80                                             # the signs of V of layer 0
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], -want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], -want[0])
    raw[0, 1] ^= 0x80
    assert all(torch.equal(x, y) for x, y in zip(run(), want))
    cache.close()


@requires_gpu
def test_prompts_with_a_table_of_nonsense_stay_inside_the_pool():
    from paper_2511_21759_b200 import binding as B
    rng = np.random.default_rng(8)
    cache, b, q, *_ = setup(rng, [300, 300], [250, 250], [50, 50], 2, 1, 64, 16, columns=5000)
    table, length = b.table.clone(), b.len_after.clone()
    want = cache.attention(0, b, q, right=0)
    b.table.fill_(-5)
    b.table[1] = 2 ** 31 - 1
    assert bool((cache.attention(0, b, q) == 0).all()) and cache.status() == B.ODB_ERR_STATE
    b.len_after.fill_(2 ** 31 - 1)
    b.first.fill_(-2 ** 31)
    assert bool((cache.attention(0, b, q, right=0) == 0).all()) and cache.status() == B.ODB_ERR_ARG
    starts = b.row_start.clone()
    for bad in ([0, 1, 2 ** 31 - 1], [-9, -3, -1], [1, 0, 2]):
        b.row_start.copy_(torch.tensor(bad, dtype=torch.int32))
        cache.attention(0, b, q)
        assert cache.status() == B.ODB_ERR_ARG
    b.row_start.copy_(starts), b.table.copy_(table), b.len_after.copy_(length), b.first.fill_(50)
    assert torch.equal(cache.attention(0, b, q, right=0), want) and cache.status() == 0
    cache.close()


# ---- refusals ---------------------------------------------------------------------------------------------------------

@requires_gpu
def test_calls_that_are_refused():
    P = paged()
    from paper_2511_21759_b200 import binding as B
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 2, 64, 16, 4, dtype=torch.float8_e5m2)
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 2, 64, 16, 4, dtype=E4M3, kv=torch.zeros(1, 2, 4, 2, 16, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        P.PagedCache(1, 4, 2, 64, 16, 4, scales=torch.ones(1, 2, 4, 2, 1, device="cuda"))
    for scales in (torch.ones(1, 2, 4, 2, 2, device="cuda"), torch.ones(1, 2, 4, 2, 1, dtype=torch.float64, device="cuda"), torch.ones(1, 2, 4, 2, 1),
                   torch.ones(1, 2, 4, 2, 2, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            P.PagedCache(1, 4, 2, 64, 16, 4, dtype=E4M3, scales=scales)
    cache = P.PagedCache(1, 4, 2, 64, 16, 4, dtype=E4M3)
    assert cache.scales.shape == (1, 2, 4, 2, 1) and cache.kv.dtype == E4M3
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    rope = P.Rope(64)
    for kw in (dict(row_pos=i32([9]), row_slot=i32([9])), dict(row_seq=i32([0]), row_pos=i32([9]), row_slot=i32([9]))):   # without requests' lengths
        with pytest.raises(B.OdbError) as e:
            cache.norm_rope_store(0, P.Batch(cache, **kw), q, kv, kv, rope)
        assert e.value.status == B.ODB_ERR_ARG
    b = P.Batch(cache, len_after=i32([10]), row_seq=i32([0]), row_pos=i32([9]), row_slot=i32([9]))
    cache.norm_rope_store(0, b, q, kv, kv, rope)
    for wrong in (kv.float(), kv.cpu(), kv[:, :1], torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            cache.load(0, b, k_out=wrong)
        with pytest.raises(ValueError):
            cache.load(0, b, v_out=wrong)
    flat = torch.zeros(3, 300, dtype=torch.bfloat16, device="cuda")
    rows = P.Batch(cache, row_slot=i32([0, 1, 2]))
    for k_out, v_out in ((flat[:, :128], flat[:, :128]), (flat[:, :128], flat[:, 64:192]), (flat[:, 4:132], flat[:, 136:264])):
        with pytest.raises(B.OdbError) as e:                           # the same rows, rows that overlap, an address off its boundary
            cache.load(0, rows, k_out=k_out, v_out=v_out)
        assert e.value.status == B.ODB_ERR_ARG
    for layer in (-1, 1):
        with pytest.raises(B.OdbError) as e:
            cache.load(layer, rows)
        assert e.value.status == B.ODB_ERR_ARG
    many = B.odb_paged_batch(max_rows=2 ** 29, row_slot=rows.row_slot.data_ptr())      # 32-bit numbers: refused before anything is read
    assert B.lib().odb_paged_load(cache.handle, 0, C.byref(many), flat.data_ptr(), 128, flat.data_ptr() + 2 ** 50, 128, None) == B.ODB_ERR_SHAPE
    other = P.PagedCache(1, 4, 2, 64, 16, 5, dtype=E4M3)
    with pytest.raises(ValueError):
        other.load(0, rows)
    assert cache.status() == 0
    cache.close()
    other.close()
