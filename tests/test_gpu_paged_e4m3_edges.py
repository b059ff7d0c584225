"""The paged cache in 8 bits where its calls meet what earlier ones left behind and numbers at the ends of their ranges.  Bounds are derived
beside each test, before its first run."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O
from test_gpu_paged import dev, paged
from test_gpu_paged_e4m3 import E4M3, VALUES, check, codes_of, i32, make, pool_values, random_pool, setup
from test_paged_e4m3_host import kernel

LOW = 2.0 ** O.LOW_EXP


def binding():
    from paper_2511_21759_b200 import binding as B
    return B


def kernel_of(batch, cache):
    """The kernel that an attention of the batch takes (test_paged_e4m3_host.kernel)."""
    room = cache.workspace.numel() > binding().lib().odb_paged_workspace_bytes(cache.cfg)
    return kernel(batch.n_seqs, batch.max_rows, batch.max_new, cache.n_heads // cache.n_kv_heads, cache.n_kv_heads,
                  batch.table.shape[1] * cache.page_size, room=room)


# ---- positions that nobody has written ----------------------------------------------------------------------------------

def dirty_scales(rng, shape):
    """What memory may hold: NaN, infinities, negative numbers, the largest scale, zero, numbers that are no powers of two."""
    kinds = np.array([np.nan, np.inf, -np.inf, -3.0, 2.0 ** 119, 0.0, 1.7e38, 2.0 ** -100, 5.5], np.float32)
    return torch.from_numpy(kinds[rng.integers(0, len(kinds), shape)])


def store_rows(cache, layer, b, rng, rows, size=1.0):
    """Rows of random values through norm_rope_store without norm and rotation; V, which is what K is too, in 64 bits."""
    KV, D = cache.n_kv_heads, cache.head_dim
    x = torch.from_numpy((rng.standard_normal((rows, KV * D)) * size).astype(np.float32)).to(torch.bfloat16)
    q = torch.zeros(rows, cache.n_heads * D, dtype=torch.bfloat16, device="cuda")
    cache.norm_rope_store(layer, b, q, x.cuda(), x.cuda(), paged().Rope(0))
    return x.double().numpy().reshape(rows, KV, D)


@requires_gpu
@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("chunks", [[8, 8], [1, 1, 1, 30], [5, 60, 3, 100], [17]])
def test_blocks_filled_by_parts_under_the_whole_length_start_afresh(page, chunks):
    """A prompt stored chunk by chunk with the length of the whole from the first on, in pages of other requests' values and of any memory:
    codes and scales are those of a block that held nothing."""
    P = paged()
    rng = np.random.default_rng(page + len(chunks))
    layers, KV, D, n_pages = 3, 3, 64, 40 if page < 1024 else 3
    pool = random_pool(rng, layers, n_pages, KV, page, D)
    cache = make(layers, 6, KV, D, page, n_pages, (pool[0], dirty_scales(rng, pool[1].shape)))
    total = sum(chunks) + 9                                       # the last positions are never written
    free = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).cuda()
    table = torch.full((1, O.pages_of(total, page)), -1, dtype=torch.int32, device="cuda")
    want = [np.zeros((O.pages_of(total, O.BLOCK), KV, O.BLOCK, D)) for _ in range(layers)]
    exps = [np.full((O.pages_of(total, O.BLOCK), KV), O.LOW_EXP) for _ in range(layers)]
    at = 0
    for i, n in enumerate(chunks):
        b = P.Batch(cache, table=table, free_pages=free, len_before=i32([total if i else 0]), len_after=i32([total]), first=i32([at]), count=i32([n]),
                    max_rows=n)
        cache.layout(b)
        for layer in range(layers):
            v = store_rows(cache, layer, b, rng, n, 2.0 ** rng.integers(-3, 4))
            for blk in range(at // O.BLOCK, (at + n - 1) // O.BLOCK + 1):
                rows = [p for p in range(blk * O.BLOCK, (blk + 1) * O.BLOCK) if at <= p < at + n]
                for h in range(KV):
                    want[layer][blk, h], exps[layer][blk, h] = O.quantise_block(want[layer][blk, h], exps[layer][blk, h], v[[p - at for p in rows], h],
                                                                               [p - blk * O.BLOCK for p in rows], total - blk * O.BLOCK)
        at += n
        got, scales, pages = pool_values(cache), cache.scales.cpu().numpy().astype(np.float64), table.cpu().numpy()[0]
        for p in range(at):
            pg, off, blk = pages[p // page], p % page, p // O.BLOCK
            for layer in range(layers):
                assert (scales[layer, :, pg, :, off // O.BLOCK] == 2.0 ** exps[layer][blk]).all(), (i, p, layer)
                assert (got[layer, :, pg, :, off] == want[layer][blk, :, p % O.BLOCK]).all(), (i, p, layer)
    assert cache.status() == 0
    cache.close()


@requires_gpu
def test_a_new_cache_has_scales_that_ask_for_nothing():
    """Rows stored by maps of the caller's own, without layout, into pages that nobody has held."""
    P = paged()
    rng = np.random.default_rng(1)
    torch.full((1 << 22,), float("nan"), device="cuda")           # memory that the allocator may hand out again
    cache = P.PagedCache(2, 4, 2, 64, 32, 30, dtype=E4M3)
    assert bool((cache.scales == LOW).all())
    b = P.Batch(cache, len_after=i32([16]), row_seq=i32([0] * 4), row_pos=i32(range(4)), row_slot=i32(range(64, 68)))
    v = store_rows(cache, 1, b, rng, 4)
    for h in range(2):
        want, e = O.quantise_block(np.zeros((16, 64)), O.LOW_EXP, v[:, h], range(4), 16)
        for i in range(2):
            assert cache.scales[1, i, 2, h, 0].item() == 2.0 ** e
            assert np.array_equal(VALUES[codes_of(cache.kv)[1, i, 2, h, :4]] * 2.0 ** e, want[:4])
    cache.close()


@requires_gpu
@pytest.mark.parametrize("layers,KV,page,seqs", [(1, 1, 16, 1), (5, 3, 32, 7), (2, 8, 64, 300)])
def test_layout_touches_the_scales_of_the_pages_it_hands_out_and_no_others(layers, KV, page, seqs):
    P, B = paged(), binding()
    rng = np.random.default_rng(seqs)
    before = rng.integers(0, 5 * page, seqs)
    after = rng.integers(0, 5 * page, seqs)
    after[0] = before[0] + 3 * page                               # someone takes some
    held, need = ([O.pages_of(int(n), page) for n in v] for v in (before, after))
    n_pages = sum(max(a, b) for a, b in zip(held, need)) + 3
    scales = dirty_scales(rng, (layers, 2, n_pages, KV, page // 16))
    cache = make(layers, KV, KV, 64, page, n_pages, (random_pool(rng, layers, n_pages, KV, page, 64)[0], scales))
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((seqs, 9), -1, np.int32)
    at = 0
    for s in range(seqs):
        table[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    free = np.concatenate([order[at:], np.full(at, -7, np.int32)])
    batch = lambda rows, **kw: P.Batch(cache, table=dev(table), free_pages=dev(free), len_before=i32(before), len_after=i32(after), first=i32(np.zeros(seqs)),
                                       count=i32(kw.get("count", np.zeros(seqs))), max_rows=rows)
    bits = lambda t: t.cpu().view(torch.int32)
    bad = batch(0, count=after)                                   # rows that do not fit: nothing is handed out
    cache.layout(bad)
    assert cache.status() == B.ODB_ERR_SHAPE and torch.equal(bits(cache.scales), bits(scales))
    good = batch(1)
    cache.layout(good)
    assert cache.status() == 0
    now = good.table.cpu().numpy()
    taken = [now[s, i] for s in range(seqs) for i in range(held[s], need[s])]
    assert taken and len(set(taken)) == len(taken)
    want = scales.clone()
    want[:, :, taken] = LOW
    assert torch.equal(bits(cache.scales), bits(want))
    cache.close()


@requires_gpu
def test_layout_of_a_free_list_of_nonsense_touches_no_scales():
    P, B = paged(), binding()
    rng = np.random.default_rng(6)
    scales = dirty_scales(rng, (2, 2, 6, 2, 2))
    cache = make(2, 2, 2, 64, 32, 6, (random_pool(rng, 2, 6, 2, 32, 64)[0], scales))
    for page in (-1, 6, 2 ** 31 - 1, -2 ** 31):
        b = P.Batch(cache, table=i32([[-1] * 4]), free_pages=i32([page] * 6), len_before=i32([0]), len_after=i32([100]), first=i32([0]), count=i32([100]), max_rows=100)
        cache.layout(b)
        assert cache.status() == B.ODB_ERR_STATE and bool((b.row_slot == -1).all())
        assert torch.equal(cache.scales.cpu().view(torch.int32), scales.view(torch.int32))
    cache.close()


# ---- scores at the end of their range -----------------------------------------------------------------------------------

@pytest.fixture(params=["narrow", "wide", "wide without room"])
def columns(request):
    return {"narrow": 1, "wide": 5000, "wide without room": -5000}[request.param]


def exact_setup(rng, n, new, G, D, columns, k, v, k_exp, v_exp, q):
    """One request of n positions, 2 K/V heads: values k, v [n][2][D] as codes under the blocks' exponents k_exp, v_exp [blocks][2] (all of
    them exact); q [new][2 G][D] at the last positions."""
    P = paged()
    page, blocks = 16, O.pages_of(n, 16)
    n_pages = blocks + 2
    codes, scales = (t.numpy() for t in random_pool(rng, 1, n_pages, 2, page, D, poison=True))
    order = rng.permutation(n_pages)[:blocks]
    for i, (x, e) in enumerate(((k, k_exp), (v, v_exp))):
        for blk in range(blocks):
            part = x[blk * 16:(blk + 1) * 16]
            for h in range(2):
                y = part[:, h] / 2.0 ** e[blk, h]
                assert np.array_equal(O.e4m3_round(y), y)
                c = np.searchsorted(VALUES[:127], np.abs(y)).astype(np.uint8) | np.where(np.signbit(y), 128, 0).astype(np.uint8)
                codes[0, i, order[blk], h, :len(part)] = c
                scales[0, i, order[blk], h, 0] = 2.0 ** e[blk, h]
    cache = make(1, 2 * G, 2, D, page, n_pages, (torch.from_numpy(codes), torch.from_numpy(scales)), room=columns > 0)
    table = np.full((1, blocks + abs(columns)), 10 ** 6, np.int32)
    table[0, :blocks] = order
    b = P.Batch(cache, table=dev(table), len_after=i32([n]), first=i32([n - new]), row_start=i32([0, new]), max_rows=new, max_new=new)
    qb = torch.from_numpy(q.astype(np.float32)).to(torch.bfloat16)
    assert np.array_equal(qb.double().numpy(), q)
    return cache, b, qb.cuda()


@requires_gpu
@pytest.mark.parametrize("new", [2, 3, 40, 250])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.25, -0.25])
def test_a_score_of_zero_stays_zero_whatever_factors_it(new, D, scale, columns):
    """Queries of 2^100 in one dim, keys under a scale of 2^119 that are zero there: all scores are zero, a row's output is the mean of what
    it sees (weights are equal, so that their rounding is none of the mean's): rounded to bf16, and the sums in fp32."""
    rng = np.random.default_rng(new + D)
    n, G = 300, 4
    k = rng.integers(-7, 8, (n, 2, D)) * 2.0 ** 119
    k[..., 5] = 0.0
    v = rng.integers(-8, 9, (n, 2, D)) * 1.0
    q = np.zeros((new, 2 * G, D))
    q[..., 5] = 2.0 ** 100
    blocks = O.pages_of(n, 16)
    cache, b, qb = exact_setup(rng, n, new, G, D, columns, k, v, np.full((blocks, 2), 119), np.zeros((blocks, 2), int), q)
    lse = torch.empty(new, 2 * G, device="cuda")
    out = cache.attention(0, b, qb, scale=scale, right=0, lse=lse).double().cpu().numpy()
    assert cache.status() == 0
    for r in range(new):
        ok = n - new + r + 1
        want = np.repeat(v[:ok].mean(0), G, 0)
        assert (np.abs(out[r] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * 8).all(), r
        assert np.allclose(lse[r].cpu().numpy(), np.log(ok), rtol=2.0 ** -21, atol=0), r
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new,G,columns", [(4, 4, 1), (40, 4, 1), (40, 4, 5000), (40, 4, -5000), (250, 4, 5000), (250, 4, -5000)])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_that_are_large_small_zero_or_not_finite_in_every_kernel(new, G, columns, D):
    """A row's queries are its own matter.  (Many rows' kernels round the scores of 32 packed rows first where one of them is beyond 2^22: the
    others keep their values, not their last bits.)"""
    rng = np.random.default_rng(24)
    cache, b, q, qf, *rest = setup(rng, [400], [new], [400 - new], 2 * G, 2, D, 16, columns=columns)
    assert kernel_of(b, cache) == {(4, 1): 16, (40, 1): 16, (40, 5000): 1, (40, -5000): 1, (250, 5000): 2, (250, -5000): 1}[new, columns]
    x = q.clone()
    x[0] *= 2.0 ** 100
    x[1] *= 2.0 ** -120
    x[2] = 0.0
    x[3, 1, 5] = float("inf")
    x[3, 2, 6] = float("nan")
    out = cache.attention(0, b, x, right=0)
    assert cache.status() == 0
    assert bool(torch.isnan(out[3, 2]).all()) and bool(torch.isfinite(out[:3]).all()) and bool(torch.isfinite(out[4:]).all())
    check(out[1:3], None, x[1:3].float().cpu().numpy(), *rest[:3], np.array([0, 2]), [400 - new + 1], D, right=0)
    x[3, 1:3] = 0.0                                               # the row's other heads against the oracle, and its two by themselves
    check(cache.attention(0, b, x, right=0)[3:4], None, x[3:4].float().cpu().numpy(), *rest[:3], np.array([0, 1]), [400 - new + 3], D, right=0)
    keep = [0] + list(range(3, 2 * G))
    same = cache.attention(0, b, x, right=0)[3, keep]
    assert bool(torch.isfinite(out[3, keep]).all()) and torch.allclose(out[3, keep].float(), same.float(), rtol=2.0 ** -7, atol=2.0 ** -16)   # a step, and a sum's roundings
    if new > 4:
        check(out[4:20], None, x[4:20].float().cpu().numpy(), *rest[:3], np.array([0, 16]), [400 - new + 4], D, right=0)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new", [2, 5, 45, 240])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [2.0 ** 20, -2.0 ** 20, 2.0 ** 23])
def test_scores_beyond_2_to_22_with_winners_and_ties(new, D, scale, columns):
    """Whole numbers times a power of two: every product and sum is exact, and rows have the mean of their winners, whose blocks have different
    scales of K and of V.  A tie's weights round alike (by 2^-8 in bf16), the output by 2^-8; the others' weights are 0.  The log-sum-exp: the
    scale's rounding, a product's and the two of its way to base e, 2^-24 each."""
    rng = np.random.default_rng(new + D)
    n, G = 333, 4
    blocks = O.pages_of(n, 16)
    k = rng.integers(-1, 2, (n, 2, D)) * (rng.random((n, 2, D)) < 0.1) * 1.0
    for j in rng.integers(0, n, 60):                              # the same key in many blocks
        k[j] = k[3]
    v = rng.integers(-8, 9, (n, 2, D)) * 1.0
    e = rng.integers(-4, 1, (2, blocks, 2))
    v = v * 2.0 ** np.repeat(e[1], 16, 0)[:n][..., None]
    q = rng.integers(-2, 3, (new, 2 * G, D)) * 1.0
    cache, b, qb = exact_setup(rng, n, new, G, D, columns, k, v, e[0], e[1], q)
    lse = torch.empty(new, 2 * G, device="cuda")
    out = cache.attention(0, b, qb, scale=scale, right=0, lse=lse).double().cpu().numpy()
    lse = lse.double().cpu().numpy()
    assert cache.status() == 0
    ties = 0
    for r in range(new):
        ok = n - new + r + 1
        for h in range(2 * G):
            x = k[:ok, h // G] @ q[r, h] * scale
            win = x == x.max()
            ties += win.sum() > 1
            want, mag = v[:ok, h // G][win].mean(0), np.abs(v[:ok, h // G][win]).mean(0)
            assert (np.abs(out[r, h] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * mag).all(), (r, h)
            assert abs(lse[r, h] - (x.max() + np.log(win.sum()))) <= 2.0 ** -21 * (1 + abs(x.max())), (r, h)
    assert ties
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new", [2, 40, 250])
@pytest.mark.parametrize("scale", [8.0, -2.0 ** -8])
def test_queries_of_the_largest_numbers_meet_keys_of_the_smallest(new, scale, columns):
    """Queries of 2^127, keys under the smallest scales: scores of some 2^20 and 2^30, exact but for the scale's rounding; bounds as above."""
    rng = np.random.default_rng(new)
    n, G, D = 333, 4, 64
    blocks = O.pages_of(n, 16)
    k = rng.integers(-1, 2, (n, 2, D)) * (rng.random((n, 2, D)) < 0.1) * 2.0 ** -98
    e = np.stack([rng.integers(-100, -97, (blocks, 2)), np.zeros((blocks, 2), int)])
    v = rng.integers(-8, 9, (n, 2, D)) * 1.0
    q = rng.integers(-1, 2, (new, 2 * G, D)) * 2.0 ** 127
    cache, b, qb = exact_setup(rng, n, new, G, D, columns, k, v, e[0], e[1], q)
    lse = torch.empty(new, 2 * G, device="cuda")
    out = cache.attention(0, b, qb, scale=scale, right=0, lse=lse).double().cpu().numpy()
    lse = lse.double().cpu().numpy()
    assert cache.status() == 0
    for r in range(new):
        ok = n - new + r + 1
        for h in range(2 * G):
            x = k[:ok, h // G] @ q[r, h] * scale
            win = x == x.max()
            want, mag = v[:ok, h // G][win].mean(0), np.abs(v[:ok, h // G][win]).mean(0)
            assert (np.abs(out[r, h] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * mag).all(), (r, h)
            assert abs(lse[r, h] - (x.max() + np.log(win.sum()))) <= 2.0 ** -21 * (1 + abs(x.max())), (r, h)
    cache.close()


# ---- many small weights beside a large one ------------------------------------------------------------------------------

@requires_gpu
@pytest.mark.parametrize("new", [1, 2, 4, 40, 250])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gap", [20, 24, 27])
@pytest.mark.parametrize("at", [0, 2000])
def test_small_weights_beside_a_large_one_reach_the_output(new, D, gap, at, columns):
    """One key, whose V is zero, takes a weight 2^gap times that of each of 4000 others, whose V are one.  Weights in f16: off by 2^-11 of
    themselves or by half of 2^-24, in a unit in which the row's largest product of weight and scale is 2^6 at least: 2^-31 of it a weight.
    In bf16, 2^-8.  The gap's own roundings, in fp32 at 27, are below 2^-17; the output's, 2^-8."""
    rng = np.random.default_rng(new + D)
    n, G = 4001 + new, 4
    blocks = O.pages_of(n, 16)
    k, v = np.zeros((n, 2, D)), np.ones((n, 2, D))
    k[at, :, 3], v[at] = 1.0, 0.0
    q = np.zeros((new, 2 * G, D))
    q[..., 3] = 1.0
    cache, b, qb = exact_setup(rng, n, new, G, D, columns, k, v, np.full((blocks, 2), -8), np.full((blocks, 2), -8), q)
    out = cache.attention(0, b, qb, scale=gap * float(np.log(2.0)), right=0).double().cpu().numpy()
    assert cache.status() == 0
    others = n - new + np.arange(new)
    small = others * 2.0 ** -gap
    want = small / (1 + small)
    tol = want * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -17) + others * 2.0 ** -31
    assert (np.abs(out - want[:, None, None]) <= tol[:, None, None]).all(), (np.abs(out - want[:, None, None]).max(), want.max())
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new,G,takes", [(1, 4, 8), (4, 4, 16), (1, 1, 8)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gap", [27, 34])
def test_small_weights_in_shares_of_many_keys(new, G, takes, D, gap):
    """The same for many requests over the same pages, whose CTAs have long shares: in the kernel of few rows half of f16's last step is 2^-40 of
    the row's largest product of weight and scale."""
    P = paged()
    n, seqs = 8001, 100
    blocks = O.pages_of(n, 16)
    k, v = np.zeros((n, 2, D)), np.ones((n, 2, D))
    k[40, :, 3], v[40] = 1.0, 0.0
    q = np.zeros((new, 2 * G, D))
    q[..., 3] = 1.0
    cache, b, qb = exact_setup(np.random.default_rng(D), n, new, G, D, 1, k, v, np.full((blocks, 2), -8), np.full((blocks, 2), -8), q)
    many = P.Batch(cache, table=b.table.repeat(seqs, 1), len_after=i32([n] * seqs), first=i32([n - new] * seqs), row_start=i32(np.arange(seqs + 1) * new),
                   max_rows=seqs * new, max_new=new)
    assert kernel_of(many, cache) == takes
    out = cache.attention(0, many, qb.repeat(seqs, 1, 1), scale=gap * float(np.log(2.0))).double().cpu().numpy()
    assert cache.status() == 0
    want = (n - 1) * 2.0 ** -gap / (1 + (n - 1) * 2.0 ** -gap)
    assert (np.abs(out - want) <= want * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -17) + (n - 1) * 2.0 ** -40).all(), (np.abs(out - want).max(), want)
    cache.close()


@requires_gpu
@pytest.mark.parametrize("new", [1, 4, 40, 250])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("exp", [-100, 105, "zeros"])
def test_values_under_the_smallest_and_under_large_scales(new, D, exp, columns):
    """V of whole numbers under one exponent, or zeros, whose blocks have the smallest scale; scores that rise by 20 along the keys.  bf16 has
    eight significant bits, steps of 2^-7 from 1 on: a weight's rounding behind the copy is half of that, 2^-8 of the weight, and so is the
    output's (2^-9, half a step at the end of an octave, is not the bound).  A score's roundings, fp32 at 30, stay below 2^-13 of a weight."""
    rng = np.random.default_rng(new + D)
    n, G = 700, 4
    blocks, e = O.pages_of(n, 16), -100 if exp == "zeros" else exp
    k = rng.integers(-1, 2, (n, 2, D)) * (rng.random((n, 2, D)) < 0.2) * 1.0
    k[..., 3] = (np.arange(n) // 47)[:, None]                      # 0 .. 14, by which the scores rise
    k_exp = np.zeros((blocks, 2), int)
    v = rng.integers(-8, 9, (n, 2, D)) * 2.0 ** e * (exp != "zeros")
    q = rng.integers(-2, 3, (new, 2 * G, D)) * 0.25
    q[..., 3] = 1.5
    cache, b, qb = exact_setup(rng, n, new, G, D, columns, k, v, k_exp, np.full((blocks, 2), e), q)
    lse = torch.empty(new, 2 * G, device="cuda")
    out = cache.attention(0, b, qb, scale=1.0, right=0, lse=lse).double().cpu().numpy()
    lse = lse.double().cpu().numpy()
    assert cache.status() == 0
    for r in range(new):
        ok = n - new + r + 1
        for h in range(2 * G):
            x = k[:ok, h // G] @ q[r, h]
            z = x.max() + np.log(np.exp(x - x.max()).sum())
            w = np.exp(x - z)
            want, mag = w @ v[:ok, h // G], w @ np.abs(v[:ok, h // G])
            assert (np.abs(out[r, h] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mag).all(), (r, h)
            assert abs(lse[r, h] - z) <= 2.0 ** -16, (r, h)
    cache.close()


# ---- a store directly in front --------------------------------------------------------------------------------------------

@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,room,takes", [(40, False, 1), (250, False, 1), (250, True, 2), (3, False, 16)])
def test_a_store_directly_in_front_of_the_attention(new, room, takes, D):
    """The same forwards with new values each time: with the device idle between the two calls, one behind the other, and replayed from a graph."""
    P = paged()
    rng = np.random.default_rng(new)
    G, KV, page, lens = 4, 2, 16, [400, 333]
    cache, b, *_ = setup(rng, lens, [new, new], [n - new for n in lens], KV * G, KV, D, page, columns=5000 if room else -5000)
    table = b.table.cpu().numpy()
    pos = np.concatenate([np.arange(n - new, n) for n in lens])
    seq = np.repeat([0, 1], new)
    full = P.Batch(cache, table=b.table, len_after=b.len_after, first=b.first, row_start=b.row_start, row_seq=i32(seq), row_pos=i32(pos),
                   row_slot=i32(table[seq, pos // page] * page + pos % page), max_new=new)
    assert kernel_of(full, cache) == takes
    rope = P.Rope(D)
    x = torch.empty(2 * new, (G + 2) * KV * D, dtype=torch.bfloat16, device="cuda")
    q, out = (torch.empty(2 * new, KV * G, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a, c = KV * G * D, KV * (G + 1) * D
    inputs = [torch.randn(x.shape, device="cuda").to(torch.bfloat16) * 2.0 ** (i % 5 - 2) for i in range(12)]
    first = cache.kv.view(torch.uint8).clone(), cache.scales.clone()

    def start(y):
        cache.kv.view(torch.uint8).copy_(first[0])
        cache.scales.copy_(first[1])
        x.copy_(y)

    def forward(between=lambda: None):
        cache.norm_rope_store(0, full, x[:, :a], x[:, a:c], x[:, c:], rope, q_out=q)
        between()
        cache.attention(0, full, q, right=0, out=out)

    def passes(run):
        got = []
        for y in inputs:
            start(y)
            run()
            got.append(out.clone())
        return got

    want = passes(lambda: forward(torch.cuda.synchronize))
    assert cache.status() == 0 and all(bool(torch.isfinite(w).all()) for w in want) and not torch.equal(want[0], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        forward()
    for _ in range(5):
        assert all(torch.equal(u, w) for u, w in zip(passes(forward), want))
        assert all(torch.equal(u, w) for u, w in zip(passes(g.replay), want))
    cache.close()
