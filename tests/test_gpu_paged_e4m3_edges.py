"""The paged cache in 8 bits where its calls meet what earlier ones left behind and numbers at the ends of their ranges.  Bounds are derived
beside each test, before its first run."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from oracle import paged_oracle as O
from test_gpu_paged import dev, paged
from test_gpu_paged_e4m3 import E4M3, VALUES, codes_of, i32, make, pool_values, random_pool, setup
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
