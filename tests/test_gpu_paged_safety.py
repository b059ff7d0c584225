"""The paged operators with arguments, maps and objects that are not what they should be: what is refused, what the status word says,
and that the next call is not touched by it."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from test_gpu_paged import _check, _setup, dev, paged


def binding():
    from paper_2511_21759_b200 import binding as B
    return B


def i32(v):
    return dev(np.asarray(v, np.int32))


# ---- rows that do not follow one another ------------------------------------------------------------------------------

def _bad_row_starts(n, rows):
    """row_start arrays of n requests that do not ascend from 0 or more to rows or less."""
    by_turns = np.where(np.arange(n + 1) % 2, rows, 0)
    good = np.linspace(0, rows, n + 1).astype(np.int64)
    back = good.copy()
    back[n // 2] = rows
    early, late, far = good.copy(), good.copy(), good.copy()
    early[0] = -1
    late[-1] = rows + 1
    far[n // 2] = 2 ** 31 - 1
    return dict(by_turns=by_turns, descending=good[::-1], back=back, early=early, late=late, far=far, all_negative=np.full(n + 1, -2 ** 31))


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("seqs", [7, 40])
@pytest.mark.parametrize("new", [1, 8, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_a_row_start_that_does_not_ascend_is_no_work_and_leaves_nothing_behind(D, new, seqs, columns):
    """The grid has CTAs for rows that follow one another: of requests that overlap an item could be left without its last part, and its
    count of arrivals with a remainder for the next call."""
    B = binding()
    rng = np.random.default_rng(seqs + new)
    lens, rows = [150 + 7 * (i % 11) for i in range(seqs)], seqs * new
    cache, b, q, *_ = _setup(rng, lens, [new] * seqs, [n - new for n in lens], 4, 1, D, 16, columns=columns)
    want_lse = torch.empty(rows, 4, device="cuda")
    want = cache.attention(0, b, q, right=0, lse=want_lse)
    assert cache.status() == B.ODB_OK
    good = b.row_start.clone()
    for name, bad in _bad_row_starts(seqs, rows).items():
        b.row_start.copy_(i32(bad))
        out, lse = torch.full_like(q, 3.0), torch.full((rows, 4), 3.0, device="cuda")
        cache.attention(0, b, q, right=0, out=out, lse=lse)
        assert cache.status() == B.ODB_ERR_ARG, name
        assert bool((out == 3.0).all()) and bool((lse == 3.0).all()), name
        b.row_start.copy_(good)
        for _ in range(2):
            lse = torch.empty(rows, 4, device="cuda")
            assert torch.equal(cache.attention(0, b, q, right=0, lse=lse), want) and torch.equal(lse, want_lse), name
        assert cache.status() == B.ODB_OK
    cache.close()


# ---- streams and memory -----------------------------------------------------------------------------------------------

def _delay():
    torch.cuda._sleep(400_000_000)                                # some 0.2 s of the current stream


def _forward(cache, page=16):
    """A small forward over the cache, everything but the cache itself made on the current stream: (batch, rope, qkv)."""
    P = paged()
    n, H, KV, D = 40, cache.n_heads, cache.n_kv_heads, cache.head_dim
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    table = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")
    batch = P.Batch(cache, table=table, free_pages=free, len_before=i32([0]), len_after=i32([n]), first=i32([0]), count=i32([n]), max_rows=n)
    qkv = torch.randn(n, (H + 2 * KV) * D, generator=g, device="cuda").to(torch.bfloat16)
    return batch, P.Rope(D), qkv


def _run(cache, batch, rope, qkv):
    cache.layout(batch)
    a, c = cache.n_heads * cache.head_dim, (cache.n_heads + cache.n_kv_heads) * cache.head_dim
    q = cache.norm_rope_store(0, batch, qkv[:, :a], qkv[:, a:c], qkv[:, c:], rope)
    return cache.attention(0, batch, q, right=0)


@requires_gpu
def test_memory_of_a_cache_a_batch_and_a_rope_is_not_given_back_before_another_stream_is_done_with_it():
    P = paged()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(one):
        cache = P.PagedCache(1, 4, 2, 64, 16, 1024)
        batch, rope, qkv = _forward(cache)
        want = _run(cache, batch, rope, qkv)
    torch.full((1,), 255, dtype=torch.uint8, device="cuda")      # loads the kernel: that may wait for the device
    torch.cuda._sleep(1)
    torch.cuda.synchronize()
    mine = {"workspace": cache.workspace, "kv": cache.kv, "row_start": batch.row_start, "row_seq": batch.row_seq, "row_pos": batch.row_pos,
            "row_slot": batch.row_slot, "turns": rope.turns}
    sizes = {name: (t.numel() * t.element_size(), t.data_ptr()) for name, t in mine.items()}
    del mine
    with torch.cuda.stream(two):
        batch.len_before.fill_(40)                               # its pages are held: the layout changes nothing
        _delay()
        got = _run(cache, batch, rope, qkv)
    cache.close()
    del cache, batch, rope
    with torch.cuda.stream(one):                                 # stream two has not begun: none of that memory may come back
        taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n, _ in sizes.values() for _ in range(3)]
    assert not two.query()
    spans = [(t.data_ptr(), t.data_ptr() + t.numel()) for t in taken]
    for name, (n, p) in sizes.items():
        assert all(p + n <= a or b <= p for a, b in spans), name
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@requires_gpu
def test_a_call_waits_for_the_stream_its_batch_was_used_on():
    """Two caches share a forward's maps: what the first one's layout writes on its stream the second one reads on another."""
    P = paged()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = (P.PagedCache(1, 4, 2, 64, 16, 8, kv=torch.zeros(1, 2, 8, 2, 16, 64, dtype=torch.bfloat16, device="cuda")) for _ in range(2))
    batch, rope, qkv = _forward(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(two):
        b.status()
    with torch.cuda.stream(one):
        a.status()
        batch.row_pos.fill_(-1)
        batch.row_slot.fill_(-1)
        _delay()
        a.layout(batch)
    with torch.cuda.stream(two):
        q = b.norm_rope_store(0, batch, qkv[:, :256], qkv[:, 256:384], qkv[:, 384:], rope)
        out = b.attention(0, batch, q, right=0)
    torch.cuda.synchronize()
    batch.len_before.fill_(40)
    assert torch.equal(out, _run(a, batch, rope, qkv))
    assert torch.equal(a.kv, b.kv)


@requires_gpu
def test_a_capture_leaves_the_order_of_the_calls_around_it():
    """A call captured on another stream is no work of that stream: the next one still waits for the last that ran."""
    P = paged()
    one, two, three = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(one):
        cache = P.PagedCache(1, 4, 2, 64, 16, 8)
        batch, rope, qkv = _forward(cache)
        want = _run(cache, batch, rope, qkv)
    torch.cuda.synchronize()
    batch.len_before.fill_(40)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=two):
        held = _run(cache, batch, rope, qkv)
    assert cache._raw == one.cuda_stream
    with torch.cuda.stream(three):
        assert torch.equal(_run(cache, batch, rope, qkv), want)
        assert cache._raw == batch._raw == three.cuda_stream
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want)
    cache.close()


@requires_gpu
def test_a_batch_without_a_layout_has_no_rows():
    """What a batch makes itself holds nothing that was in that memory before."""
    P = paged()
    cache = P.PagedCache(1, 4, 2, 64, 16, 8, kv=torch.zeros(1, 2, 8, 2, 16, 64, dtype=torch.bfloat16, device="cuda"))
    n = 24
    for _ in range(40):                                          # what the allocator has next: plausible slots and row starts
        torch.arange(n, dtype=torch.int32, device="cuda")
    batch = P.Batch(cache, table=torch.zeros(n - 1, 1, dtype=torch.int32, device="cuda"), len_after=i32([16] * (n - 1)), first=i32([0] * (n - 1)), max_rows=n)
    assert bool((batch.row_start == -1).all()) and all(bool((t == -1).all()) and t.shape == (n,) for t in (batch.row_seq, batch.row_pos, batch.row_slot))
    x = torch.ones(n, 8 * 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full((n, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    cache.norm_rope_store(0, batch, x[:, :256], x[:, 256:384], x[:, 384:], P.Rope(64), q_out=out)
    assert cache.status() == 0
    cache.attention(0, batch, x[:, :256], out=out)
    assert bool((out == 3.0).all()) and bool((cache.kv == 0).all()) and cache.status() == binding().ODB_ERR_ARG
    cache.close()


@requires_gpu
def test_a_layout_comes_behind_the_making_of_its_batch_on_another_stream():
    P = paged()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    cache = P.PagedCache(1, 4, 2, 64, 16, 8)
    ints = [i32(v) for v in ([0], [40], [0], [40])]
    table, free = torch.full((1, 4), -1, dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(two):
        cache.status()
    with torch.cuda.stream(one):
        _delay()
        batch = P.Batch(cache, table=table, free_pages=free, **dict(zip(("len_before", "len_after", "first", "count"), ints)), max_rows=44)
    with torch.cuda.stream(two):
        cache.layout(batch)
    torch.cuda.synchronize()
    assert batch.row_start.cpu().tolist() == [0, 40] and batch.row_pos.cpu().tolist() == list(range(40)) + [-1] * 4
    cache.close()


# ---- rows far apart ---------------------------------------------------------------------------------------------------

@requires_gpu
@pytest.mark.parametrize("rows,stride", [(17, 1 << 30), (100, (1 << 27) + 8), (100, 1 << 27)])
def test_attention_writes_rows_that_are_far_apart(rows, stride):
    """A row's offset within its tile passes 2^31 pieces of 16 bytes (34 GB from the first row to the last)."""
    if torch.cuda.mem_get_info()[0] < 45 << 30:
        pytest.skip("45 GB of free memory are wanted")
    rng = np.random.default_rng(6)
    cache, b, q, qf, keys, values, start = _setup(rng, [300], [rows], [300 - rows], 2, 2, 64, 16, columns=5000)
    wide = torch.empty((rows - 1) * stride + 128, dtype=torch.bfloat16, device="cuda")
    out = wide.as_strided((rows, 128), (stride, 1))
    out.fill_(3.0)
    cache.attention(0, b, q, right=0, out=out)
    assert cache.status() == 0
    _check(out.reshape(rows, 2, 64), None, qf, keys, values, start, [300 - rows], 64, right=0)
    del wide, out
    torch.cuda.empty_cache()
    cache.close()


# ---- a batch of another cache -----------------------------------------------------------------------------------------

@requires_gpu
def test_a_batch_made_for_a_cache_of_other_pages_or_heads_is_refused():
    """Its arrays were checked against that cache: a free list of fewer pages, tensors of fewer heads would be passed on unseen."""
    P = paged()
    first = P.PagedCache(1, 4, 2, 64, 16, 8)
    batch, rope, qkv = _forward(first)
    q, k, v = qkv[:, :256], qkv[:, 256:384], qkv[:, 384:]
    for other in (dict(n_pages=9), dict(n_pages=7), dict(n_heads=8), dict(n_kv_heads=4), dict(head_dim=128), dict(page_size=32)):
        cache = P.PagedCache(**(dict(n_layers=1, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8) | other))
        for call in (lambda: cache.layout(batch), lambda: cache.norm_rope_store(0, batch, q, k, v, rope), lambda: cache.attention(0, batch, q)):
            with pytest.raises(ValueError):
                call()
        assert cache.status() == 0
        cache.close()
    like = P.PagedCache(3, 4, 2, 64, 16, 8)                       # another number of layers
    want = _run(first, batch, rope, qkv)
    batch.len_before.fill_(40)
    assert torch.equal(_run(like, batch, rope, qkv), want)
    like.close()
    first.close()


# ---- outputs that overlap inputs --------------------------------------------------------------------------------------

def _spans(t):
    """The bytes of a [rows][width] bf16 tensor, by rows."""
    return {(t.data_ptr() + 2 * r * t.stride(0) + 2 * i) for r in range(t.shape[0]) for i in range(t.shape[1])}


def _views(flat, rows, width, unit):
    """[rows][width] views of a buffer at offsets and strides that are multiples of `unit` elements, those on their own and those between others'."""
    for stride in (width, width + unit, width + 2 * unit, 2 * width, 2 * width + unit, 3 * width):
        for offset in (0, unit, 2 * unit, width - unit, width, width + unit, 2 * width, 2 * width + unit, rows * width, rows * width - unit, 3 * rows * width):
            if offset + (rows - 1) * stride + width <= flat.numel():
                yield flat.as_strided((rows, width), (stride, 1), offset)


@requires_gpu
@pytest.mark.parametrize("rows", [1, 2, 5])
def test_attention_refuses_an_output_that_overlaps_its_queries_and_no_other(rows):
    B = binding()
    rng = np.random.default_rng(14)
    cache, b, q0, *_ = _setup(rng, [60], [rows], [60 - rows], 1, 1, 64, 16)
    want = cache.attention(0, b, q0, right=0).view(rows, 64)
    flat = torch.zeros(8 * rows * 64, dtype=torch.bfloat16, device="cuda")
    seen = {True: 0, False: 0}
    for q in _views(flat, rows, 64, 8):
        for out in _views(flat, rows, 64, 8):
            q.copy_(q0.view(rows, 64))
            clash = bool(_spans(q) & _spans(out))
            seen[clash] += 1
            if clash:
                with pytest.raises(B.OdbError) as e:
                    cache.attention(0, b, q, right=0, out=out)
                assert e.value.status == B.ODB_ERR_ARG
            else:
                cache.attention(0, b, q, right=0, out=out)
                assert torch.equal(out, want) and torch.equal(q, q0.view(rows, 64))
    assert min(seen.values()) > 20
    cache.close()


@requires_gpu
def test_norm_rope_store_refuses_an_output_that_overlaps_its_inputs_but_for_q_itself():
    P, B = paged(), binding()
    cache = P.PagedCache(1, 1, 1, 64, 16, 4)
    rows = 3
    b = P.Batch(cache, row_pos=i32([5, 6, 7]), row_slot=i32([5, 6, 7]))
    rope = P.Rope(64)
    flat = torch.zeros(8 * rows * 64, dtype=torch.bfloat16, device="cuda")
    other = torch.ones(rows, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(rows, 64, device="cuda").to(torch.bfloat16)
    want = cache.norm_rope_store(0, b, x, other, other, rope).view(rows, 64)
    for source in _views(flat, rows, 64, 4):
        for out in _views(flat, rows, 64, 4):
            same = source.data_ptr() == out.data_ptr() and source.stride() == out.stride()
            clash = bool(_spans(source) & _spans(out))
            for at in "qkv":
                source.copy_(x)
                args = [source if n == at else x if n == "q" else other for n in "qkv"]
                if clash and not (same and at == "q"):
                    with pytest.raises(B.OdbError) as e:
                        cache.norm_rope_store(0, b, *args, rope, q_out=out)
                    assert e.value.status == B.ODB_ERR_ARG
                else:
                    cache.norm_rope_store(0, b, *args, rope, q_out=out)
                    assert torch.equal(out, want)
    cache.close()


# ---- what the attention's tables and lengths lead to ------------------------------------------------------------------

WINDOW = dict(left=40, right=0, sinks=3)


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("new", [1, 9, 60])
@pytest.mark.parametrize("D", [64, 128])
def test_a_page_that_is_none_sets_the_status_word_where_some_row_sees_it(D, new, page, columns):
    B = binding()
    rng = np.random.default_rng(new + page)
    n = 700
    cache, b, q, *_ = _setup(rng, [n, 80], [new, 1], [n - new, 79], 4, 1, D, page, columns=columns)
    table = b.table.clone()
    for mask in (dict(right=0), WINDOW):
        want = cache.attention(0, b, q, **mask)
        assert cache.status() == B.ODB_OK
        lo = n - new - 40                                        # the first position that the window lets some row see
        for p in range(-(-n // page)):
            for none in (-1, cache.n_pages, 2 ** 31 - 1):
                b.table.copy_(table)
                b.table[0, p] = none
                got = cache.attention(0, b, q, **mask)
                seen = "left" not in mask or p == 0 or (p + 1) * page > lo
                assert cache.status() == (B.ODB_ERR_STATE if seen else B.ODB_OK), (p, none)
                if not seen:
                    assert torch.equal(got, want), p
                elif none == -1:                                 # zeros: as if the page were there and cleared
                    b.table.copy_(table)
                    keep = cache.kv[0, :, table[0, p]].clone()
                    cache.kv[0, :, table[0, p]] = 0
                    assert torch.equal(got, cache.attention(0, b, q, **mask)), p
                    cache.kv[0, :, table[0, p]] = keep
        b.table.copy_(table)
        cache.status()
    cache.close()


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("new", [1, 20])
def test_a_window_behind_the_keys_needs_the_pages_of_the_sinks_only(new, columns):
    """Rows at positions whose window begins behind the last key: the pages between the sinks and the end may be gone."""
    B = binding()
    rng = np.random.default_rng(new)
    cache, b, q, *_ = _setup(rng, [40], [new], [200], 4, 1, 64, 16, columns=columns)
    want = cache.attention(0, b, q, **WINDOW)
    b.table[0, 1:3] = -1
    assert torch.equal(cache.attention(0, b, q, **WINDOW), want) and cache.status() == B.ODB_OK
    b.table[0, 0] = -1
    assert bool((cache.attention(0, b, q, **WINDOW) == 0).all()) and cache.status() == B.ODB_ERR_STATE
    cache.close()


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("seqs", [2, 40])
@pytest.mark.parametrize("new", [1, 20])
def test_a_length_that_the_table_has_no_entries_for_is_cut_and_sets_the_status_word(new, seqs, columns):
    B = binding()
    rng = np.random.default_rng(seqs)
    n = 64
    cache, b, q, *_ = _setup(rng, [n] * seqs, [new] * seqs, [n - new] * seqs, 4, 1, 64, 16, columns=columns)
    b.table[:, 4:] = b.table[:, :1]                               # entries behind the length: pages all the same
    width = b.table.shape[1] * 16
    for len1, cut in ((width, width), (width + 1, width), (2 ** 31 - 1, width), (-1, 0), (-2 ** 31, 0)):
        b.len_after.fill_(n)
        b.len_after[seqs - 1] = cut
        want = cache.attention(0, b, q, right=0)
        assert cache.status() == B.ODB_OK
        b.len_after[seqs - 1] = len1
        assert torch.equal(cache.attention(0, b, q, right=0), want)
        assert cache.status() == (B.ODB_OK if len1 == cut else B.ODB_ERR_ARG), len1
    cache.close()


# ---- very long prompts ------------------------------------------------------------------------------------------------

@requires_gpu
def test_attention_of_a_prompt_of_262144_rows():
    """More key tiles of 16 packed rows than 32 bits count, of 256 far fewer; a window keeps the work small."""
    P = paged()
    n, H, KV, D, page = 262144, 32, 8, 64, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    cache = P.PagedCache(1, H, KV, D, page, n // page)
    cache.kv.normal_(generator=g)
    q = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    table = torch.randperm(n // page, generator=g, device="cuda").to(torch.int32)[None]
    batch = P.Batch(cache, table=table, len_after=i32([n]), first=i32([0]), row_start=i32([0, n]), max_rows=n, max_new=n)
    lse = torch.empty(n, H, device="cuda")
    out = cache.attention(0, batch, q, left=63, right=0, sinks=2, lse=lse)
    assert cache.status() == 0 and bool(out.isfinite().all())
    pages = table[0].cpu().numpy()
    for a in (0, 61, 4095, 131071, 200001, n - 3):                # three rows each: the keys that they see, put together
        rows = np.arange(a, a + 3)
        lo = max(0, a - 63)
        seen = np.concatenate([np.arange(min(2, lo)), np.arange(lo, a + 3)])
        k, v = (cache.kv[0, i, pages[seen // page], :, seen % page].float().cpu().numpy() for i in (0, 1))
        sinks = min(2, lo)
        # the same differences of positions from the keys behind the sinks on: first key lo becomes number `sinks`
        _check(out[rows], lse[rows], q[rows].float().cpu().numpy(), [k], [v], np.array([0, 3]), [a - lo + sinks], D, left=63, right=0, sinks=2)
    del q, out, lse
    cache.close()


# ---- norm, rotation, store: what is not turned, not normed, not stored --------------------------------------------------

@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rot", [0, 8, 24, 56])
@pytest.mark.parametrize("inter", [False, True])
def test_values_behind_the_turned_ones_pass_whatever_they_are(inter, rot, D):
    """An infinity, a NaN or a negative zero behind rot_dim changes no other value and is stored as it is (a NaN as a NaN)."""
    P = paged()
    rng = np.random.default_rng(rot + D)
    rows, H, KV = 9, 4, 2
    clean = dev(rng.standard_normal((rows, H + 2 * KV, D)).astype(np.float32)).to(torch.bfloat16)
    dirty, at = clean.clone(), torch.zeros_like(clean, dtype=torch.bool)
    for r in range(rows):
        for h in range(H + KV):
            for x in (float("inf"), float("-inf"), float("nan"), -0.0):
                j = int(rng.integers(rot, D))
                dirty[r, h, j], at[r, h, j] = x, True
    results = []
    for x in (clean, dirty):
        cache = P.PagedCache(1, H, KV, D, 16, 1, kv=torch.zeros(1, 2, 1, KV, 16, D, dtype=torch.bfloat16, device="cuda"))
        b = P.Batch(cache, row_pos=i32(np.arange(rows) * 977), row_slot=i32(np.arange(rows)))
        q = cache.norm_rope_store(0, b, x[:, :H].contiguous(), x[:, H:H + KV].contiguous(), x[:, H + KV:].contiguous(), P.Rope(rot, interleaved=inter))
        results.append(torch.cat([q, cache.kv[0, 0, 0].transpose(0, 1)[:rows]], 1))
        cache.close()
    (a, b), poison = (t.view(torch.int16) for t in results), dirty[:, :H + KV]
    at = at[:, :H + KV]
    assert torch.equal(a[~at], b[~at])
    got = results[1][at]
    nan = poison[at].isnan()
    assert bool(got[nan].isnan().all()) and torch.equal(got[~nan].view(torch.int16), poison[at][~nan].view(torch.int16))
    assert torch.equal(results[0][..., rot:].contiguous().view(torch.int16), clean[:, :H + KV, rot:].contiguous().view(torch.int16))


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
def test_a_row_without_a_position_stores_nothing_whatever_its_slot(D):
    P = paged()
    rng = np.random.default_rng(D)
    cache = P.PagedCache(1, 2, 2, D, 16, 1, kv=torch.full((1, 2, 1, 2, 16, D), 5.0, dtype=torch.bfloat16, device="cuda"))
    x = dev(rng.standard_normal((6, 2, D)).astype(np.float32)).to(torch.bfloat16)
    b = P.Batch(cache, row_pos=i32([3, -1, 0, -2 ** 31, 7, -1]), row_slot=i32([0, 1, 2, 3, -1, -1]))
    out = torch.full_like(x, 7.0)
    cache.norm_rope_store(0, b, x, x, x, P.Rope(D), q_out=out)
    assert bool((out[[1, 3, 5]] == 7.0).all()) and not bool((out[[0, 2, 4]] == 7.0).any())
    kept = cache.kv[0, :, 0].transpose(1, 2)                       # [K, V][position][head][value]
    assert bool((kept[:, [1, 3, 4, 5]] == 5.0).all()) and bool((kept[:, 6:] == 5.0).all())
    assert torch.equal(kept[1, [0, 2]], x[[0, 2]]) and torch.equal(kept[0, 2], x[2])     # position 0 turns nothing
    cache.close()


@requires_gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,KV,rows", [(1, 1, 1), (2, 1, 33), (6, 2, 7), (16, 16, 20), (9, 3, 65)])
def test_a_norm_of_the_queries_or_of_the_keys_alone(H, KV, rows, D):
    """Units of queries, keys and values share a warp; those with a gain form their sums among themselves."""
    P = paged()
    rng = np.random.default_rng(H + rows)
    x = dev(rng.standard_normal((rows, (H + 2 * KV) * D)).astype(np.float32)).to(torch.bfloat16)
    pos, gain = i32(rng.integers(0, 5000, rows)), {n: dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float32)) for n in "qk"}
    rope, n_pages = P.Rope(D), -(-rows // 16)

    def result(which):
        cache = P.PagedCache(1, H, KV, D, 16, n_pages, kv=torch.zeros(1, 2, n_pages, KV, 16, D, dtype=torch.bfloat16, device="cuda"))
        b = P.Batch(cache, row_pos=pos, row_slot=i32(np.arange(rows)))
        q = cache.norm_rope_store(0, b, x[:, :H * D], x[:, H * D:(H + KV) * D], x[:, (H + KV) * D:], rope,
                                  q_gain=gain["q"] if "q" in which else None, k_gain=gain["k"] if "k" in which else None)
        assert cache.status() == 0
        kv = cache.kv.clone()
        cache.close()
        return q, kv

    both, none, q_only, k_only = (result(w) for w in ("qk", "", "q", "k"))     # both and neither are compared with the oracle elsewhere
    assert not torch.equal(both[0], none[0]) and not torch.equal(both[1], none[1])
    assert torch.equal(q_only[0], both[0]) and torch.equal(q_only[1], none[1])
    assert torch.equal(k_only[0], none[0]) and torch.equal(k_only[1], both[1])


@requires_gpu
@pytest.mark.parametrize("columns", [1, 5000])
@pytest.mark.parametrize("counts", [[1, 37, 5], [300, 290], [310], [1, 1, 1]])
def test_attention_without_a_hint(counts, columns):
    """The longest request is not known: whatever kernel the mean picks."""
    rng = np.random.default_rng(9)
    lens = [320] * len(counts)
    firsts = [n - c for n, c in zip(lens, counts)]
    cache, b, q, qf, keys, values, start = _setup(rng, lens, counts, firsts, 8, 2, 128, 32, columns=columns)
    batch = paged().Batch(cache, table=b.table, len_after=b.len_after, first=b.first, row_start=b.row_start, max_rows=sum(counts))
    assert batch.max_new == 0 and batch._c.max_new == 0
    lse = torch.empty(sum(counts), 8, device="cuda")
    out = cache.attention(0, batch, q, right=0, lse=lse)
    assert cache.status() == 0
    _check(out, lse, qf, keys, values, start, firsts, 128, right=0)
    cache.close()
