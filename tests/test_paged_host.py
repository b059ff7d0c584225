"""The paged cache's host side and its oracle on a machine without a GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import paged_oracle as O


def B():
    from paper_2511_21759_b200 import binding
    return binding


# ---- the oracle against independent statements of the same thing --------------------------------------------------------

def test_oracle_layout_conserves_pages_and_places_rows():
    rng = np.random.default_rng(0)
    page, n = 16, 12
    length = np.zeros(n, np.int64)
    n_pages = n * 8
    table, free = np.full((n, 8), -1, np.int32), rng.permutation(n_pages).astype(np.int32)
    where = {}                                               # (request, position) -> slot, as long as the position is held
    for _ in range(30):
        after = rng.integers(0, 8 * page + 1, n)
        count = np.minimum(after, 5)
        first = after - count
        table, free, start, seq, pos, slot = O.layout(table, free, length, after, first, count, page, int(count.sum()) + 2)
        held = [p for s in range(n) for p in table[s, :O.pages_of(int(after[s]), page)]]
        n_free = n_pages - len(held)
        assert sorted(held + list(free[:n_free])) == list(range(n_pages))
        for s in range(n):
            for p in range(int(min(length[s], after[s]))):   # what is held on both sides stays where it is
                now = table[s, p // page] * page + p % page
                assert where[s, p] == now
            for p in range(int(after[s])):
                where[s, p] = table[s, p // page] * page + p % page
        assert start[-1] == count.sum() and (seq[start[-1]:] == -1).all()
        for r in range(start[-1]):
            assert slot[r] == where[seq[r], pos[r]] and first[seq[r]] <= pos[r] < after[seq[r]]
        length = after


def test_oracle_attention_is_a_masked_softmax_over_all_pairs():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((30, 2, 8)), rng.standard_normal((30, 2, 8))
    pos = np.arange(20, 25)
    for mask in (dict(), dict(right=0), dict(left=3, right=2, sinks=2), dict(left=0, right=0)):
        out, lse, _, _ = O.attention(q, k, v, pos, **mask)
        for h in range(4):
            s = q[:, h] @ k[:, h // 2].T / np.sqrt(8)
            j, p = np.arange(30)[None], pos[:, None]
            hide = np.zeros((5, 30), bool)
            if "right" in mask:
                hide |= j > p + mask["right"]
            if "left" in mask:
                hide |= (j < p - mask["left"]) & (j >= mask.get("sinks", 0))
            w = np.where(hide, 0, np.exp(s))
            assert np.allclose(out[:, h], (w / w.sum(1, keepdims=True)) @ v[:, h // 2]) and np.allclose(lse[:, h], np.log(w.sum(1)))
    out, lse, _, _ = O.attention(q, k[:0], v[:0], pos)
    assert (out == 0).all() and (lse == -np.inf).all()


def test_oracle_rotation_keeps_relative_positions():
    rng = np.random.default_rng(2)
    for inter in (False, True):
        f, m = O.frequencies(16)
        a, b = rng.standard_normal((1, 1, 24)), rng.standard_normal((1, 1, 24))
        at = lambda x, p: O.norm_rope(x, None, 0, np.array([p]), f, m, inter)[0, 0]
        assert np.isclose(at(a, 7) @ at(b, 3), at(a, 104) @ at(b, 100))
        assert np.array_equal(at(a, 9)[16:], a[0, 0, 16:])


# ---- host calls of the library ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("scaling,name", [(0, "none"), (1, "linear"), (2, "ntk"), (3, "yarn")])
@pytest.mark.parametrize("rot", [8, 64, 128])
def test_rope_frequencies(scaling, name, rot):
    turns, mag = (C.c_uint64 * 64)(), C.c_float()
    factor = 1.0 if scaling == 0 else 8.0
    assert B().lib().odb_rope_frequencies(rot, 10000.0, scaling, factor, 4096.0, 1.0, 32.0, turns, C.byref(mag)) == 0
    f, m = O.frequencies(rot, 10000.0, name, factor, 4096)
    got = np.array(turns[: rot // 2], dtype=np.uint64).astype(np.float64) / 2.0 ** 64
    assert np.allclose(got, f / (2 * np.pi), rtol=1e-14, atol=2.0 ** -60) and np.isclose(mag.value, m, rtol=1e-7)


def test_rope_frequencies_refuses():
    b = B()
    turns, mag = (C.c_uint64 * 64)(), C.c_float()
    call = lambda rot=64, theta=1e4, sc=0, f=1.0, n=4096.0, lo=1.0, hi=32.0, t=turns: b.lib().odb_rope_frequencies(rot, theta, sc, f, n, lo, hi, t, C.byref(mag))
    assert call() == b.ODB_OK and call(rot=0) == b.ODB_OK
    for kw in (dict(rot=4), dict(rot=136), dict(rot=-8)):
        assert call(**kw) == b.ODB_ERR_SHAPE, kw
    for kw in (dict(theta=0.9), dict(theta=float("nan")), dict(sc=4), dict(sc=-1), dict(sc=1, f=0.5), dict(sc=3, f=2.0, n=0.0),
               dict(sc=3, f=2.0, lo=32.0), dict(sc=2, f=float("inf")), dict(t=None)):
        assert call(**kw) == b.ODB_ERR_ARG, kw


def test_sizes_and_configurations():
    b = B()
    size = lambda **kw: (lambda c: (b.lib().odb_paged_kv_bytes(C.byref(c)), b.lib().odb_paged_workspace_bytes(C.byref(c))))(
        b.odb_paged_config(*(dict(n_layers=3, n_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=10) | kw).values()))
    kv, ws = size()
    assert kv == 3 * 2 * 10 * 2 * 64 * 128 * 2 and ws > 0
    for kw in (dict(n_layers=0), dict(n_heads=0), dict(n_heads=9), dict(n_kv_heads=0), dict(head_dim=96), dict(page_size=8), dict(page_size=48),
               dict(page_size=2048), dict(n_pages=0), dict(n_pages=1 << 27), dict(n_heads=2048)):
        assert size(**kw) == (0, 0), kw
    assert b.lib().odb_paged_kv_bytes(None) == 0
    # slots and pool rows stay below 2^31: 2^31 - 2^16 rows of 64 values are 256 GB
    assert size(n_layers=1, n_kv_heads=1, n_heads=1, head_dim=64, page_size=1024, n_pages=(1 << 20) - 64)[0] > 0
    assert size(n_layers=1, n_kv_heads=1, n_heads=1, head_dim=64, page_size=1024, n_pages=1 << 20)[0] == 0


def test_null_arguments_are_refused():
    b = B()
    lib, out = b.lib(), C.c_void_p()
    cfg = b.odb_paged_config(1, 4, 2, 64, 16, 4)
    assert lib.odb_paged_create(None, None, 0, None, 0, None, C.byref(out)) == b.ODB_ERR_ARG
    assert lib.odb_paged_create(C.byref(cfg), None, 1 << 30, None, 1 << 30, None, C.byref(out)) == b.ODB_ERR_ARG
    assert lib.odb_paged_create(C.byref(cfg), 0x10000, 16, 0x20000, 1 << 30, None, C.byref(out)) == b.ODB_ERR_WORKSPACE
    assert lib.odb_paged_create(C.byref(cfg), 0x10010, 1 << 30, 0x20000, 1 << 30, None, C.byref(out)) == b.ODB_ERR_ARG
    batch = b.odb_paged_batch()
    assert lib.odb_paged_layout(None, C.byref(batch), None) == b.ODB_ERR_ARG
    assert lib.odb_paged_attention(None, 0, C.byref(batch), None, 0, None, 0, None, 0.0, -1, -1, 0, None) == b.ODB_ERR_ARG
    assert lib.odb_paged_norm_rope_store(None, 0, C.byref(batch), None, None, 0.0, None) == b.ODB_ERR_ARG
    assert lib.odb_paged_status(None, None) == b.ODB_ERR_ARG and lib.odb_paged_destroy(None) == b.ODB_OK
    assert C.sizeof(b.odb_paged_config) == 6 * 4 and C.sizeof(b.odb_paged_batch) == 4 * 4 + 10 * C.sizeof(C.c_void_p)
    assert C.sizeof(b.odb_paged_rows) == 10 * 8 and C.sizeof(b.odb_rope) == 24


def test_division_by_a_product():
    """The kernels' n / d: m = floor(2^(31 + l) / d) + 1 with l = ceil(log2 d), for every d that a launch can have and n to 2^31."""
    for d in list(range(1, 400)) + [592, 1000, 4095, 4096, 65537]:
        l = (d - 1).bit_length()
        m = (1 << (31 + l)) // d + (d > 1)
        assert m < 1 << 32
        ns = sorted({n for q in (0, 1, 2, 3, 1000, 65535, (2 ** 31 - 1) // d) for n in (q * d - 1, q * d, q * d + 1, q * d + d - 1) if 0 <= n < 2 ** 31} | {2 ** 31 - 1, 2 ** 30})
        assert all((n * m) >> (31 + l) == n // d for n in ns), d


def test_the_paged_attentions_successor_starts_behind_its_tmem_allocation():
    """tcgen05.alloc blocks until columns are free; a successor's CTAs that held them while they wait for this kernel would never
    give them back."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21759_b200", "csrc")
    text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, "paged_attention_tc.cu")).read())
    body = text.split("__global__")[1]
    assert 0 < body.find("tmem_alloc(") < body.find("pdl_launch_dependents()") < body.find("PagedStart start;")


def test_calls_with_another_device_current_go_to_the_caches(monkeypatch):
    """The library refuses a call while another device than the handle's is current: the object layer switches for it and back."""
    import torch

    from paper_2511_21759_b200 import paged as P
    now, seen = [0], []

    class Switch:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, now[0] = now[0], self.device

        def __exit__(self, *_):
            now[0] = self.before

    monkeypatch.setattr(P, "_current_device", lambda: now[0])
    monkeypatch.setattr(P, "_raw_stream", lambda index: 77)
    monkeypatch.setattr(torch.cuda, "device", Switch)

    class Lib:
        def odb_paged_status(self, *_):
            seen.append(("status", now[0]))
            return 5

    monkeypatch.setattr(P.B, "lib", lambda: Lib())
    cache = object.__new__(P.PagedCache)
    batch, rope = object.__new__(P.Batch), object.__new__(P.Rope)
    cache._index, cache._raw, cache.handle, cache.device = 3, 77, None, torch.device("cpu")
    cache.n_heads = cache.n_kv_heads = 1
    cache.head_dim, cache._width, cache._rows_c, cache._rows_ref = 64, 64, P.B.odb_paged_rows(), None
    batch.cache, batch._raw, batch._ref, batch.max_rows = cache, 77, None, 1
    batch._q = batch._kv = (torch.Size((1, 1, 64)), torch.Size((1, 64)))
    rope.index, rope._raw, rope._ref = 3, 77, None
    for name in ("_layout", "_store", "_attention"):
        setattr(cache, name, lambda *_, name=name: seen.append((name, now[0])) or 0)
    monkeypatch.setattr(P.PagedCache, "_rows", lambda self, *_: (0, 64))
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    for device in (0, 3):
        now[0] = device
        cache.layout(batch)
        assert cache.norm_rope_store(0, batch, x, x, x, rope, q_out=x) is x
        assert cache.attention(0, batch, x, out=x) is x
        assert cache.status() == 5 and now[0] == device
    assert seen == [(name, 3) for name in ("_layout", "_store", "_attention", "status")] * 2
