"""The paged cache in 8 bits on a machine without a GPU: its oracle, sizes and refusals, and what the compiler made of its kernels."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import paged_oracle as O

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21759_b200", "csrc")


def B():
    from paper_2511_21759_b200 import binding
    return binding


# ---- the oracle ---------------------------------------------------------------------------------------------------------

def test_oracle_rounds_to_the_nearest_code():
    torch = pytest.importorskip("torch")
    v = O.e4m3_values()
    assert np.array_equal(v, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 9, 20000), v[:127], (v[:126] + v[1:127]) / 2, [500.0, -1e9]]).astype(np.float32).astype(np.float64)
    got = O.e4m3_round(x)
    fine = np.abs(x) <= 448
    assert np.array_equal(got[fine], torch.from_numpy(x[fine]).float().to(torch.float8_e4m3fn).double().numpy())
    best = np.abs(x[fine, None] - np.concatenate([v[:127], -v[:127]])[None]).min(1)
    assert np.allclose(np.abs(got[fine] - x[fine]), best, rtol=0, atol=0)
    assert (np.abs(got[~fine]) == 448).all() and np.isnan(O.e4m3_round([np.inf, -np.inf, np.nan])).all()
    # half a step: 2^-4 of the value, or 2^-10
    assert (np.abs(got - x)[fine] <= np.maximum(2.0 ** -4 * np.abs(x[fine]), 2.0 ** -10)).all()


def test_oracle_exponents():
    for e in (-100, -7, 0, 5, 119):
        assert O.exponent_for(448 * 2.0 ** e) == e
        if e > -100:
            assert O.exponent_for(224 * 2.0 ** e) == e - 1 and O.exponent_for(224.001 * 2.0 ** e) == e
    assert O.exponent_for(0.0) == -100 and O.exponent_for(1e300) == 119


def test_oracle_block_keeps_what_is_not_written():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((16, 8))
    full, e = O.quantise_block(np.zeros((16, 8)), 0, x, list(range(16)), 16)
    assert e == O.exponent_for(np.abs(x).max()) and np.array_equal(full, O.e4m3_round(x / 2.0 ** e) * 2.0 ** e)
    small, e2 = O.quantise_block(full, e, x[:2] / 100, [3, 4], 16)
    assert e2 == e and np.array_equal(np.delete(small, [3, 4], 0), np.delete(full, [3, 4], 0))       # the exponent of what is kept
    large, e3 = O.quantise_block(full, e, x[:2] * 64, [3, 4], 10)
    assert e3 > e and np.array_equal(large[10:], full[10:])
    assert (np.abs(large[:3] - full[:3]) <= 2.0 ** (e3 - 10)).all()                                  # only the smallest steps are lost
    alone, e4 = O.quantise_block(full, e, x[:2] / 100, [0, 1], 2)                                    # nothing kept: the exponent goes down
    assert e4 == O.exponent_for(np.abs(x[:2]).max() / 100) < e


# ---- host calls ---------------------------------------------------------------------------------------------------------

def test_sizes_and_refusals():
    b = B()
    lib, out = b.lib(), C.c_void_p()
    cfg = b.odb_paged_config(3, 8, 2, 128, 64, 10)
    assert lib.odb_paged_e4m3_kv_bytes(C.byref(cfg)) == 3 * 2 * 10 * 2 * 64 * 128 == lib.odb_paged_kv_bytes(C.byref(cfg)) // 2
    assert lib.odb_paged_e4m3_scale_bytes(C.byref(cfg)) == 3 * 2 * 10 * 2 * 4 * 4
    bad = b.odb_paged_config(3, 8, 2, 96, 64, 10)
    assert lib.odb_paged_e4m3_kv_bytes(C.byref(bad)) == lib.odb_paged_e4m3_scale_bytes(C.byref(bad)) == lib.odb_paged_e4m3_kv_bytes(None) == 0
    ok = dict(cfg=C.byref(cfg), kv=0x10000, kv_bytes=1 << 30, scales=0x20000, scale_bytes=1 << 30, ws=0x30000, ws_bytes=1 << 30, out=C.byref(out))
    create = lambda **kw: (lambda a: lib.odb_paged_create_e4m3(a["cfg"], a["kv"], a["kv_bytes"], a["scales"], a["scale_bytes"], a["ws"], a["ws_bytes"], None, a["out"]))(ok | kw)
    for kw in (dict(cfg=None), dict(kv=None), dict(scales=None), dict(ws=None), dict(out=None), dict(kv=0x10010), dict(scales=0x20004), dict(ws=0x30080)):
        assert create(**kw) == b.ODB_ERR_ARG, kw
    for kw in (dict(kv_bytes=3 * 2 * 10 * 2 * 64 * 128 - 1), dict(scale_bytes=3 * 2 * 10 * 2 * 4 * 4 - 1), dict(ws_bytes=16)):
        assert create(**kw) == b.ODB_ERR_WORKSPACE, kw
    assert create(cfg=C.byref(bad)) == b.ODB_ERR_SHAPE
    assert lib.odb_paged_e4m3_layer_bytes(C.byref(cfg)) == 2 * 10 * 2 * 64 * 128 * 2
    assert lib.odb_paged_e4m3_layer_bytes(C.byref(bad)) == lib.odb_paged_e4m3_layer_bytes(None) == 0
    batch = b.odb_paged_batch()
    assert lib.odb_paged_load(None, 0, C.byref(batch), None, 0, None, 0, None) == b.ODB_ERR_ARG
    assert b.ODB_PAGED_SCALE_BLOCK == O.BLOCK


# ---- which kernel -------------------------------------------------------------------------------------------------------

def kernel(n_seqs, max_rows, max_new, group, kv_heads, longest, room=True, out_stride=4096):
    """The library's own rule, called through its exported name.  8, 16: the kernel of few rows for items of so many; 1: one Q tile of the
    tensor cores; 2: the bf16 copy of the pages; -1: refused."""
    f = B().lib()._ZN3odb30paged_e4m3_attention_kernel_ofEiiiiixxb
    f.argtypes, f.restype = [C.c_int] * 5 + [C.c_longlong] * 2 + [C.c_bool], C.c_int
    return f(n_seqs, max_rows, max_new, group, kv_heads, longest, out_stride, room)


@pytest.mark.parametrize("n_seqs,max_rows,max_new,group,kv_heads,longest,with_room,without", [
    (1, 1, 1, 4, 8, 640, 8, 8), (48, 48, 1, 4, 8, 8192, 8, 8), (48, 48, 0, 4, 8, 8192, 8, 8),          # single tokens
    (4, 4, 1, 12, 8, 8192, 16, 16), (2, 6, 3, 4, 8, 8192, 16, 16), (2, 4, 2, 4, 8, 8192, 8, 8),         # of large groups; a few rows
    (16, 80, 5, 4, 8, 8192, 8, 8), (16, 128, 8, 4, 8, 8192, 16, 16), (16, 144, 9, 4, 8, 8192, 1, 1),
    (2, 64, 32, 4, 8, 64, 16, 16), (16, 512, 32, 4, 8, 4096, 1, 1), (16, 1536, 96, 4, 8, 4096, 1, 1), (16, 1552, 97, 4, 8, 4096, 2, 1),                                     # little work; blocks
    (1, 4096, 4096, 4, 8, 4096, 2, 1), (4, 4900, 1536, 1, 32, 1536, 2, 1),                              # prompts that are alike
    (1, 4096, 0, 4, 8, 4096, 2, 1), (4, 4096, 0, 4, 8, 4096, 2, 1), (16, 2048, 0, 4, 8, 4096, 1, 1),    # whose longest is not known
    (48, 2095, 2048, 4, 8, 8192, 1, 1),                                                                # one among single tokens
    (1, 4096, 4096, 130, 1, 4096, 16, 16),                                                              # a group that no Q tile holds
    (1, 262144, 262144, 4, 8, 262144, 2, 1), (1, 1000000, 1000000, 4, 8, 1000000, 2, -1),               # only two Q tiles can count them
    (1, 1 << 20, 1 << 20, 4, 8, 1 << 20, -1, -1),
])
def test_kernel_of_requests(n_seqs, max_rows, max_new, group, kv_heads, longest, with_room, without):
    assert kernel(n_seqs, max_rows, max_new, group, kv_heads, longest) == with_room
    assert kernel(n_seqs, max_rows, max_new, group, kv_heads, longest, room=False) == without


def test_rows_far_apart_take_the_kernel_of_few_rows():
    at = lambda stride: kernel(1, 4096, 4096, 4, 8, 4096, out_stride=stride)
    assert at(1 << 27) == 2 and at((1 << 27) + 8) == 16 and at(1 << 40) == 16


def test_the_successor_starts_behind_the_tmem_allocation():
    """tcgen05.alloc blocks until columns are free; a successor's CTAs that held them while they wait for this kernel would never
    give them back."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "paged_e4m3_attention_tc.cu")).read())
    body = text.split("__global__")[1]
    assert 0 < body.find("paged_tc_alloc(") < body.find("pdl_launch_dependents()") < body.find("PagedStart start;")


def test_load_with_another_device_current_goes_to_the_caches(monkeypatch):
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
    monkeypatch.setattr(P.PagedCache, "_rows", lambda self, *_: (0, 64))
    cache, batch = object.__new__(P.PagedCache), object.__new__(P.Batch)
    cache._index, cache._raw, cache.handle, cache.n_kv_heads = 3, 77, None, 1
    cache._load = lambda *_: seen.append(now[0]) or 0
    batch.cache, batch._raw, batch._ref, batch._kv = cache, 77, None, ()
    x, y = torch.zeros(1, 64), torch.zeros(1, 64)
    for device in (0, 3):
        now[0] = device
        k, v = cache.load(0, batch, k_out=x, v_out=y)
        assert k is x and v is y and now[0] == device
    assert seen == [3, 3]


# ---- registers ----------------------------------------------------------------------------------------------------------

def _kernels(source):
    """{kernel, template arguments: (registers per thread, spilled bytes)} of a source."""
    r = subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas", "-v", "-c", os.path.join(CSRC, source),
                        "-o", os.devnull], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-2000:]
    out = {}
    for b in re.split(r"ptxas info\s*: Compiling entry function '", r.stderr)[1:]:
        m = re.search(r".*\d(paged_[a-z_0-9]+_kernel)(I(?:L[ib]\d+E)+E)?", b.split("'", 1)[0])
        key = (m.group(1), *map(int, re.findall(r"L[ib](\d+)E", m.group(2) or "")))
        assert key not in out
        out[key] = (int(re.search(r"Used (\d+) registers", b).group(1)), sum(int(x) for x in re.findall(r"(\d+) bytes spill", b)))
    return out


LAUNCHES = {  # source: {kernel: (threads, CTAs on an SM, bytes that may be spilled: stores and loads)}
    "paged_e4m3_store.cu": {("paged_e4m3_store_kernel", d, i, w): (128, 7, 40) for d in (64, 128) for i in (0, 1) for w in (0, 1)},
    "paged_load.cu": {("paged_load_kernel", d, f): (256, 4, 0) for d in (64, 128) for f in (0, 1)} | {("paged_expand_kernel", d): (256, 8, 0) for d in (64, 128)},
    "paged_e4m3_attention.cu": {("paged_e4m3_attention_kernel", d, n): (160, 3 if n == 8 else 2, 0) for d in (64, 128) for n in (8, 16)},
    "paged_e4m3_attention_tc.cu": {("paged_e4m3_attention_tc_kernel", d): (256, 2, 160 if d == 128 else 0) for d in (64, 128)} |
                                  {("paged_merge_kernel", d): (128, 8, 0) for d in (64, 128)},
}


@pytest.mark.parametrize("source", LAUNCHES)
def test_kernels_fit(source):
    seen = _kernels(source)
    assert set(seen) == set(LAUNCHES[source])
    for kernel, (threads, ctas, most) in LAUNCHES[source].items():
        registers, spills = seen[kernel]
        # a scheduler's quarter of the registers goes to whole warps
        assert -(-ctas * threads // 128) * 32 * (-(-registers // 8) * 8) <= 16384 and spills <= most, (kernel, registers, spills)
        if kernel[0] == "paged_e4m3_attention_tc_kernel":
            assert registers == 128, kernel                 # what its warpgroups divide among themselves
