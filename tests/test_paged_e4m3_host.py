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
    batch = b.odb_paged_batch()
    assert lib.odb_paged_load(None, 0, C.byref(batch), None, 0, None, 0, None) == b.ODB_ERR_ARG
    assert b.ODB_PAGED_SCALE_BLOCK == O.BLOCK


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


LAUNCHES = {  # source: {kernel: (threads, CTAs on an SM)}
    "paged_e4m3_store.cu": {("paged_e4m3_store_kernel", d, i, w): (64, 4) for d in (64, 128) for i in (0, 1) for w in (0, 1)},
    "paged_load.cu": {("paged_load_kernel", d, f): (256, 4) for d in (64, 128) for f in (0, 1)},
    "paged_e4m3_attention.cu": {("paged_e4m3_attention_kernel", d, n): (160, 3 if n == 8 else 2) for d in (64, 128) for n in (8, 16)},
}


@pytest.mark.parametrize("source", LAUNCHES)
def test_kernels_fit_and_spill_nothing(source):
    seen = _kernels(source)
    assert set(seen) == set(LAUNCHES[source])
    for kernel, (threads, ctas) in LAUNCHES[source].items():
        registers, spills = seen[kernel]
        # a scheduler's quarter of the registers goes to whole warps
        assert -(-ctas * threads // 128) * 32 * (-(-registers // 8) * 8) <= 16384 and spills == 0, (kernel, registers, spills)
