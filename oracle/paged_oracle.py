"""Paged K/V cache operators on the CPU, in 64 bits and one request, row or head at a time: what block tables, slot maps, the
fused norm / rotation / store and attention over pages compute, written from their definitions (include/odb.h)."""
from __future__ import annotations

import numpy as np


def pages_of(length: int, page: int) -> int:
    return -(-length // page)


def layout(table, free_pages, len_before, len_after, first, count, page: int, max_rows: int):
    """(table, free_pages, row_start, row_seq, row_pos, row_slot) after the forward's lengths; the arguments stay."""
    table, free_pages = table.copy(), free_pages.copy()
    n_pages = len(free_pages)
    held = [pages_of(int(n), page) for n in len_before]
    need = [pages_of(int(n), page) for n in len_after]
    pool = list(free_pages[: n_pages - sum(held)])
    for s in range(len(held)):
        pool += list(table[s, need[s]:held[s]])
    for s in range(len(held)):
        for i in range(held[s], need[s]):
            table[s, i] = pool.pop()
    n_before = n_pages - sum(held)
    free_pages[n_before:max(n_before, len(pool))] = pool[n_before:]
    row_start = np.zeros(len(held) + 1, np.int32)
    maps = np.full((3, max_rows), -1, np.int32)
    r = 0
    for s in range(len(held)):
        for i in range(int(count[s])):
            pos = int(first[s]) + i
            maps[:, r] = s, pos, table[s, pos // page] * page + pos % page
            r += 1
        row_start[s + 1] = r
    return table, free_pages, row_start, maps[0], maps[1], maps[2]


def frequencies(rot_dim, theta=500000.0, scaling="none", factor=1.0, original_len=8192, beta_slow=1.0, beta_fast=32.0):
    """Radians per position of every pair, and the magnitude of cosine and sine."""
    if scaling == "ntk":
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = theta ** (-2.0 * np.arange(rot_dim // 2) / max(rot_dim, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        turns = original_len * f / (2 * np.pi)
        keep = np.clip((turns - beta_slow) / (beta_fast - beta_slow), 0, 1)
        return f * (keep + (1 - keep) / factor), 0.1 * np.log(factor) + 1
    return f, 1.0


def norm_rope(x, gain, eps, pos, freq, magnitude, interleaved):
    """x [rows][heads][head_dim] -> normalised (gain not None) and turned by pos; float64."""
    x = x.astype(np.float64)
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
    half = len(freq)
    R = 2 * half
    a, b = (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(half), np.arange(half, R))
    t = pos.astype(np.float64)[:, None, None] * freq
    y = x.copy()
    y[..., a] = magnitude * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
    y[..., b] = magnitude * (x[..., b] * np.cos(t) + x[..., a] * np.sin(t))
    return y


def visible(length, pos, left=-1, right=-1, sinks=0):
    """Truth value per key j < length for a row at position pos."""
    j = np.arange(length)
    ok = np.ones(length, bool)
    if right >= 0:
        ok &= j <= pos + right
    if left >= 0:
        ok &= (j >= pos - left) | (j < sinks)
    return ok


def attention(q, keys, values, pos, scale=None, left=-1, right=-1, sinks=0):
    """q [rows][heads][hd], keys and values [len][kv heads][hd], pos [rows].  Returns the output, the log-sum-exp, and the
    weights' sum of |v| (what an error of the weights is measured by) and of |q k| (the scores' scale)."""
    rows, H, D = q.shape
    KV = keys.shape[1]
    scale = 1 / np.sqrt(D) if scale is None else scale
    out, mag = np.zeros((rows, H, D)), np.zeros((rows, H, D))
    lse, size = np.full((rows, H), -np.inf), np.zeros((rows, H))
    for r in range(rows):
        ok = visible(len(keys), int(pos[r]), left, right, sinks)
        if not ok.any():
            continue
        for h in range(H):
            k, v = keys[ok, h * KV // H].astype(np.float64), values[ok, h * KV // H].astype(np.float64)
            x = q[r, h].astype(np.float64)
            s = (k @ x) * scale
            m = s.max()
            e = np.exp(s - m)
            w = e / e.sum()
            out[r, h], mag[r, h] = w @ v, w @ np.abs(v)
            lse[r, h] = m + np.log(e.sum())
            size[r, h] = (np.abs(k) @ np.abs(x)).max() * abs(scale)
    return out, lse, mag, size
