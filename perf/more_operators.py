"""The paged cache in 8 bits, as a program that serves a language model meets it.

K and V of every request lie in pages as e4m3 with a scale, a power of two, for each block of 16 positions and K/V head.  Three operators:

  write      queries and keys of every head normalised and turned by their position, keys and values quantised into their slots,
             and the blocks that were touched read back
  read       rows of requests from their slots, as bf16
  attention  rows of each request against its pages, with grouped heads, a window and first tokens that stay visible

`run` computes one pass of one operator, with the package's calls where `own` is true and with elementary torch operations where it is
not.  The pool is e4m3 [layers][2][pages][kv heads][page][head dim], the scales fp32 [layers][2][pages][kv heads][page / 16].

The definitions.  write: y = x / sqrt(mean(x^2) + eps) * gain, then the pairs (i, i + R/2) (half) or (2i, 2i+1) (interleaved) of the
first R dims turned by the angle pos * f_i, cosine and sine multiplied by the method's magnitude; queries rounded to bf16.  Of a block
of 16 positions, one head, K or V: e is the smallest integer with max |x| <= 448 * 2^e over what the call writes of it; where positions
below the request's length are not written by the call, e is at least the block's exponent from before, and their codes are rounded
again under e.  Codes are e4m3(x * 2^-e), to the nearest, ties to even; the scale is 2^e.  read: code * scale (exact in bf16).
attention: key j of a request with `len` keys is visible to position p when j < len, j <= p + right and (j >= p - left or j < sinks);
softmax of q k / sqrt(head dim) over the visible keys, k and v being code * scale; rows that see no key give zeros and a log-sum-exp of
-infinity.
"""
import math
import random

import torch

own = False

_UNLIMITED = 1 << 30
_BLOCK = 16                # positions of a scale
_LOW, _HIGH = -100, 119    # exponents of scales


# ---- the cases ----------------------------------------------------------------------------------------------------

def _write(name, seqs, lo, hi, new, heads, kv_heads, dim, page, rot, interleaved, norm, scaling, factor, middle=False):
    return _named(name, dict(op="write", seqs=seqs, lo=lo, hi=hi, new=new, heads=heads, kv_heads=kv_heads, dim=dim, page=page, rot=rot,
                             interleaved=interleaved, norm=norm, scaling=scaling, factor=factor, middle=middle))


def _read(name, seqs, lo, hi, kv_heads, dim, page):
    return _named(name, dict(op="read", seqs=seqs, lo=lo, hi=hi, new=0, kv_heads=kv_heads, dim=dim, page=page, middle=False))


def _attention(name, seqs, lo, hi, new, heads, kv_heads, dim, page, left=-1, right=-1, sinks=0, middle=False):
    return _named(name, dict(op="attention", seqs=seqs, lo=lo, hi=hi, new=new, heads=heads, kv_heads=kv_heads, dim=dim,
                             page=page, left=left, right=right, sinks=sinks, middle=middle))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token for each of 48 requests: blocks that are filled a row at a time, their scales growing
        _write("write_48_tokens", 48, 1, 8192, 1, 32, 8, 128, 64, 128, False, True, "none", 1.0),
        # blocks of 32 rows of sixteen requests, in the middle of scales' blocks, half of each head turned in interleaved pairs
        _write("write_16x32_part", 16, 700, 4096, 32, 32, 32, 128, 16, 64, True, True, "yarn", 8.0, middle=True),
        # the refresh of a batch: some 25000 rows of 32 + 2 x 8 heads
        _write("write_refresh", 16, 1200, 1999, 0, 32, 8, 128, 64, 128, False, True, "none", 1.0),
        # one short request leaves for another place
        _read("read_577", 1, 577, 577, 8, 128, 16),
        # a batch of sixteen does
        _read("read_16", 16, 3000, 8192, 8, 128, 64),
        # one token of one short request: latency
        _attention("token8_577", 1, 577, 577, 1, 32, 8, 128, 16),
        # one token each of a ragged batch
        _attention("token8_batch_48", 48, 1, 8192, 1, 32, 8, 128, 64, right=0),
        # one token of two very long requests: the work has to be split along the keys
        _attention("token8_long", 2, 100000, 131072, 1, 32, 8, 128, 64, right=0),
        # a window of 4096 with four first tokens kept, head dim 64, sixteen long requests
        _attention("token8_window", 16, 5000, 32768, 1, 16, 4, 64, 32, left=4095, right=0, sinks=4),
        # block steps in the middle of the sequences: 32 rows against all cached keys, in both directions
        _attention("block8_16x32", 16, 700, 4096, 32, 32, 8, 128, 64, middle=True),
        # the refresh of a ragged batch: every row against every row of its request, one K/V head per query head
        _attention("refresh8_4", 4, 900, 1536, 0, 32, 32, 128, 64),
        # a causal prompt of 4096 tokens
        _attention("prompt8_4096", 1, 4096, 4096, 0, 32, 8, 128, 64, right=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "write", "read", "token", "token", "window", "block", "rows"))
    page = rng.choice((16, 32, 64, 128))
    dim = rng.choice((64, 128, 128))
    kv = rng.choice((1, 2, 4, 8))
    group = rng.choice((1, 2, 3, 4, 5, 8))
    if kind == "write":
        rot = dim if rng.random() < 0.6 else rng.choice([r for r in (16, 24, 32, 48, 64, 96) if r < dim])
        scaling = rng.choice(("none", "none", "linear", "ntk", "yarn"))
        seqs = _log(rng, 1, 64)
        whole = rng.random() < 0.4
        new = 0 if whole else rng.choice((1, 1, 5, 16, 32, 47))
        rows = 25000 * 48 * 128 // max((group + 2) * kv * dim, 48 * 128)
        hi = _log(rng, max(50, new), max(60, rows // seqs)) if whole else _log(rng, max(50, new), min(32768, 350000 // seqs))
        return _write(None, seqs, max(1, new, hi // 3), hi, new, kv * group, kv, dim, page, rot, rng.random() < 0.4, rng.random() < 0.75, scaling,
                      1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 32.0)), middle=rng.random() < 0.5)
    if kind == "read":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 20, min(32768, 130000 // seqs))
        return _read(None, seqs, max(1, hi // 4), hi, kv, dim, page)
    if kind == "token":
        seqs = _log(rng, 1, 128)
        hi = _log(rng, 20, min(131072, 350000 // seqs))
        return _attention(None, seqs, rng.choice((1, max(1, hi // 2), hi)), hi, 1, kv * group, kv, dim, page, right=rng.choice((-1, 0)))
    if kind == "window":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 50, min(65536, 350000 // seqs))
        return _attention(None, seqs, max(1, hi // 3), hi, rng.choice((1, 1, 4, 16)), kv * group, kv, dim, page,
                          left=_log(rng, 16, 8192) - 1, right=0, sinks=rng.choice((0, 1, 4, 64, 100)))
    if kind == "block":
        seqs = _log(rng, 1, 32)
        new = rng.choice((2, 7, 16, 32, 64))
        hi = _log(rng, max(80, new), min(16384, 65536 // seqs))
        return _attention(None, seqs, max(new, hi // 2), hi, new, kv * group, kv, dim, page, middle=True)
    seqs = _log(rng, 1, 8)
    hi = _log(rng, 100, 4096 // seqs + 100)
    causal = rng.random() < 0.5
    return _attention(None, seqs, max(1, hi // 2), hi, 0, kv * group, kv, dim, page, right=0 if causal else -1,
                      left=_log(rng, 64, 2048) if causal and rng.random() < 0.3 else -1, sinks=0)


# ---- lengths, which the case alone decides ------------------------------------------------------------------------

def _lens(c):
    """(positions, first position, rows) of every request."""
    rng = random.Random("%(seqs)d %(lo)d %(hi)d %(new)d %(page)d" % c)
    out = []
    for s in range(c["seqs"]):
        n = c["hi"] if s == 0 else rng.randint(c["lo"], c["hi"])
        k = min(n, c["new"]) if c["new"] else n
        first = rng.randrange(0, n - k + 1) if c["middle"] else n - k
        out.append((n, first, k))
    return out


def _pages(n, page):
    return -(-n // page)


def _touched(c):
    """(request, first position, positions) of the scales' blocks that a write touches, as far as the request goes."""
    out = []
    for s, (n, first, k) in enumerate(_lens(c)):
        lo, hi = first // _BLOCK * _BLOCK, min(n, _pages(first + k, _BLOCK) * _BLOCK)
        out.append((s, lo, hi - lo))
    return out


def _span(c, n, first, k):
    """Keys that at least one row of the request sees, and pairs of a row and a key it sees."""
    left = _UNLIMITED if c["left"] < 0 else c["left"]
    right = _UNLIMITED if c["right"] < 0 else c["right"]
    top = min(n, first + k - 1 + right + 1)
    low = min(max(0, first - left), top)
    keys = top - low + min(c["sinks"], low)
    if c["left"] < 0 and c["right"] < 0:
        return keys, n * k
    pairs = 0
    for p in range(first, first + k):
        hi = min(n, p + right + 1)
        lo = min(max(0, p - left), hi)
        pairs += hi - lo + min(c["sinks"], lo)
    return keys, pairs


def work(c):
    KV, D = c["kv_heads"], c["dim"]
    position = 2 * KV * D + 2 * KV * 4 / _BLOCK           # bytes of a position in the pool, K and V, and its part of the scales
    if c["op"] == "read":
        n = sum(k for _, _, k in _lens(c))
        return {"bytes": n * (position + 4 * KV * D + 4), "flops": 2 * n * KV * D}
    if c["op"] == "write":
        n, back = sum(k for _, _, k in _lens(c)), sum(t[2] for t in _touched(c))
        values = n * (c["heads"] + 2 * KV) * D
        # in: projection, what was there of the touched blocks, maps; out: queries, the touched blocks in the pool and as they read
        return {"bytes": 2 * values + (back - n) * position + 12 * n + 2 * n * c["heads"] * D + back * (position + 4 * KV * D + 4),
                "flops": 10 * values}
    spans = [(k,) + _span(c, n, f, k) for n, f, k in _lens(c)]
    rows = sum(s[0] for s in spans)
    return {"bytes": 4 * rows * c["heads"] * D + 4 * rows * c["heads"] + position * sum(s[1] for s in spans),
            "flops": 4 * c["heads"] * D * sum(s[2] for s in spans)}


# ---- inputs -------------------------------------------------------------------------------------------------------

_EPS, _THETA, _ORIGINAL = 1e-6, 500000.0, 8192


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    KV, D, P = c["kv_heads"], c["dim"], c["page"]
    lens = _lens(c)
    held = [_pages(n, P) for n, _, _ in lens]
    n_pages = sum(held) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(held)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(held), device="cuda")[None, :] < ints(held).long()[:, None]] = order[: sum(held)]
    counts = [k for _, _, k in lens]
    rows = sum(counts)
    starts = [0]
    for k in counts:
        starts.append(starts[-1] + k)
    # what the pool holds: normal values whose size differs from block to block, under the exponent that their largest one needs
    shape = (1, 2, n_pages, KV, P // _BLOCK)
    size = torch.exp2(torch.rand(shape, generator=g, device="cuda") * 2 - 1)
    pool = torch.empty(*shape, _BLOCK, D, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(shape, device="cuda")
    for i in range(2):
        for at in range(0, n_pages, 4096):
            x = torch.randn(1, min(4096, n_pages - at), KV, P // _BLOCK, _BLOCK, D, generator=g, device="cuda")
            x *= size[:, i, at:at + 4096, :, :, None, None]
            e = _exponent(x.abs().amax((-1, -2)))
            scales[:, i, at:at + 4096] = _two(e)
            pool[:, i, at:at + 4096] = (x * _two(-e)[..., None, None]).to(torch.float8_e4m3fn)
    s = {"case": c, "n_pages": n_pages, "table": table, "lens": ints([n for n, _, _ in lens]), "first": ints([f for _, f, _ in lens]),
         "row_start": ints(starts), "max_new": max(counts), "rows": rows, "pool": pool.view(1, 2, n_pages, KV, P, D), "scales": scales}
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)
    slots = lambda seq, pos: (table.long()[seq, pos // P] * P + pos % P).to(torch.int32)
    if c["op"] == "attention":
        s.update(q=(normal(rows, c["heads"], D) * 1.5).to(torch.bfloat16), out=torch.empty(rows, c["heads"], D, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(rows, c["heads"], dtype=torch.float32, device="cuda"))
        return s
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), ints(counts).long())
    pos = s["first"].long()[seq] + torch.arange(rows, device="cuda") - s["row_start"].long()[seq]
    rows_out = lambda n: torch.empty(n, KV, D, dtype=torch.bfloat16, device="cuda")
    if c["op"] == "read":
        s.update(slot=slots(seq, pos), k=rows_out(rows), v=rows_out(rows))
        return s
    touched = _touched(c)
    back_n = ints([t[2] for t in touched]).long()
    back_seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), back_n)
    back_pos = torch.arange(back_seq.numel(), device="cuda") - (back_n.cumsum(0) - back_n)[back_seq] + ints([t[1] for t in touched]).long()[back_seq]
    # one projection's output, its parts side by side; rows of different size
    qkv = normal(rows, (c["heads"] + 2 * KV) * D) * torch.exp2(torch.rand(rows, 1, generator=g, device="cuda") * 3 - 1.5)
    s.update(qkv=qkv.to(torch.bfloat16), row_seq=seq.to(torch.int32), row_pos=pos.to(torch.int32), row_slot=slots(seq, pos),
             back_slot=slots(back_seq, back_pos), q_out=torch.empty(rows, c["heads"], D, dtype=torch.bfloat16, device="cuda"),
             k=rows_out(back_seq.numel()), v=rows_out(back_seq.numel()),
             q_gain=1 + 0.2 * normal(D), k_gain=1 + 0.2 * normal(D))
    return s


def _two(e, dtype=torch.float32):
    """2^e, exactly."""
    if dtype == torch.float64:
        return ((e.long() + 1023) << 52).view(dtype)
    return ((e.int() + 127) << 23).view(dtype)


def _exponent(top):
    """The smallest e with top <= 448 * 2^e, in the scales' range: 448 = 0.875 * 2^9."""
    m, e = torch.frexp(top)
    return (e - 9 + (m > 0.875)).clamp(_LOW, _HIGH).masked_fill(top == 0, _LOW)


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"write": _own_write, "read": _own_read, "attention": _own_attention}[op](s)
    return {"write": _plain_write, "read": _plain_read, "attention": _plain_attention}[op](s)


def _handles(s):
    """The cache and batch objects that a program keeps next to its buffers."""
    if "batch" in s:
        return s["cache"], s["batch"]
    from paper_2511_21759_b200 import paged
    c = s["case"]
    heads = c["kv_heads"] if c["op"] == "read" else c["heads"]
    cache = paged.PagedCache(n_layers=1, n_heads=heads, n_kv_heads=c["kv_heads"], head_dim=c["dim"], page_size=c["page"],
                             n_pages=s["n_pages"], kv=s["pool"], scales=s["scales"])
    if c["op"] == "attention":
        batch = paged.Batch(cache, table=s["table"], len_after=s["lens"], first=s["first"], row_start=s["row_start"],
                            max_rows=s["rows"], max_new=s["max_new"])
    elif c["op"] == "read":
        batch = paged.Batch(cache, row_slot=s["slot"])
    else:
        batch = paged.Batch(cache, len_after=s["lens"], row_seq=s["row_seq"], row_pos=s["row_pos"], row_slot=s["row_slot"], max_new=s["max_new"])
        s["back"] = paged.Batch(cache, row_slot=s["back_slot"])
        s["rope"] = paged.Rope(c["rot"], theta=_THETA, interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"],
                               original_len=_ORIGINAL)
    s["cache"], s["batch"] = cache, batch
    return cache, batch


def _own_write(s):
    cache, batch = _handles(s)
    c = s["case"]
    a, b = c["heads"] * c["dim"], (c["heads"] + c["kv_heads"]) * c["dim"]
    qkv = s["qkv"]
    cache.norm_rope_store(0, batch, qkv[:, :a], qkv[:, a:b], qkv[:, b:], s["rope"],
                          q_gain=s["q_gain"] if c["norm"] else None, k_gain=s["k_gain"] if c["norm"] else None, eps=_EPS, q_out=s["q_out"])
    k, v = cache.load(0, s["back"], k_out=s["k"], v_out=s["v"])
    return {"q": s["q_out"], "k": k, "v": v}


def _own_read(s):
    cache, batch = _handles(s)
    k, v = cache.load(0, batch, k_out=s["k"], v_out=s["v"])
    return {"k": k, "v": v}


def _own_attention(s):
    cache, batch = _handles(s)
    c = s["case"]
    cache.attention(0, batch, s["q"], left=c["left"], right=c["right"], sinks=c["sinks"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _values(s, i, slot):
    """K (0) or V (1) of slots, [..][kv heads][head dim] in 32 bits."""
    P = s["case"]["page"]
    page, off = slot.long() // P, slot.long() % P
    codes = s["pool"].view(torch.uint8)[0, i, page, :, off].view(torch.float8_e4m3fn)
    return codes.float() * s["scales"][0, i, page, :, off // _BLOCK][..., None]


def _plain_read(s):
    return {n: _values(s, i, s["slot"]).to(torch.bfloat16) for i, n in enumerate("kv")}


def _frequencies(c, dtype):
    """Turns of each pair in radians per position, and the magnitude of cosine and sine."""
    R, f = c["rot"], c["factor"]
    i = torch.arange(R // 2, device="cuda", dtype=dtype)
    theta = _THETA * f ** (R / (R - 2)) if c["scaling"] == "ntk" else _THETA
    freq = torch.exp(i * (-2.0 / R * math.log(theta)))
    if c["scaling"] == "linear":
        return freq / f, 1.0
    if c["scaling"] == "yarn":
        turns = _ORIGINAL * freq / (2 * math.pi)
        keep = ((turns - 1) / 31).clamp(0, 1)
        return freq * (keep + (1 - keep) / f), 0.1 * math.log(f) + 1
    return freq, 1.0


def _norm_turn(x, gain, cos, sin, c):
    """x [rows][heads][dim] in 32 bits."""
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * gain
    R = c["rot"]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., : R // 2], x[..., R // 2:R])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_write(s):
    c = s["case"]
    H, KV, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    x = s["qkv"].float().view(-1, H + 2 * KV, D)
    freq, mag = _frequencies(c, torch.float64)
    angle = s["row_pos"][:, None].double() * freq         # far positions: in 64 bits
    cos, sin = (torch.cos(angle) * mag).float()[:, None, :], (torch.sin(angle) * mag).float()[:, None, :]
    q = _norm_turn(x[:, :H], s["q_gain"] if c["norm"] else None, cos, sin, c).to(torch.bfloat16)
    k = _norm_turn(x[:, H:H + KV], s["k_gain"] if c["norm"] else None, cos, sin, c)
    new = torch.stack([k, x[:, H + KV:]], 1)              # [rows][2][kv heads][dim]
    # the blocks of positions: their rows follow one another
    seq, pos, slot = s["row_seq"].long(), s["row_pos"].long(), s["row_slot"].long()
    wide = s["table"].shape[1] * P // _BLOCK
    block, mine = torch.unique_consecutive(seq * wide + pos // _BLOCK, return_inverse=True)
    n, dev = block.numel(), x.device
    top = torch.zeros(n, 2, KV, device=dev).index_reduce_(0, mine, new.abs().amax(-1), "amax")
    written = torch.zeros(n, _BLOCK, dtype=torch.bool, device=dev)
    written[mine, pos % _BLOCK] = True
    live = (block % wide * _BLOCK)[:, None] + torch.arange(_BLOCK, device=dev) < s["lens"].long()[block // wide][:, None]
    kept = live & ~written
    at = torch.zeros(n, dtype=torch.long, device=dev)
    at[mine] = slot - pos % _BLOCK                        # the block's first slot
    page, part, off = at // P, at % P // _BLOCK, (at % P)[:, None] + torch.arange(_BLOCK, device=dev)
    before = torch.frexp(s["scales"][0][:, page, :, part])[1] - 1          # [n][2][kv heads]
    e = _exponent(top)
    e = torch.where(kept.any(1)[:, None, None], torch.maximum(e, before), e)
    # codes of the whole block: what was there, rounded again where the exponent has grown, and the new rows over it
    pool = s["pool"].view(torch.uint8)[0]
    old = pool[:, page[:, None], :, off]                  # [n][16][2][kv heads][dim]
    code = (old.view(torch.float8_e4m3fn).float() * _two(before - e)[:, None, :, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    code = torch.where(kept[:, :, None, None, None], code, old)
    code[mine, pos % _BLOCK] = (new * _two(-e)[mine][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    pool[:, page[:, None], :, off] = code
    s["scales"][0][:, page, :, part] = _two(e)
    return {"q": q, **{name: _values(s, i, s["back_slot"]).to(torch.bfloat16) for i, name in enumerate("kv")}}


def _plain_attention(s):
    c = s["case"]
    H, KV, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    B, G, dev = c["seqs"], c["heads"] // c["kv_heads"], s["q"].device
    L = s["table"].shape[1] * P
    table = s["table"].clamp(min=0).long()

    def keys(i):
        code = s["pool"].view(torch.uint8)[0, i][table].view(torch.float8_e4m3fn).float()      # [B][pages][KV][P][D]
        scale = s["scales"][0, i][table].repeat_interleave(_BLOCK, -1)[..., None]
        return code.mul_(scale).permute(0, 2, 1, 3, 4).reshape(B, KV, L, D)

    start, lens, first = s["row_start"].long(), s["lens"].long(), s["first"].long()
    seq = torch.repeat_interleave(torch.arange(B, device=dev), start[1:] - start[:-1])
    i = torch.arange(s["rows"], device=dev) - start[seq]
    q = torch.zeros(B, s["max_new"], H, D, device=dev)
    q[seq, i] = s["q"].float()
    q = q.view(B, s["max_new"], KV, G, D).permute(0, 2, 3, 1, 4).reshape(B, KV, G * s["max_new"], D)
    j = torch.arange(L, device=dev)
    p = (first[:, None] + torch.arange(s["max_new"], device=dev))[:, :, None]
    seen = (j < lens[:, None])[:, None, :]
    if c["right"] >= 0:
        seen = seen & (j <= p + c["right"])
    if c["left"] >= 0:
        seen = seen & ((j >= p - c["left"]) | (j < c["sinks"]))
    score = torch.matmul(q, keys(0).transpose(-1, -2)) * (1 / math.sqrt(D))
    score = score.view(B, KV, G, s["max_new"], L).masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = (score - top).exp_()
    del score
    total = e.sum(-1, keepdim=True)
    v = torch.where((j < lens[:, None])[:, None, :, None], keys(1), torch.zeros((), device=dev))
    out = torch.matmul(e.view(B, KV, -1, L), v).view(B, KV, G, s["max_new"], D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (total.log() + top)[..., 0]
    rows = lambda t: t.permute(0, 3, 1, 2, *range(4, t.dim())).reshape(B, s["max_new"], H, *t.shape[4:])[seq, i]
    return {"out": rows(out).to(torch.bfloat16), "lse": rows(lse)}


# ---- 64 bits ------------------------------------------------------------------------------------------------------

def _e4m3(x):
    """The nearest number of three bits behind the first, down to steps of 2^-9; ties to even."""
    step = _two(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4, torch.float64)
    return torch.round(x / step) * step


def exact(c, seed):
    s = prepare(c, seed)
    KV, D, P = c["kv_heads"], c["dim"], c["page"]

    def pool(i, n):                                       # K or V of request n: [kv heads][positions of its pages][dim], and exponents
        pages = s["table"][n, :_pages(int(s["lens"][n]), P)].long()
        codes = s["pool"][0, i].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double().permute(1, 0, 2, 3).reshape(KV, -1, D)
        e = torch.round(torch.log2(s["scales"][0, i][pages].double())).long().permute(1, 0, 2).reshape(KV, -1)
        return codes, e

    two = lambda e: _two(e, torch.float64).repeat_interleave(_BLOCK, 1)[..., None]      # of the blocks, by positions

    if c["op"] == "read":
        both = []
        for i in range(2):
            rows = []
            for n, (length, first, k) in enumerate(_lens(c)):
                codes, e = pool(i, n)
                rows.append((codes * two(e))[:, first:first + k].transpose(0, 1))
            both.append(torch.cat(rows))
        return {"k": both[0], "v": both[1]}
    H = c["heads"]
    if c["op"] == "write":
        freq, mag = _frequencies(c, torch.float64)
        turn = torch.polar(torch.full((), float(mag), dtype=torch.float64, device="cuda"), s["row_pos"].double()[:, None] * freq)
        R, h = c["rot"], c["rot"] // 2
        x = s["qkv"].view(-1, H + 2 * KV, D)
        q = x[:, :H].double()                             # a pair as a complex number, turned by a product
        if c["norm"]:
            q = q / (q.pow(2).sum(-1, keepdim=True) / D + _EPS).sqrt() * s["q_gain"].double()
        re, im = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, h), slice(h, R))
        z = torch.complex(q[..., re].contiguous(), q[..., im].contiguous()) * turn[:, None, :]
        q[..., re], q[..., im] = z.real, z.imag
        # V, block by block; K has none: a value that lies next to the border between two codes, or the largest of a block next to the
        # border between two exponents, takes either side by the last bit of a sum in 32 bits
        out, r = [], 0
        for n, ((length, first, k), (_, lo, count)) in enumerate(zip(_lens(c), _touched(c))):
            codes, e = pool(1, n)
            new = x[r:r + k, H + KV:].double().transpose(0, 1)
            r += k
            a, b = lo // _BLOCK, _pages(lo + count, _BLOCK)
            v = codes[:, a * _BLOCK:b * _BLOCK].clone()
            fresh = torch.zeros(KV, (b - a) * _BLOCK, D, dtype=torch.float64, device="cuda")
            fresh[:, first - lo:first - lo + k] = new
            top = fresh.abs().view(KV, b - a, -1).amax(-1)
            need = torch.ceil(torch.log2(top.clamp(min=2.0 ** -120) / 448)).long().clamp(_LOW, _HIGH)
            need -= ((top <= 448 * _two(need - 1, torch.float64)) & (need > _LOW)).long()      # the logarithm's own rounding
            need += (top > 448 * _two(need, torch.float64)).long()
            at = torch.arange(a * _BLOCK, b * _BLOCK, device="cuda")
            kept = ((at < length) & ((at < first) | (at >= first + k))).view(b - a, _BLOCK)
            now = torch.where(kept.any(1), torch.maximum(need, e[:, a:b]), need)
            v = _e4m3(v * two(e[:, a:b] - now)) * two(now)
            v[:, first - lo:first - lo + k] = (_e4m3(fresh * two(-now)) * two(now))[:, first - lo:first - lo + k]
            out.append(v[:, :count].transpose(0, 1))
        return {"q": q, "k": None, "v": torch.cat(out)}
    out = torch.zeros(s["rows"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((s["rows"], H), -math.inf, dtype=torch.float64, device="cuda")
    r = 0
    for n, (length, first, k) in enumerate(_lens(c)):
        kv = [codes * two(e) for codes, e in (pool(0, n), pool(1, n))]
        pos = torch.arange(first, first + k, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None, :]
        hidden = torch.zeros(k, length, dtype=torch.bool, device="cuda")
        if c["right"] >= 0:
            hidden |= key - pos > c["right"]
        if c["left"] >= 0:
            hidden |= (pos - key > c["left"]) & (key >= c["sinks"])
        for h in range(H):
            kd, vd = (t[h * KV // H, :length] for t in kv)
            a = (s["q"][r:r + k, h].double() @ kd.t()) / math.sqrt(D)
            a[hidden] = -math.inf
            z = torch.logsumexp(a, -1)
            w = torch.exp(a - z[:, None])
            w[torch.isinf(z)] = 0
            out[r:r + k, h], lse[r:r + k, h] = w @ vd, z
        r += k
    return {"out": out, "lse": lse}
