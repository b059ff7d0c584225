"""The paged-cache operators, as a program that serves a language model meets them.

Requests of different lengths share one pool of K/V pages.  A forward goes through three operators:

  layout     block tables and slot maps from request lengths: every request's table grows or shrinks from
             ceil(len_before / page) to ceil(len_after / page) pages, pages given back are the first to be handed
             out again, and every row of the forward gets its request, position and slot
  norm_rope  queries and keys of every head normalised, turned by their position, keys and values stored into
             their slots
  attention  rows of each request against its pages, with grouped heads, a window and first tokens that stay
             visible

`run` computes one pass of one operator, with the package's calls where `own` is true and with elementary torch
operations in 32 bits where it is not.  The pool is bf16 [layers][2][pages][kv heads][page][head dim].

The definitions.  layout: free list F of n = n_pages - sum(held) entries; G pages given back (requests in order, then
pages in order) are appended, T pages are taken from the end (requests in order, then pages in order), the first
n + G - T entries remain.  Row r of request s is position first[s] + i; its slot is table[s][pos // page] * page +
pos % page.  Rows behind the last one have request, position and slot -1.  norm_rope: y = x / sqrt(mean(x^2) + eps) *
gain, then the pairs (i, i + R/2) (half) or (2i, 2i+1) (interleaved) of the first R dims turned by the angle
pos * f_i, cosine and sine multiplied by the method's magnitude; one rounding.  attention: key j of a request with
`len` keys is visible to position p when j < len, j <= p + right and (j >= p - left or j < sinks); softmax of
q k / sqrt(head dim) over the visible keys; rows that see no key give zeros and a log-sum-exp of -infinity.
"""
import math
import random

import torch

own = False

_UNLIMITED = 1 << 30


# ---- the cases ----------------------------------------------------------------------------------------------------

def _layout(name, seqs, page, lo, hi, step, mix):
    return _named(name, dict(op="layout", seqs=seqs, page=page, lo=lo, hi=hi, step=step, mix=mix))


def _norm_rope(name, rows, heads, kv_heads, dim, page, rot, interleaved, norm, scaling, factor, far):
    return _named(name, dict(op="norm_rope", rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, page=page, rot=rot,
                             interleaved=interleaved, norm=norm, scaling=scaling, factor=factor, far=far))


def _attention(name, seqs, lo, hi, new, heads, kv_heads, dim, page, left=-1, right=-1, sinks=0, middle=False):
    return _named(name, dict(op="attention", seqs=seqs, lo=lo, hi=hi, new=new, heads=heads, kv_heads=kv_heads, dim=dim,
                             page=page, left=left, right=right, sinks=sinks, middle=middle))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one block step of a small batch: nearly every request keeps its pages, launch and call are the whole cost
        _layout("layout_step_16", 16, 64, 300, 2000, 32, False),
        # a busy server's iteration: new requests, finished ones, shortened ones and steps, long prompts among them
        _layout("layout_mixed_1000", 1000, 16, 1, 900, 32, True),
        # one token for each of eight requests (grouped heads, whole-head rotation)
        _norm_rope("norm_rope_8_tokens", 8, 32, 8, 128, 64, 128, False, True, "none", 1.0, 4096),
        # blocks of 32 rows of sixteen requests, half of each head turned in interleaved pairs, context scaled by parts
        _norm_rope("norm_rope_512_part", 512, 32, 32, 128, 16, 64, True, True, "yarn", 8.0, 60000),
        # the refresh of a batch: 25568 rows of 32 + 2 x 8 heads
        _norm_rope("norm_rope_25568", 25568, 32, 8, 128, 64, 128, False, True, "none", 1.0, 2048),
        # one token of one short request: latency
        _attention("token_577", 1, 577, 577, 1, 32, 8, 128, 16),
        # one token each of a ragged batch
        _attention("token_batch_48", 48, 1, 8192, 1, 32, 8, 128, 64, right=0),
        # one token of two very long requests: the work has to be split along the keys
        _attention("token_long", 2, 100000, 131072, 1, 32, 8, 128, 64, right=0),
        # a window of 4096 with four first tokens kept, head dim 64, sixteen long requests
        _attention("token_window", 16, 3000, 32768, 1, 16, 4, 64, 32, left=4095, right=0, sinks=4),
        # block steps in the middle of the sequences: 32 rows against all cached keys, in both directions
        _attention("block_16x32", 16, 700, 4096, 32, 32, 8, 128, 64, middle=True),
        # the refresh of a ragged batch: every row against every row of its request, one K/V head per query head
        _attention("refresh_4", 4, 900, 1536, 0, 32, 32, 128, 64),
        # a causal prompt of 4096 tokens
        _attention("prompt_4096", 1, 4096, 4096, 0, 32, 8, 128, 64, right=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("layout", "norm_rope", "norm_rope", "token", "token", "window", "block", "rows"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "layout":
        seqs = _log(rng, 1, 1000)
        return _layout(None, seqs, page, 1, _log(rng, 40, min(60000, 900000 // seqs)), rng.choice((1, 16, 32, 64)), rng.random() < 0.6)
    dim = rng.choice((64, 128, 128))
    kv = rng.choice((1, 2, 4, 8))
    group = rng.choice((1, 2, 3, 4, 5, 8))
    if kind == "norm_rope":
        rot = dim if rng.random() < 0.6 else rng.choice([r for r in (16, 24, 32, 48, 64, 96) if r < dim])
        scaling = rng.choice(("none", "none", "linear", "ntk", "yarn"))
        rows = _log(rng, 1, 25568 * 48 * 128 // ((group + 2) * kv * dim) if (group + 2) * kv * dim > 48 * 128 else 25568)
        return _norm_rope(None, rows, kv * group, kv, dim, page, rot, rng.random() < 0.4, rng.random() < 0.75, scaling,
                          1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 32.0)), _log(rng, 1000, 130000))
    if kind == "token":
        seqs = _log(rng, 1, 128)
        hi = _log(rng, 20, min(131072, 400000 // seqs))
        return _attention(None, seqs, rng.choice((1, max(1, hi // 2), hi)), hi, 1, kv * group, kv, dim, page, right=rng.choice((-1, 0)))
    if kind == "window":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 50, min(65536, 400000 // seqs))
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

def _requests(c):
    """(len_before, len_after, first, count) of every request of a layout case."""
    rng = random.Random("%(seqs)d %(page)d %(lo)d %(hi)d %(step)d" % c)
    out = []
    for s in range(c["seqs"]):
        n = rng.randint(c["lo"], c["hi"])
        u = rng.random() if c["mix"] else 1.0
        if u < 0.10:                                    # a new request: its prompt comes in as a whole
            out.append((0, n, 0, n))
        elif u < 0.20:                                  # a finished one gives everything back
            out.append((n, 0, 0, 0))
        elif u < 0.25:                                  # a response found to be shorter, refreshed
            m = max(1, n - rng.randint(1, max(1, n // 2)))
            out.append((n, m, 0, m))
        elif u < 0.30:                                  # a request that waits
            out.append((n, n, 0, 0))
        else:                                           # a step: the rows behind, or the open block's again
            k = min(c["step"], c["hi"])
            out.append((n, n + k, n, k) if rng.random() < 0.4 else (n, n, max(0, n - k), min(n, k)))
    return out


def _lens(c):
    """(keys, first position, rows) of every request of an attention case."""
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
    if c["op"] == "layout":
        req = _requests(c)
        rows = sum(r[3] for r in req)
        moved = sum(abs(_pages(r[1], c["page"]) - _pages(r[0], c["page"])) for r in req)
        return {"bytes": 4 * (4 * len(req) + len(req) + 1 + 3 * rows + 2 * moved), "flops": 0}
    if c["op"] == "norm_rope":
        values = c["rows"] * (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": 4 * values + 8 * c["rows"], "flops": 10 * values}
    spans = [(k,) + _span(c, n, f, k) for n, f, k in _lens(c)]
    rows = sum(s[0] for s in spans)
    return {"bytes": 4 * rows * c["heads"] * c["dim"] + 4 * rows * c["heads"] + 4 * c["kv_heads"] * c["dim"] * sum(s[1] for s in spans),
            "flops": 4 * c["heads"] * c["dim"] * sum(s[2] for s in spans)}


# ---- inputs -------------------------------------------------------------------------------------------------------

_EPS, _THETA, _ORIGINAL = 1e-6, 500000.0, 8192


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    s = {"case": c}
    P = c["page"]
    if c["op"] == "layout":
        req = _requests(c)
        held = [_pages(r[0], P) for r in req]
        need = [_pages(r[1], P) for r in req]
        n_pages = max(sum(held), sum(need)) + 8
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        width = max(max(held), max(need))
        table = torch.full((len(req), width), -1, dtype=torch.int32, device="cuda")
        h = ints(held).long()
        table[torch.arange(width, device="cuda")[None, :] < h[:, None]] = order[: sum(held)]
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[: n_pages - sum(held)] = order[sum(held):]
        s.update(table=table, free=free, n_pages=n_pages, rows=sum(r[3] for r in req) + 5,
                 **{k: ints([r[i] for r in req]) for i, k in enumerate(("len_before", "len_after", "first", "count"))})
        s.update(row_start=torch.empty(len(req) + 1, dtype=torch.int32, device="cuda"),
                 **{k: torch.empty(s["rows"], dtype=torch.int32, device="cuda") for k in ("row_seq", "row_pos", "row_slot")})
        return s
    H, KV, D = c["heads"], c["kv_heads"], c["dim"]
    if c["op"] == "norm_rope":
        n = c["rows"]
        n_pages = _pages(n, P) + 3
        qkv = normal(n, (H + 2 * KV) * D) * 1.5           # one projection's output, its parts side by side
        s.update(n_pages=n_pages, qkv=qkv, pool=normal(1, 2, n_pages, KV, P, D),
                 pos=torch.randint(0, c["far"], (n,), generator=g, device="cuda", dtype=torch.int32),
                 slot=torch.randperm(n_pages * P, generator=g, device="cuda")[:n].to(torch.int32),
                 q_out=torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"),
                 q_gain=1 + 0.2 * torch.randn(D, generator=g, device="cuda"), k_gain=1 + 0.2 * torch.randn(D, generator=g, device="cuda"))
        return s
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
    s.update(n_pages=n_pages, table=table, lens=ints([n for n, _, _ in lens]), first=ints([f for _, f, _ in lens]),
             row_start=ints(starts), max_new=max(counts), max_len=max(n for n, _, _ in lens), rows=rows,
             pool=torch.empty(1, 2, n_pages, KV, P, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g),
             q=normal(rows, H, D) * 1.5, out=torch.empty(rows, H, D, dtype=torch.bfloat16, device="cuda"),
             lse=torch.empty(rows, H, dtype=torch.float32, device="cuda"))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"layout": _own_layout, "norm_rope": _own_norm_rope, "attention": _own_attention}[op](s)
    return {"layout": _plain_layout, "norm_rope": _plain_norm_rope, "attention": _plain_attention}[op](s)


def _handles(s):
    """The cache and batch objects that a program keeps next to its buffers."""
    if "batch" in s:
        return s["cache"], s["batch"]
    from paper_2511_21759_b200 import paged
    c = s["case"]
    if c["op"] == "layout":
        cache = paged.PagedCache(n_layers=1, n_heads=1, n_kv_heads=1, head_dim=64, page_size=c["page"], n_pages=s["n_pages"])
        batch = paged.Batch(cache, table=s["table"], free_pages=s["free"], len_before=s["len_before"], len_after=s["len_after"],
                            first=s["first"], count=s["count"], row_start=s["row_start"], row_seq=s["row_seq"],
                            row_pos=s["row_pos"], row_slot=s["row_slot"])
    else:
        cache = paged.PagedCache(n_layers=1, n_heads=c["heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"],
                                 page_size=c["page"], n_pages=s["n_pages"], kv=s["pool"])
        if c["op"] == "norm_rope":
            batch = paged.Batch(cache, row_pos=s["pos"], row_slot=s["slot"])
            s["rope"] = paged.Rope(c["rot"], theta=_THETA, interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"],
                                   original_len=_ORIGINAL)
        else:
            batch = paged.Batch(cache, table=s["table"], len_after=s["lens"], first=s["first"], row_start=s["row_start"],
                                max_rows=s["rows"], max_new=s["max_new"])
    s["cache"], s["batch"] = cache, batch
    return cache, batch


def _own_layout(s):
    cache, batch = _handles(s)
    cache.layout(batch)
    return {k: s[k] for k in ("table", "free", "row_start", "row_seq", "row_pos", "row_slot")}


def _own_norm_rope(s):
    cache, batch = _handles(s)
    c = s["case"]
    a, b = c["heads"] * c["dim"], (c["heads"] + c["kv_heads"]) * c["dim"]
    qkv = s["qkv"]
    cache.norm_rope_store(0, batch, qkv[:, :a], qkv[:, a:b], qkv[:, b:], s["rope"],
                          q_gain=s["q_gain"] if c["norm"] else None, k_gain=s["k_gain"] if c["norm"] else None, eps=_EPS, q_out=s["q_out"])
    return {"q": s["q_out"], "pool": s["pool"]}


def _own_attention(s):
    cache, batch = _handles(s)
    c = s["case"]
    cache.attention(0, batch, s["q"], left=c["left"], right=c["right"], sinks=c["sinks"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_layout(s):
    P, dev = s["case"]["page"], s["table"].device
    held, need = (s["len_before"].long() + P - 1) // P, (s["len_after"].long() + P - 1) // P
    table, free, n_pages = s["table"], s["free"], s["n_pages"]
    col = torch.arange(table.shape[1], device=dev)[None, :]
    n = n_pages - int(held.sum())
    given = table[(col >= need[:, None]) & (col < held[:, None])]
    wanted = (col >= held[:, None]) & (col < need[:, None])
    pages = torch.cat([free[:n], given])
    take = int(wanted.sum())
    left = pages.numel() - take
    table = table.masked_scatter(wanted, pages[left:].flip(0))
    free = torch.cat([pages[:left][:n_pages], free[left:]]) if left > n else free.clone()
    count = s["count"].long()
    start = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), count.cumsum(0)])
    rows = int(start[-1])
    pad = lambda v: torch.cat([v, torch.full((s["rows"] - rows,), -1, dtype=v.dtype, device=dev)]).to(torch.int32)
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=dev), count)
    pos = s["first"].long()[seq] + torch.arange(rows, device=dev) - start[seq]
    slot = table[seq, pos // P].long() * P + pos % P
    return {"table": table, "free": free, "row_start": start.to(torch.int32), "row_seq": pad(seq), "row_pos": pad(pos), "row_slot": pad(slot)}


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


def _norm_turn(x, gain, pos, freq, mag, c):
    """x [rows][heads][dim] in 32 bits."""
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * gain
    R = c["rot"]
    angle = pos[:, None].float() * freq[None, :]
    cos, sin = torch.cos(angle)[:, None, :] * mag, torch.sin(angle)[:, None, :] * mag
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., : R // 2], x[..., R // 2:R])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., R:]], -1).to(torch.bfloat16)


def _plain_norm_rope(s):
    c = s["case"]
    H, KV, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    x = s["qkv"].float().view(-1, H + 2 * KV, D)
    freq, mag = _frequencies(c, torch.float32)
    q = _norm_turn(x[:, :H], s["q_gain"] if c["norm"] else None, s["pos"], freq, mag, c)
    k = _norm_turn(x[:, H:H + KV], s["k_gain"] if c["norm"] else None, s["pos"], freq, mag, c)
    page, off = s["slot"].long() // P, s["slot"].long() % P
    s["pool"][0, 0, page, :, off] = k
    s["pool"][0, 1, page, :, off] = x[:, H + KV:].to(torch.bfloat16)
    return {"q": q, "pool": s["pool"]}


def _plain_attention(s):
    c = s["case"]
    H, KV, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    B, G, dev = c["seqs"], c["heads"] // c["kv_heads"], s["q"].device
    L = s["table"].shape[1] * P
    keys = lambda i: s["pool"][0, i][s["table"].clamp(min=0).long()].float().permute(0, 2, 1, 3, 4).reshape(B, KV, L, D)
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

def exact(c, seed):
    if c["op"] == "layout":
        return None                                       # whole numbers: the plain form's own
    s = prepare(c, seed)
    H, KV, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    if c["op"] == "norm_rope":
        freq, mag = _frequencies(c, torch.float64)
        turn = torch.polar(torch.full((), float(mag), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * freq)
        R, h = c["rot"], c["rot"] // 2

        def one(x, gain):                                 # a pair as a complex number, turned by a product
            x = x.double()
            if c["norm"]:
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + _EPS).sqrt() * gain.double()
            y = x.clone()
            re, im = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, h), slice(h, R))
            z = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * turn[:, None, :]
            y[..., re], y[..., im] = z.real, z.imag
            return y

        x = s["qkv"].view(-1, H + 2 * KV, D)
        pool = s["pool"].double()
        flat = pool.permute(0, 1, 2, 4, 3, 5).reshape(2, -1, KV, D)
        flat[0, s["slot"].long()] = one(x[:, H:H + KV], s["k_gain"])
        flat[1, s["slot"].long()] = x[:, H + KV:].double()
        pool = flat.view(1, 2, s["n_pages"], P, KV, D).permute(0, 1, 2, 4, 3, 5).contiguous()
        return {"q": one(x[:, :H], s["q_gain"]), "pool": pool}
    out = torch.zeros(s["rows"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((s["rows"], H), -math.inf, dtype=torch.float64, device="cuda")
    r = 0
    for n, (length, first, k) in enumerate(_lens(c)):
        kv = s["pool"][0][:, s["table"][n, :_pages(length, P)].long()]        # [2][pages][KV][P][D]
        kv = kv.permute(0, 2, 1, 3, 4).reshape(2, KV, -1, D)[:, :, :length]
        pos = torch.arange(first, first + k, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None, :]
        hidden = torch.zeros(k, length, dtype=torch.bool, device="cuda")
        if c["right"] >= 0:
            hidden |= key - pos > c["right"]
        if c["left"] >= 0:
            hidden |= (pos - key > c["left"]) & (key >= c["sinks"])
        for h in range(H):
            kd, vd = kv[0, h * KV // H].double(), kv[1, h * KV // H].double()
            a = (s["q"][r:r + k, h].double() @ kd.t()) / math.sqrt(D)
            a[hidden] = -math.inf
            z = torch.logsumexp(a, -1)
            w = torch.exp(a - z[:, None])
            w[torch.isinf(z)] = 0
            out[r:r + k, h], lse[r:r + k, h] = w @ vd, z
        r += k
    return {"out": out, "lse": lse}
