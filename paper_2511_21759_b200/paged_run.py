"""A small server loop over the paged cache: python -m paper_2511_21759_b200.paged_run [--layers N] [--requests N] [--blocks N]

Attention layers with grouped heads over requests of different lengths, decoded block by block as the method does: a refresh of
every request at the start of its block (all rows, keys in both directions), a few steps of the block's rows against the cached
keys, then the next block.  Between them the requests change: a response is found to be shorter and its last pages go back, a
request ends, a new one takes its place and its pages.  Per forward

    layout                                     once: block tables, slots, rows
    QKV projection -> norm_rope_store -> attention -> output projection        per layer

The projections are the library's GEMM; weights and inputs are synthetic (seeded).  Prints what every forward held and took.
"""
from __future__ import annotations

import argparse
import ctypes as C

import torch

from . import binding as B
from . import engine as E
from . import paged


class Layers:
    """Attention layers: per layer packed QKV and output projections, gains of the q and k norms."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, seed: int = 0):
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim = n_layers, n_heads, n_kv_heads, head_dim
        self.d = n_heads * head_dim
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
        w = lambda out, inp: E.pack_weight((normal(out, inp) * inp ** -0.5).to(torch.bfloat16))
        self.qkv_width = (n_heads + 2 * n_kv_heads) * head_dim
        self.wqkv = [w(self.qkv_width, self.d) for _ in range(n_layers)]
        self.wo = [w(self.d, self.d) for _ in range(n_layers)]
        self.q_gain = [1 + 0.2 * normal(head_dim) for _ in range(n_layers)]
        self.k_gain = [1 + 0.2 * normal(head_dim) for _ in range(n_layers)]

    @staticmethod
    def project(x: torch.Tensor, packed: torch.Tensor, width: int) -> torch.Tensor:
        """bf16 rows through a packed weight, bf16 out."""
        rows, d = x.shape
        out = torch.empty(rows, width, dtype=torch.float32, device=x.device)
        scratch = torch.empty(16 * rows * width * 4 + 1024, dtype=torch.uint8, device=x.device)
        st = torch.cuda.current_stream(x.device)
        B.check(B.lib().odb_debug_gemm(x.data_ptr(), packed.data_ptr(), out.data_ptr(), scratch.data_ptr(), scratch.numel(), rows, width, d, 0,
                                       C.c_void_p(st.cuda_stream)), "odb_debug_gemm")
        return out.to(torch.bfloat16)

    def forward(self, cache: paged.PagedCache, batch: paged.Batch, rows: int, h: torch.Tensor, rope: paged.Rope, seen=None, **mask) -> torch.Tensor:
        """One forward of the batch's `rows` rows; h [rows][d] float32 residual stream.  seen(layer, qkv, q, out): a look at
        every layer's tensors."""
        cache.layout(batch)
        if rows == 0:
            return h
        a, b = self.d, self.d + self.n_kv_heads * self.head_dim
        for layer in range(self.n_layers):
            qkv = self.project(h.to(torch.bfloat16), self.wqkv[layer], self.qkv_width)
            q = cache.norm_rope_store(layer, batch, qkv[:, :a], qkv[:, a:b], qkv[:, b:], rope, q_gain=self.q_gain[layer], k_gain=self.k_gain[layer])
            out = cache.attention(layer, batch, q, **mask)
            if seen is not None:
                seen(layer, qkv, q, out)
            h = h + self.project(out.view(rows, self.d), self.wo[layer], self.d).float()
        return h


class Server:
    """Requests with a prompt and a response in blocks, their pages in one pool."""

    def __init__(self, layers: Layers, page_size: int, n_pages: int, longest: int, block: int):
        self.layers, self.block, self.page_size = layers, block, page_size
        self.cache = paged.PagedCache(layers.n_layers, layers.n_heads, layers.n_kv_heads, layers.head_dim, page_size, n_pages)
        self.rope = paged.Rope(layers.head_dim)
        self.width = -(-longest // page_size)
        self.free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((0, self.width), -1, dtype=torch.int32, device="cuda")
        self.length = []          # positions held, per place in the batch
        self.total = []           # prompt + response
        self.start = []           # of the open block

    def add(self, prompt: int, response: int):
        """A request in the first empty place, or in a new one; it holds nothing yet."""
        for i, total in enumerate(self.total):
            if total == 0:
                break
        else:
            i = len(self.total)
            self.table = torch.cat([self.table, torch.full((1, self.width), -1, dtype=torch.int32, device="cuda")])
            self.length.append(0)
            self.total.append(0)
            self.start.append(0)
        self.total[i], self.start[i] = prompt + response, prompt
        return i

    def forward(self, kind: str, seen=None, seed: int = 0):
        """kind "refresh": all rows of all requests; "step": the rows of the open blocks.  Lengths that changed since the last
        forward (responses cut, requests ended or begun) take effect here.  Returns the batch and the rows' output."""
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        first = [0 if kind == "refresh" else s for s in self.start]
        count = [n if kind == "refresh" else max(0, min(self.block, n - s)) for n, s in zip(self.total, self.start)]
        rows = sum(count)
        batch = paged.Batch(self.cache, table=self.table, free_pages=self.free, len_before=i32(self.length), len_after=i32(self.total),
                            first=i32(first), count=i32(count), max_rows=rows, max_new=max(count, default=0))
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        h = torch.randn(rows, self.layers.d, generator=g, device="cuda")
        h = self.layers.forward(self.cache, batch, rows, h, self.rope, None if seen is None else lambda *a: seen(self, batch, first, count, *a))
        self.length = list(self.total)
        status = self.cache.status()
        if status:
            raise B.OdbError(status, "forward")
        return batch, h


def run(layers: Layers, requests: int = 6, blocks: int = 3, block: int = 32, page_size: int = 16, steps: int = 2, seen=None, say=print):
    """The loop of this file's heading; every request has `blocks` blocks of response.  Returns the server."""
    longest = 40 * requests + 64 + blocks * block
    server = Server(layers, page_size, requests * (-(-longest // page_size)), longest, block)
    for i in range(requests):
        server.add(40 * i + 17, blocks * block)
    held = lambda: sum(-(-n // page_size) for n in server.length)
    n = 0
    for b in range(blocks):
        for kind in ["refresh"] + ["step"] * steps:
            batch, h = server.forward(kind, seen, seed=n)
            say(f"block {b} {kind:7s}: {batch.max_rows:5d} rows, {held():4d} of {server.cache.n_pages} pages held, |h| {h.square().mean().sqrt().item():.4f}")
            n += 1
            if kind == "refresh" and b == 0:
                server.total[1] -= block                    # a response found to be shorter: a block of it is gone
        for i in range(len(server.start)):
            server.start[i] += block
        if b == 0:
            server.total[0] = 0                             # a request ends, another takes its place
            server.add(73, blocks * block)
            server.start[0] = 73
    return server


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--blocks", type=int, default=3)
    a = ap.parse_args()
    run(Layers(a.layers, 32, 8, 128), a.requests, a.blocks)


if __name__ == "__main__":
    main()
