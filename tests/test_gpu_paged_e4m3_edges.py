"""The paged cache in 8 bits where its calls meet what earlier ones left behind and numbers at the ends of their ranges.  Bounds are derived
beside each test, before its first run."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from test_gpu_paged import paged
from test_gpu_paged_e4m3 import i32, setup
from test_paged_e4m3_host import kernel


def binding():
    from paper_2511_21759_b200 import binding as B
    return B


def kernel_of(batch, cache):
    """The kernel that an attention of the batch takes (test_paged_e4m3_host.kernel)."""
    room = cache.workspace.numel() > binding().lib().odb_paged_workspace_bytes(cache.cfg)
    return kernel(batch.n_seqs, batch.max_rows, batch.max_new, cache.n_heads // cache.n_kv_heads, cache.n_kv_heads,
                  batch.table.shape[1] * cache.page_size, room=room)


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
