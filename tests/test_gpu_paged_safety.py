"""The paged operators with arguments, maps and objects that are not what they should be: what is refused, what the status word says,
and that the next call is not touched by it."""
import numpy as np
import pytest
import torch

from gpu_common import requires_gpu
from test_gpu_paged import _setup, dev, paged


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
