"""Object layer of the paged K/V cache (odb_paged_* of include/odb.h): owns or borrows the device buffers, checks what a
pointer cannot say (types, devices, shapes, strides) and marshals arguments.  No arithmetic happens in this file.

A forward over requests of different lengths, one layer after the other:

    cache = PagedCache(n_layers, n_heads, n_kv_heads, head_dim, page_size, n_pages)
    batch = Batch(cache, table=..., free_pages=..., len_before=..., len_after=..., first=..., count=..., max_rows=...)
    cache.layout(batch)                                       # tables, slots, row maps: once a forward
    for layer in range(n_layers):
        q = cache.norm_rope_store(layer, batch, q, k, v, rope, q_gain=..., k_gain=...)
        o = cache.attention(layer, batch, q, right=0)

Every call is enqueued on the current stream of the cache's device and returns at once; status() waits and says what the
device found.  A cache is used by one thread and on one stream at a time: a call on another stream than the one before waits for
that one, and so it does for the stream that its Batch was made or used on; the memory of these objects and of a Rope is not given back
before the streams that used it are through.  In a graph's capture nothing is waited for: what the graph uses is to be kept, and its
replays ordered, by its owner.  Tensors that are passed to a call follow torch's own rules for streams.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from . import binding as B

_BF16, _F32 = torch.bfloat16, torch.float32
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
_ROWS = struct.Struct("=QqQqQqQqQQ")          # odb_paged_rows, filled in one go
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class _OnStream:
    """What is known of the memory that an object holds: the stream it was last used on."""

    def _made(self, index: int, tensors):
        self._raw, self._memory = _raw_stream(index), tensors

    def _follow(self, st, raw: int):
        """To stream st: the other one's work comes first, and the memory stays until st's is done too."""
        st.wait_stream(torch.cuda.ExternalStream(self._raw, device=st.device))
        for t in self._memory:
            if t is not None:
                t.record_stream(st)
        self._raw = raw


class Rope(_OnStream):
    """Rotation of the first rot_dim values of a head: pairs (i, i + rot_dim / 2), or (2i, 2i + 1) where interleaved.
    scaling: "none", "linear", "ntk" or "yarn" with a factor (odb_rope_frequencies)."""

    def __init__(self, rot_dim: int, theta: float = 500000.0, *, interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
                 original_len: float = 8192, beta_slow: float = 1.0, beta_fast: float = 32.0, device="cuda"):
        if scaling not in SCALINGS:
            raise ValueError(f"scaling {scaling!r}: one of {', '.join(SCALINGS)}")
        host = (C.c_uint64 * max(1, rot_dim // 2))()
        mag = C.c_float()
        B.check(B.lib().odb_rope_frequencies(rot_dim, theta, SCALINGS[scaling], factor, original_len, beta_slow, beta_fast, host,
                                             C.byref(mag)), "odb_rope_frequencies")
        self.rot_dim, self.interleaved, self.magnitude = rot_dim, interleaved, mag.value
        # fractions of a turn per position, 64-bit patterns
        self.turns = torch.tensor([C.c_int64(v).value for v in host], dtype=torch.int64, device=device)
        self.index = self.turns.get_device()
        if self.turns.is_cuda:
            self._made(self.index, (self.turns,))
        self._c = B.odb_rope(self.turns.data_ptr(), rot_dim, 1 if interleaved else 0, mag.value)
        self._ref = C.byref(self._c)

    def _follow(self, st, raw: int):
        """The numbers were there when the constructor returned and are read only: caches on several streams wait for none."""
        self.turns.record_stream(st)
        self._raw = raw


class Batch(_OnStream):
    """The device arrays of one forward (odb_paged_batch); arrays that a call needs and that are not given are made here (-1 until
    layout fills them: nothing is stored by such maps, and an attention is refused by the status word), those that are given are used
    as they are: int32, contiguous, on the cache's device.  It serves every cache of the same device, pages and heads, and every
    forward of the same requests and rows: its arrays may be written in place (one copy of all lengths takes 3 us on the host, a new
    Batch 22, 11 with all arrays given).  max_rows: rows of the forward (known where row arrays are given); max_new: rows of the longest
    request, a hint that picks the attention's kernel: worth giving where the requests' rows are known on the host (without it up to a
    fifth slower, where several requests of 128 to 1024 rows x heads of a group are alike)."""

    _INPUTS = ("len_before", "len_after", "first", "count", "table", "free_pages", "row_start", "row_seq", "row_pos", "row_slot")

    def __init__(self, cache: "PagedCache", *, table=None, free_pages=None, len_before=None, len_after=None, first=None, count=None,
                 row_start=None, row_seq=None, row_pos=None, row_slot=None, max_rows: Optional[int] = None, max_new: Optional[int] = None):
        given = dict(len_before=len_before, len_after=len_after, first=first, count=count, table=table, free_pages=free_pages,
                     row_start=row_start, row_seq=row_seq, row_pos=row_pos, row_slot=row_slot)
        for name, t in given.items():
            if t is not None and (not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.device != cache.device or not t.is_contiguous()):
                raise ValueError(f"{name}: a contiguous int32 tensor on {cache.device} is wanted")
        seqs = {name: given[name].shape for name in ("len_before", "len_after", "first", "count") if given[name] is not None}
        if table is not None:
            if table.dim() != 2 or (table.shape[0] and table.shape[1] < 1):
                raise ValueError("table: [requests][pages of the longest request]")
            seqs["table"] = table.shape[:1]
        if row_start is not None:
            seqs["row_start"] = torch.Size([row_start.numel() - 1]) if row_start.dim() == 1 else row_start.shape
        if len(set(seqs.values())) > 1 or any(len(v) != 1 for v in seqs.values()):
            raise ValueError(f"one entry a request is wanted: {({k: tuple(v) for k, v in seqs.items()})}")
        n_seqs = next(iter(seqs.values()))[0] if seqs else 0
        rows = {given[n].numel() for n in ("row_seq", "row_pos", "row_slot") if given[n] is not None}
        if len(rows | ({max_rows} - {None})) > 1:
            raise ValueError("row_seq, row_pos and row_slot have max_rows entries")
        if free_pages is not None and free_pages.numel() < cache.n_pages:
            raise ValueError(f"free_pages: {cache.n_pages} entries are wanted")
        self.n_seqs = n_seqs
        self.max_rows = rows.pop() if rows else (max_rows or 0)
        self.max_new = max_new or 0
        maps = [name for name in ("row_seq", "row_pos", "row_slot") if given[name] is None]
        sizes = [self.max_rows] * len(maps)
        if row_start is None and seqs:
            maps.append("row_start")
            sizes.append(n_seqs + 1)
        if maps:
            given.update(zip(maps, torch.full((sum(sizes),), -1, dtype=torch.int32, device=cache.device).split(sizes)))
        self._made(cache._index, tuple(given.values()))
        for name, t in given.items():
            setattr(self, name, t)
        self.cache = cache
        self._c = B.odb_paged_batch(n_seqs, self.max_rows, self.max_new, table.shape[1] if table is not None else 1,
                                    *[None if given[n] is None else given[n].data_ptr() for n in self._INPUTS])
        self._ref = C.byref(self._c)
        # shapes of its rows, heads apart and together
        n, d = self.max_rows, cache.head_dim
        self._q = (torch.Size((n, cache.n_heads, d)), torch.Size((n, cache.n_heads * d)))
        self._kv = (torch.Size((n, cache.n_kv_heads, d)), torch.Size((n, cache.n_kv_heads * d)))
        self._lse = torch.Size((n, cache.n_heads))


class PagedCache(_OnStream):
    """A pool of K/V pages (bf16 [n_layers][2][n_pages][n_kv_heads][page_size][head_dim]) and the calls over it.  kv: a
    tensor of that shape to use; otherwise one is allocated (not cleared: what no request has written reaches no result)."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, *, kv=None, device=None):
        lib = B.lib()
        self.cfg = B.odb_paged_config(n_layers, n_heads, n_kv_heads, head_dim, page_size, n_pages)
        self.n_layers, self.n_heads, self.n_kv_heads, self.head_dim, self.page_size, self.n_pages = \
            n_layers, n_heads, n_kv_heads, head_dim, page_size, n_pages
        self.handle = C.c_void_p()
        if not lib.odb_paged_kv_bytes(C.byref(self.cfg)):
            raise B.OdbError(B.ODB_ERR_SHAPE, "odb_paged_create")
        shape = (n_layers, 2, n_pages, n_kv_heads, page_size, head_dim)
        if kv is None:
            kv = torch.empty(shape, dtype=torch.bfloat16, device=device or "cuda")
        elif tuple(kv.shape) != shape or kv.dtype != torch.bfloat16 or not kv.is_cuda or not kv.is_contiguous():
            raise ValueError(f"kv: a contiguous bfloat16 CUDA tensor of shape {shape} is wanted")
        self.kv = kv
        self.device = kv.device
        self.workspace = torch.empty(lib.odb_paged_workspace_bytes(C.byref(self.cfg)), dtype=torch.uint8, device=self.device)
        self._index = self.device.index
        self._made(self._index, (self.workspace, kv))
        with torch.cuda.device(self.device):
            B.check(lib.odb_paged_create(C.byref(self.cfg), kv.data_ptr(), kv.numel() * 2, self.workspace.data_ptr(),
                                         self.workspace.numel(), C.c_void_p(self._raw), C.byref(self.handle)), "odb_paged_create")
        self._shape = (self.device, n_heads, n_kv_heads, head_dim, page_size, n_pages)     # what a batch depends on
        self._gain_shape = torch.Size((head_dim,))
        self._new, self._width = kv.new_empty, n_heads * head_dim       # outputs: bf16 on the cache's device (1.4 us; torch.empty 3.1)
        self._rows_c = B.odb_paged_rows()
        self._rows_ref = C.byref(self._rows_c)
        self._layout, self._store, self._attention = lib.odb_paged_layout, lib.odb_paged_norm_rope_store, lib.odb_paged_attention

    def close(self):
        if self.handle:
            B.lib().odb_paged_destroy(self.handle)
            self.handle = C.c_void_p()

    def _there(self, call, *args, **kwargs):
        """The call with the cache's device current: the library takes no other."""
        with torch.cuda.device(self._index):
            return call(*args, **kwargs)

    def _current(self, a, b) -> int:
        """The current stream's handle; it follows the streams that the cache and the objects a and b used with it come from."""
        raw = _raw_stream(self._index)
        if (raw != self._raw or raw != a._raw or raw != b._raw) and not torch.cuda.is_current_stream_capturing():
            st = torch.cuda.current_stream(self.device)
            for x in (self, a, b):
                if raw != x._raw:
                    x._follow(st, raw)
        return raw

    def _other(self, batch: Batch):
        """A batch that was made for another cache: its tensors were checked against that one's pages and heads."""
        if batch.cache._shape != self._shape:
            raise ValueError("the batch was made for a cache of other pages, heads or device")

    def _wrong(self, t, what: str, heads: int, rows: int):
        if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.device != self.device:
            return ValueError(f"{what}: a bfloat16 tensor on {self.device} is wanted")
        return ValueError(f"{what}: [{rows}][{heads}][{self.head_dim}] with a row's values together is wanted, got {tuple(t.shape)} by {t.stride()}")

    # The checks of a tensor are most of what a small call costs on the host: each question is asked once, of the tensor's own methods.
    def _rows(self, t, what: str, heads: int, shapes):
        """(pointer, elements from row to row) of [rows][heads][head_dim], the last two dims together or apart; shapes: the two."""
        if t.dtype is _BF16 and t.get_device() == self._index:
            shape = t.shape
            if shape == shapes[0]:
                stride, head, last = t.stride()
                if last == 1 and (heads == 1 or head == self.head_dim):
                    return t.data_ptr(), stride if shape[0] > 1 else shapes[1][1]     # of one row: any number
            elif shape == shapes[1]:
                stride, last = t.stride()
                if last == 1:
                    return t.data_ptr(), stride if shape[0] > 1 else shapes[1][1]
        raise self._wrong(t, what, heads, shapes[0][0])

    def _gain(self, t, what: str):
        if t is None:
            return 0
        if t.dtype is _F32 and t.get_device() == self._index and t.shape == self._gain_shape and t.is_contiguous():
            return t.data_ptr()
        raise ValueError(f"{what}: a contiguous float32 tensor of {self.head_dim} values on {self.device} is wanted")

    def layout(self, batch: Batch):
        """Block tables, free list and row maps of the forward (odb_paged_layout); the batch's arrays are updated."""
        if batch.cache is not self:
            self._other(batch)
        if _current_device() != self._index:
            return self._there(self.layout, batch)
        status = self._layout(self.handle, batch._ref, self._current(batch, batch))
        if status:
            raise B.OdbError(status, "odb_paged_layout")

    def norm_rope_store(self, layer: int, batch: Batch, q, k, v, rope: Rope, *, q_gain=None, k_gain=None, eps: float = 1e-6, q_out=None):
        """Norm of every q and k head (where a gain is given), rotation by row_pos, K and V into row_slot
        (odb_paged_norm_rope_store).  q, k, v: [max_rows][heads][head_dim] or [max_rows][heads * head_dim], slices of one
        projection's output as they are.  Returns q_out (a new tensor where none is given; q itself may be given, other rows that overlap
        q, k or v are refused)."""
        if _current_device() != self._index:
            return self._there(self.norm_rope_store, layer, batch, q, k, v, rope, q_gain=q_gain, k_gain=k_gain, eps=eps, q_out=q_out)
        if batch.cache is not self:
            self._other(batch)
        if rope.index != self._index:
            raise ValueError(f"rope: on {self.device} it is wanted")
        qp, qs = self._rows(q, "q", self.n_heads, batch._q)
        kp, ks = self._rows(k, "k", self.n_kv_heads, batch._kv)
        vp, vs = self._rows(v, "v", self.n_kv_heads, batch._kv)
        if q_out is None:
            q_out = self._new(batch.max_rows, self.n_heads, self.head_dim)
            op, os_ = q_out.data_ptr(), self._width
        else:
            op, os_ = (qp, qs) if q_out is q else self._rows(q_out, "q_out", self.n_heads, batch._q)
        _ROWS.pack_into(self._rows_c, 0, qp, qs, kp, ks, vp, vs, op, os_, self._gain(q_gain, "q_gain"), self._gain(k_gain, "k_gain"))
        status = self._store(self.handle, layer, batch._ref, self._rows_ref, rope._ref, eps, self._current(batch, rope))
        if status:
            raise B.OdbError(status, "odb_paged_norm_rope_store")
        return q_out

    def attention(self, layer: int, batch: Batch, q, *, left: int = -1, right: int = -1, sinks: int = 0, scale: float = 0.0, out=None, lse=None):
        """Attention of the batch's rows over their requests' pages (odb_paged_attention): a row at position p sees the
        keys j < len_after with j <= p + right and (j >= p - left or j < sinks); -1: no limit; causal: right=0.
        scale 0: 1 / sqrt(head_dim).  lse: float32 [max_rows][n_heads] to be filled.  Returns out (a new tensor where none
        is given; one whose rows overlap q's is refused)."""
        if _current_device() != self._index:
            return self._there(self.attention, layer, batch, q, left=left, right=right, sinks=sinks, scale=scale, out=out, lse=lse)
        if batch.cache is not self:
            self._other(batch)
        qp, qs = self._rows(q, "q", self.n_heads, batch._q)
        if out is None:
            out = self._new(batch.max_rows, self.n_heads, self.head_dim)
            op, os_ = out.data_ptr(), self._width
        else:
            op, os_ = self._rows(out, "out", self.n_heads, batch._q)
        lp = None
        if lse is not None:
            if lse.dtype is not _F32 or lse.get_device() != self._index or lse.shape != batch._lse or not lse.is_contiguous():
                raise ValueError(f"lse: a contiguous float32 tensor {list(batch._lse)} on {self.device} is wanted")
            lp = lse.data_ptr()
        status = self._attention(self.handle, layer, batch._ref, qp, qs, op, os_, lp, scale, left, right, sinks, self._current(batch, batch))
        if status:
            raise B.OdbError(status, "odb_paged_attention")
        return out

    def status(self) -> int:
        """Waits for the current stream; ODB_OK or what the device has found since the last call (read and cleared)."""
        if _current_device() != self._index:
            return self._there(self.status)
        return B.lib().odb_paged_status(self.handle, self._current(self, self))
