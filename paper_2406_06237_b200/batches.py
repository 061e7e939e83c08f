"""The operators of a batch of requests: their block tables (PageTables), an adapter of each beside a shared projection
(Adapters), and a cache in 8 bits with the attention that reads it (BlockCache).

What a batch is, on the device throughout (int32): lengths [n], the requests' tokens; starts [n + 1], request s's new tokens,
the last of its tokens, have rows starts[s] to starts[s + 1] of queries, keys and so on, later rows being padding; tables
[n, pages], the pages that hold the tokens.  The host looks at none of them, so a captured call serves batches of other
lengths.  Handles, streams and errors are those of the operators around a product (operators.py)."""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B
from .operators import _ELEMENT, _Handle, _cuda_device, _need, _on_device, _rows

_INT = torch.int32


def _vector_of(t: torch.Tensor, n: int, device, what: str, dtype=_INT) -> None:
    _need(t.dtype is dtype and t.shape == (n,) and t.is_contiguous(), f"{what} must be {str(dtype)[6:]} [{n}]")
    _on_device(t, device, what)


def _counts(*sizes: int) -> None:
    """The library counts in 32 bits."""
    _need(max(sizes) < 2 ** 31, "sizes must be under 2^31")


def _check_tables(tables: torch.Tensor, device) -> tuple[int, int, int]:
    """(sequences, pages, row stride)"""
    _need(tables.dtype is _INT and tables.dim() == 2 and (tables.shape[1] <= 1 or tables.stride(1) == 1), "tables must be int32 [sequences, pages]")
    n, pages = tables.shape
    _counts(n, pages)
    _need(n <= 1 or tables.stride(0) >= pages, "the rows of tables overlap")
    _on_device(tables, device, "tables")
    return n, pages, tables.stride(0)


def _steps(t: torch.Tensor) -> tuple[int, int]:
    """Strides of rows and heads, 0 for the one row or head that has no next one."""
    return t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0


def _overlaps(t: torch.Tensor) -> bool:
    """Whether two heads of [rows, heads, dim], the values of a head contiguous, share an element."""
    (rows, heads, dim), (row, head) = t.shape, _steps(t)
    if not t.numel():
        return False
    if heads == 1 or head >= dim:                          # the usual forms: heads within rows, or rows within heads
        if rows == 1 or row >= head * (heads - 1) + dim:
            return False
    if rows > 1 and row < dim:
        return True
    if heads > 1 and head >= row * (rows - 1) + dim:
        return False
    for h in range(heads):                                 # heads h apart: the two numbers of rows that bring them nearest
        for r in ((-(h * head // row), -(h * head // row) - 1) if rows > 1 else (0,)):
            if (r or h) and -rows < r and abs(r * row + h * head) < dim:
                return True
    return False


class Batch(NamedTuple):
    """What PageTables makes: starts, ends (sums of the lengths: what PagedCache.read takes as starts), lengths,
    slots (for PagedCache.write), positions, and the number of entries of the free list that are taken."""
    starts: torch.Tensor
    lengths: torch.Tensor
    ends: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor
    taken: torch.Tensor


class PageTables(_Handle):
    """Block tables, slot maps and row ranges of a batch, from its requests' lengths (see ans_pages_desc in the header)."""

    def __init__(self, page_size: int, device="cuda"):
        super().__init__(device)
        _need(0 < page_size <= 1 << 20, "page_size must be 1 to 2^20")
        self.page_size = page_size
        self._form = self._new_form()
        self._desc = d = B.ans_pages_desc()
        d.page_size = page_size
        self._hold()

    def buffers(self, requests: int, rows: int) -> Batch:
        """Fresh buffers for a batch of so many requests and rows (those of the new tokens, and padding)."""
        def make(n, dtype=_INT):
            return torch.empty(n, dtype=dtype, device=self.device)
        return Batch(make(requests + 1), make(requests), make(requests + 1), make(rows, torch.int64), make(rows), make(1))

    def __call__(self, tables: torch.Tensor, cached: torch.Tensor, new: torch.Tensor, free: torch.Tensor, taken: torch.Tensor,
                 rows: int | None = None, out: Batch | None = None) -> Batch:
        """cached, new: [n] tokens that request s has, and that it gets; tables: [n, pages], whose rows are completed in place
        with pages free[taken], free[taken + 1], ...; taken: [1].  rows: length of slots and positions, at least the number of
        new tokens; or out, whose buffers are written and returned.  out.lengths may be cached and out.taken may
        be taken: a loop then carries them from step to step.  A batch that does not fit is flagged (read_status) and leaves
        tables, lengths and taken as they were, starts 0 and slots -1."""
        st, d = self._enter(), self._desc
        if out is None:
            _need(rows is not None, "rows is needed where no buffers are given")
            out = self.buffers(tables.shape[0], rows)
        at = self._form.places(tables, cached, new, free, taken, *out)
        if at is None:
            self._form.keep()
            self._check(tables, cached, new, free, taken, out)
            self._form.keep(tables, cached, new, free, taken, *out)
            at = self._form.places(tables, cached, new, free, taken, *out)
        (d.d_tables, d.d_cached, d.d_new, d.d_free, d.d_taken, d.d_starts, d.d_lengths, d.d_ends, d.d_slots, d.d_positions, d.d_taken_out) = at
        B.ans_page_tables(d, self._status, st)
        return out

    def _check(self, tables, cached, new, free, taken, out):
        d, dev = self._desc, self.device
        n, d.table_pages, d.table_stride = _check_tables(tables, dev)
        for t, k, what in ((cached, n, "cached"), (new, n, "new"), (taken, 1, "taken"), (out.starts, n + 1, "out.starts"), (out.lengths, n, "out.lengths"),
                           (out.ends, n + 1, "out.ends"), (out.taken, 1, "out.taken")):
            _vector_of(t, k, dev, what)
        _need(free.dim() == 1, "free must be a vector")
        _vector_of(free, free.shape[0], dev, "free")
        _need(out.slots.dim() == 1, "out.slots must be a vector")
        rows = out.slots.shape[0]
        _vector_of(out.slots, rows, dev, "out.slots", torch.int64)
        _vector_of(out.positions, rows, dev, "out.positions")
        _counts(free.shape[0], rows)
        d.n_seqs, d.n_free, d.rows = n, free.shape[0], rows


class Adapters(_Handle):
    """out = y + scales[i] * (x A_i^T) B_i^T for the rows of each request, i its adapter: low-rank adapters beside a projection
    that all requests share, y being the projection's output (a Linear without activation).

    a: [count, rank, in features], b: [count, out features, rank], bf16, contiguous, rank up to 128; scales: [count] fp32 or None.
    They are read where they lie, at each call.  For inference, as all handles here."""

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scales: torch.Tensor | None = None):
        super().__init__(a.device)
        _need(a.dim() == 3 and b.dim() == 3, "a is [count, rank, in features], b [count, out features, rank]")
        count, rank, n_in = a.shape
        _need(b.shape[0] == count and b.shape[2] == rank, "a and b differ in count or rank")
        _need(a.dtype is torch.bfloat16 and b.dtype is torch.bfloat16, "a and b must be bf16")
        _need(a.is_contiguous() and b.is_contiguous(), "a and b must be contiguous")
        _need(0 < rank <= 128 and n_in > 0, "rank must be 1 to 128, in features positive")
        _counts(count, n_in, b.shape[1])
        _on_device(b, self.device, "b")
        if scales is not None:
            _vector_of(scales, count, self.device, "scales", torch.float32)
        self.a, self.b, self.scales = a, b, scales
        self.count, self.rank, self.in_features, self.out_features = count, rank, n_in, b.shape[1]
        self._form = self._new_form()
        self._desc = d = B.ans_adapters_desc()
        d.d_a, d.d_b, d.d_scales = a.data_ptr() or None, b.data_ptr() or None, scales.data_ptr() or None if scales is not None else None
        d.count, d.rank, d.n_in, d.n_out = count, rank, n_in, b.shape[1]
        self._hold(a, b, scales)

    def __call__(self, x: torch.Tensor, y: torch.Tensor, which: torch.Tensor, starts: torch.Tensor, x_scales: torch.Tensor | None = None,
                 out: torch.Tensor | None = None) -> torch.Tensor:
        """x: [rows, in features] bf16, or float8_e4m3fn with x_scales [rows] (what RmsNorm gives); y: [rows, out features]
        bf16 or fp32; which: [n] int32, a request's adapter, -1: none; starts: [n + 1].  Returns out, y's type; the given
        buffer if there is one, which may be y.  Rows behind the last request's are not written."""
        st, d = self._enter(), self._desc
        if out is None:
            out = torch.empty(y.shape, dtype=y.dtype, device=self.device)
        at = self._form.places(x, x_scales, y, out, which, starts)
        if at is None:
            self._form.keep()
            self._check(x, x_scales, y, out, which, starts)
            d.d_room, d.room_bytes = None, B.ans_adapters_room_bytes(d)
            self._form.keep(x, x_scales, y, out, which, starts)
            at = self._form.places(x, x_scales, y, out, which, starts)
        if d.room_bytes:
            room = torch.empty(d.room_bytes, dtype=torch.uint8, device=self.device)        # kept until the call is queued
            d.d_room = room.data_ptr()
        d.d_x, d.d_x_scales, d.d_y, d.d_out, d.d_which, d.d_starts = at
        B.ans_adapters(d, self._status, st)
        return out

    def _check(self, x, x_scales, y, out, which, starts):
        d, dev = self._desc, self.device
        _need(x.dim() == 2 and x.shape[1] == self.in_features, "x must be [rows, in features]")
        rows = x.shape[0]
        _need(x.dtype in (torch.bfloat16, torch.float8_e4m3fn), "x must be bf16 or float8_e4m3fn")
        _need(y.shape == (rows, self.out_features) and out.shape == y.shape, "y and out must be [rows, out features]")
        _need(y.dtype in (torch.bfloat16, torch.float32) and out.dtype is y.dtype, "y must be bf16 or fp32, out of y's type")
        for t, what in ((x, "x"), (y, "y"), (out, "out")):
            _on_device(t, dev, what)
        if x_scales is not None:
            _vector_of(x_scales, rows, dev, "x_scales", torch.float32)
        _need(which.dim() == 1, "which must be a vector")
        n = which.shape[0]
        _vector_of(which, n, dev, "which")
        _vector_of(starts, n + 1, dev, "starts")
        d.x_stride, d.y_stride, d.out_stride = _rows(x, "x"), _rows(y, "y"), _rows(out, "out")
        _need(rows <= 1 or not y.numel() or out.data_ptr() != y.data_ptr() or d.out_stride == d.y_stride, "out lies over y with other strides")
        _counts(rows, n)
        d.rows, d.n_seqs, d.x_dtype, d.y_dtype = rows, n, _ELEMENT[x.dtype], _ELEMENT[y.dtype]


class BlockCache(_Handle):
    """A paged cache of keys and values in 8 bits with one scale for each page and head, and the attention over it (see
    ans_block_cache_desc in the header).  A value is code * scale; write() chooses powers of two for scales, so that what
    it stores is exact in bf16 and the same on every device.

    page_size and head_dim: multiples of 16 up to 256."""

    def __init__(self, n_pages: int, page_size: int, heads: int, head_dim: int, device="cuda"):
        _need(min(n_pages, page_size, heads, head_dim) > 0, "sizes must be positive")
        device = _cuda_device(device)
        self._take(*(t for _ in "kv" for t in (torch.zeros(n_pages, heads, page_size, head_dim, dtype=torch.int8, device=device),
                                               torch.ones(n_pages, heads, dtype=torch.float32, device=device))))

    @classmethod
    def wrap(cls, k_codes, k_scales, v_codes, v_scales) -> "BlockCache":
        """A cache on existing arrays (codes [pages, heads, page_size, head_dim] int8, scales [pages, heads] fp32), used in place."""
        self = cls.__new__(cls)
        self._take(k_codes, k_scales, v_codes, v_scales)
        return self

    def _take(self, k_codes, k_scales, v_codes, v_scales):
        _Handle.__init__(self, k_codes.device)
        _need(k_codes.dim() == 4, "codes have four dimensions")
        self.n_pages, self.heads, self.page_size, self.head_dim = k_codes.shape
        for t, dtype, shape, what in ((k_codes, torch.int8, k_codes.shape, "k_codes"), (v_codes, torch.int8, k_codes.shape, "v_codes"),
                                      (k_scales, torch.float32, k_codes.shape[:2], "k_scales"), (v_scales, torch.float32, k_codes.shape[:2], "v_scales")):
            _need(t.dtype is dtype and t.shape == shape and t.is_contiguous(), f"{what} must be a contiguous {dtype} tensor of {tuple(shape)}")
            _on_device(t, self.device, what)
        for size, what in ((self.page_size, "page_size"), (self.head_dim, "head_dim")):
            _need(size % 16 == 0 and 0 < size <= 256, f"{what} must be a multiple of 16 up to 256")
        _counts(self.n_pages, self.heads)
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self._wrote, self._seen = self._new_form(), self._new_form()
        self._desc = d = B.ans_block_cache_desc()
        d.d_k_codes, d.d_k_scales, d.d_v_codes, d.d_v_scales = (t.data_ptr() or None for t in (k_codes, k_scales, v_codes, v_scales))
        d.n_pages, d.page_size, d.heads, d.head_dim = self.n_pages, self.page_size, self.heads, self.head_dim
        self._write_batch, self._attend_batch, self._attend = B.ans_batch_desc(), B.ans_batch_desc(), B.ans_attend_desc()
        self._attend_args = None
        self._hold(k_codes, k_scales, v_codes, v_scales)

    def _batch(self, b, tables, lengths, starts, rows):
        n, b.table_pages, b.table_stride = _check_tables(tables, self.device)
        _counts(rows)
        b.n_seqs = n
        _vector_of(lengths, n, self.device, "lengths")
        _vector_of(starts, n + 1, self.device, "starts")
        b.rows = rows

    def write(self, k: torch.Tensor, v: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor) -> None:
        """k, v: [rows, heads, head_dim], bf16 or fp32, rows and heads at any stride: the batch's new tokens; lengths counts
        them already.  A page's scale begins anew when its first token is written, and grows with what is written behind it."""
        st, b = self._enter(), self._write_batch
        at = self._wrote.places(k, v, tables, lengths, starts)
        if at is None:
            self._wrote.keep()
            self._check_write(k, v, tables, lengths, starts)
            self._wrote.keep(k, v, tables, lengths, starts)
            at = self._wrote.places(k, v, tables, lengths, starts)
        b.d_tables, b.d_lengths, b.d_starts = at[2:]
        dtype, ks, vs = self._write_args
        B.ans_block_cache_write(self._desc, b, at[0], at[1], dtype, ks, vs, self._status, st)

    def _check_write(self, k, v, tables, lengths, starts):
        def strides(t, what):
            _need(t.dim() == 3 and t.shape[1:] == (self.heads, self.head_dim), f"{what} must be [rows, heads, head_dim]")
            _need(t.stride(2) == 1, f"the values of a head of {what} must be contiguous")
            _on_device(t, self.device, what)
            return t.stride()[:2]

        ks, vs = strides(k, "k"), strides(v, "v")
        _need(k.dtype in (torch.bfloat16, torch.float32), "k and v must be bf16 or fp32")
        _need(v.dtype is k.dtype and v.shape == k.shape, "k and v differ")
        self._batch(self._write_batch, tables, lengths, starts, k.shape[0])
        self._write_args = (_ELEMENT[k.dtype], ks, vs)

    def attend(self, q: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor, scale: float | None = None,
               causal: bool = True, window: int = 0, longest: int | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the batch's new tokens over the cache, which holds them already.  q: [rows, query heads, head_dim] bf16,
        query heads a multiple of the cache's; scale: of the logits, head_dim ** -0.5 unless given.  causal: a token sees
        itself and what is before it, else all of its sequence's tokens; the last `window` of these if that is not 0.
        longest: the most new tokens of a request, if known on the host (results do not depend on it, time does).
        Returns out, bf16, of q's shape; the given buffer if there is one, which may be q.  Rows that see nothing are 0, rows
        behind the last request's are not written."""
        st, b, d = self._enter(), self._attend_batch, self._attend
        if q.dim() == 3 and (q.data_ptr() % 16 or q.stride(2) != 1 or q.stride(0) % 8 or q.stride(1) % 8):
            if q.data_ptr() % 16 or q.stride(2) != 1 or any(step % 8 for step in _steps(q)):
                q = q.clone(memory_format=torch.contiguous_format)
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=self.device)
        at = self._seen.places(q, out, tables, lengths, starts)
        if at is None or (scale, causal, window, longest) != self._attend_args:
            self._seen.keep()
            self._check_attend(q, out, tables, lengths, starts, scale, causal, window, longest)
            at = tuple(t.data_ptr() for t in (q, out, tables, lengths, starts))
            d.d_q, d.d_out, b.d_tables, b.d_lengths, b.d_starts = at
            self._room_bytes = B.ans_attend_room_bytes(self._desc, b, d)
            self._seen.keep(q, out, tables, lengths, starts)           # nothing is left to refuse
            self._attend_args = (scale, causal, window, longest)
        d.d_q, d.d_out, b.d_tables, b.d_lengths, b.d_starts = at
        d.room_bytes = self._room_bytes
        if self._room_bytes:
            room = torch.empty(self._room_bytes, dtype=torch.uint8, device=self.device)
            d.d_room = room.data_ptr()
        B.ans_attend(self._desc, b, d, self._status, st)
        return out

    def _check_attend(self, q, out, tables, lengths, starts, scale, causal, window, longest):
        d = self._attend
        _need(q.dim() == 3 and q.shape[2] == self.head_dim, "q must be [rows, query heads, head_dim]")
        _need(q.shape[1] > 0 and q.shape[1] % self.heads == 0, "the query heads must be a multiple of the cache's heads")
        _need(q.dtype is torch.bfloat16 and out.dtype is torch.bfloat16, "q and out must be bf16")
        _need(out.shape == q.shape and out.stride(2) == 1, "out must be of q's shape, the values of a head contiguous")
        qs, outs = _steps(q), _steps(out)
        _need(out.data_ptr() % 4 == 0 and outs[0] % 2 == 0 and outs[1] % 2 == 0, "the heads of out must start on 4 bytes")
        _need(not q.numel() or out.data_ptr() != q.data_ptr() or outs == qs, "out lies over q with other strides")
        _need(not _overlaps(out), "the heads of out lie over each other")
        _on_device(q, self.device, "q")
        _on_device(out, self.device, "out")
        _need(window >= 0, "window must not be negative")
        _need(longest is None or longest > 0, "longest must be positive")
        self._batch(self._attend_batch, tables, lengths, starts, q.shape[0])
        d.q_token_stride, d.q_head_stride, d.out_token_stride, d.out_head_stride = *qs, *outs
        d.q_heads, d.longest, d.window, d.causal = q.shape[1], min(longest or 0, q.shape[0]), min(window, 2 ** 31 - 1), int(causal)
        d.scale = self.head_dim ** -0.5 if scale is None else scale
