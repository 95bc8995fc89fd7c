"""Binding of the paged 8-bit cache (tq_pages_* of include/turboquant.h): marshalling and checks of arguments only.

A batch is `table` (int32 [n_seqs][width]: the page that holds each span of a sequence's tokens), `lens` (int32 [n_seqs]: tokens
of each sequence, those of the call among them), `starts` (int32 [n_seqs + 1]: where each sequence's rows begin in the call's
arrays; None: every sequence has max_new rows) and `max_new` (at least the most rows of a sequence).  They stay on the GPU: nothing
here waits for it, and every call can be captured into a graph (torch.cuda.graph).

Scratch memory is the binding's: every thread has its own on every stream that it calls on, and a captured call has its own in the
graph's memory.  So threads, streams and graphs may read one cache at the same time (tq_pages_attend, tq_pages_select); what writes to
it (tq_pages_append and the pool's calls) the program puts in order with everything else, as for any tensor.
"""
from __future__ import annotations

import ctypes as C
import operator
import threading

import torch

from . import _lib
from .api import TQ_BF16, TQ_F32, TurboQuantError, _check

_TYPES = {torch.float8_e4m3fn: 0, torch.int8: 1}


def _where(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TurboQuantError(f"{what}: expected a GPU tensor")


class _Scratch(threading.local):
    """A thread's scratch memory of a cache: `spaces` by stream, and `call`, the struct with that of the stream it was used on last."""

    def __init__(self, c):
        self.spaces, self.call = {}, _lib.TqPagesCall(self.without(c), 0)

    @staticmethod
    def without(c):
        c = _lib.TqPages.from_buffer_copy(c)
        c.workspace, c.workspace_bytes = 0, 0
        return c


class Pages:
    """Owns the tq_pages struct and keeps what it points to alive.

    k, v [n_pages][n_heads][page_tokens][d] (torch.float8_e4m3fn or torch.int8), k_scale, v_scale float32 [n_pages][n_heads],
    bounds bfloat16 [n_pages][n_heads][2][d] or None (needed by tq_pages_select), refs int32 [n_pages] or None (needed by the
    pool's calls).  All contiguous, on one GPU."""

    def __init__(self, k, v, k_scale, v_scale, bounds=None, refs=None):
        _where(k, "k")
        if k.dim() != 4 or k.dtype not in _TYPES:
            raise TurboQuantError(f"k: expected [n_pages][n_heads][page_tokens][d] of {' or '.join(map(str, _TYPES))}, got {tuple(k.shape)} of {k.dtype}")
        n, h, page, d = k.shape
        for t, what, dtype, shape in ((k, "k", k.dtype, (n, h, page, d)), (v, "v", k.dtype, (n, h, page, d)), (k_scale, "k_scale", torch.float32, (n, h)),
                                      (v_scale, "v_scale", torch.float32, (n, h)), (bounds, "bounds", torch.bfloat16, (n, h, 2, d)),
                                      (refs, "refs", torch.int32, (n,))):
            if t is None and what in ("bounds", "refs"):
                continue
            _where(t, what)
            if t.dtype != dtype or tuple(t.shape) != shape:
                raise TurboQuantError(f"{what}: expected {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
            if not t.is_contiguous() or t.device != k.device:
                raise TurboQuantError(f"{what}: expected a contiguous tensor on {k.device}")
        self.k, self.v, self.k_scale, self.v_scale, self.bounds, self.refs = k, v, k_scale, v_scale, bounds, refs
        self.n_pages, self.n_heads, self.page_tokens, self.d = int(n), int(h), int(page), int(d)
        self.device = k.device
        self.workspace, self._reserved = None, []
        self.c = _lib.TqPages()
        self.c.d, self.c.n_heads, self.c.page_tokens, self.c.type, self.c.n_pages = self.d, self.n_heads, self.page_tokens, _TYPES[k.dtype], self.n_pages
        self.c.k, self.c.v = k.data_ptr(), v.data_ptr()
        self.c.k_scale, self.c.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
        self.c.bounds = 0 if bounds is None else bounds.data_ptr()
        self.c.refs = 0 if refs is None else refs.data_ptr()
        self.c.workspace, self.c.workspace_bytes = 0, 0
        self._scratch = _Scratch(self.c)

    def _with_scratch(self, need: int):
        """-> the struct of a call that uses `need` bytes on the current stream (the cache's GPU is the current one), and what holds them
        until the call has been made."""
        if need == 0:
            return _Scratch.without(self.c), None
        if torch.cuda.is_current_stream_capturing():  # from the graph's memory, which stays the graph's
            space = torch.empty(need, dtype=torch.uint8, device=self.device)
            c = _Scratch.without(self.c)
            c.workspace, c.workspace_bytes = space.data_ptr(), need
            return c, space
        mine, stream = self._scratch, torch.cuda.current_stream().cuda_stream
        space = mine.spaces.get(stream)
        have = 0 if space is None else space.numel()
        if have < need:
            # at least half as much again, for sizes that creep up; torch's allocator gives the old one away in the stream's order
            space = mine.spaces[stream] = torch.empty(max(need, have + have // 2), dtype=torch.uint8, device=self.device)
        if mine.call.stream != stream or mine.call.c.workspace != space.data_ptr():
            c = _Scratch.without(self.c)
            c.workspace, c.workspace_bytes = space.data_ptr(), space.numel()
            mine.call = _lib.TqPagesCall(c, stream)
        return mine.call.c, space

    def reserve_bytes(self, need: int):
        """Make the calling thread's scratch memory on the current stream at least `need` bytes, so that no call there asks torch for more.
        It is also the workspace of this object's struct (`c`), for calls of the C ABI; one that it takes the place of there is kept."""
        if need > 0:
            with torch.cuda.device(self.device):
                c, space = self._with_scratch(need)
            if need > self.c.workspace_bytes:
                self._reserved.append(space)
                self.workspace, self.c.workspace, self.c.workspace_bytes = space, c.workspace, c.workspace_bytes
        return self

    def reserve_attend(self, n_rows, n_seqs, width, n_heads_q, max_new=1, n_chosen=0, window=0):
        """Size the workspace for tq_pages_attend calls of these sizes."""
        b = _lib.TqBatch(n_seqs=n_seqs, max_new=max_new, n_rows=n_rows, width=width, table_stride=width)
        return self.reserve_bytes(int(_lib.load().tq_pages_attend_workspace_bytes(C.byref(self.c), C.byref(b), n_heads_q, n_chosen, window)))

    def reserve_select(self, n_rows, n_seqs, width, max_new=1):
        b = _lib.TqBatch(n_seqs=n_seqs, max_new=max_new, n_rows=n_rows, width=width, table_stride=width)
        return self.reserve_bytes(int(_lib.load().tq_pages_select_workspace_bytes(C.byref(self.c), C.byref(b))))

    def reserve_pool(self, n: int = 0):
        return self.reserve_bytes(_pool_bytes(self, n))


def make_pages(n_pages: int, n_heads: int, d: int, page_tokens: int, dtype=torch.float8_e4m3fn, bounds: bool = False, device="cuda") -> Pages:
    """An empty cache: zero codes, scales 1, every page free."""
    shape = (n_pages, n_heads, page_tokens, d)
    codes = [torch.zeros(shape, dtype=torch.uint8, device=device).view(dtype) for _ in range(2)]
    scales = [torch.ones(shape[:2], dtype=torch.float32, device=device) for _ in range(2)]
    return Pages(*codes, *scales, bounds=torch.zeros((n_pages, n_heads, 2, d), dtype=torch.bfloat16, device=device) if bounds else None,
                 refs=torch.zeros(n_pages, dtype=torch.int32, device=device))


def _ints(t, what, shape, device):
    _where(t, what)
    if t.dtype != torch.int32 or tuple(t.shape) != shape:
        raise TurboQuantError(f"{what}: expected int32 {shape}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_contiguous() or t.device != device:
        raise TurboQuantError(f"{what}: expected a contiguous tensor on {device}")
    return t.data_ptr()


def _int32(x, what):
    """(a ctypes argument would lose what lies above 32 bits)"""
    try:
        v = operator.index(x)
    except TypeError:
        raise TurboQuantError(f"{what}: expected a whole number, got {x!r}") from None
    if not -2**31 <= v < 2**31:
        raise TurboQuantError(f"{what}: {v} has more than 32 bits")
    return v


def _batch(p: Pages, n_rows, table, lens, starts, max_new: int):
    """n_rows None: a call without rows."""
    _where(table, "table")
    if table.dtype != torch.int32 or table.dim() != 2 or (table.numel() and table.shape[1] > 1 and table.stride(1) != 1) or table.device != p.device:
        raise TurboQuantError(f"table: expected int32 [n_seqs][width] with contiguous rows on {p.device}, got {table.dtype} {tuple(table.shape)}")
    n, width = table.shape
    if n > 1 and table.stride(0) < width:
        raise TurboQuantError("table: rows overlap")
    max_new = _int32(max_new, "max_new")
    if max_new < 0 or (starts is None and n_rows is not None and n_rows < n * max_new):
        raise TurboQuantError(f"max_new: {n} sequences of {max_new} rows each, and {n_rows} rows")
    b = _lib.TqBatch()
    b.n_seqs, b.max_new, b.n_rows, b.width = n, max_new, n_rows or 0, width
    b.table_stride = table.stride(0) if n > 1 else width
    b.table, b.lens = table.data_ptr(), 0 if lens is None else _ints(lens, "lens", (n,), p.device)
    b.starts = 0 if starts is None else _ints(starts, "starts", (n + 1,), p.device)
    return b


def _rows(t, what, p: Pages, dtype=None, shape=None):
    """-> (address, dtype number, elements between rows, between heads)."""
    _where(t, what)
    if t.dtype not in (torch.float32, torch.bfloat16) or (dtype is not None and t.dtype != dtype):
        raise TurboQuantError(f"{what}: unsupported dtype {t.dtype}")
    if t.dim() != 3 or t.shape[2] != p.d or (shape is not None and t.shape != shape):
        raise TurboQuantError(f"{what}: expected [rows][heads][{p.d}]{'' if shape is None else f' as {tuple(shape)}'}, got {tuple(t.shape)}")
    if t.stride(2) != 1 or t.device != p.device:
        raise TurboQuantError(f"{what}: expected contiguous vectors on {p.device}")
    return (C.c_void_p(t.data_ptr()), TQ_F32 if t.dtype == torch.float32 else TQ_BF16, t.stride(0) if t.shape[0] > 1 else 0,
            t.stride(1) if t.shape[1] > 1 else 0)


def _writable(t, what):
    if any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
        raise TurboQuantError(f"{what}: rows overlap")


def _call(p: Pages, name: str, *args, need: int = 0):
    """One library call on the current stream of the cache's GPU, with `need` bytes of scratch memory."""
    with torch.cuda.device(p.device):
        c, space = p._with_scratch(need)
        _check(getattr(_lib.load(), name)(C.byref(c), *args, C.c_void_p(torch.cuda.current_stream().cuda_stream)), name)


def _check_heads(n, p: Pages):
    if n <= 0 or n % p.n_heads:
        raise TurboQuantError(f"q: {n} heads for {p.n_heads} heads of the cache")


def tq_pages_append(p: Pages, k, v, table, lens, starts, max_new: int):
    """Store new keys and values [rows][n_heads][d] (float32 or bfloat16)."""
    st = _lib.call().pages_append(p.c, p.k, k, v, table, lens, starts, max_new)
    if st is not None:
        return _check(st, "tq_pages_append")
    pk, dtype, row, head = _rows(k, "k", p)
    pv, _, row_v, head_v = _rows(v, "v", p, k.dtype, k.shape)
    if k.shape[1] != p.n_heads:
        raise TurboQuantError(f"k: {k.shape[1]} heads for {p.n_heads} heads of the cache")
    if (row, head) != (row_v, head_v):
        raise TurboQuantError("k and v: expected the same strides")
    b = _batch(p, k.shape[0], table, lens, starts, max_new)
    _call(p, "tq_pages_append", C.byref(b), pk, pv, dtype, row, head)


def tq_pages_attend(p: Pages, q, table, lens, starts, max_new: int, scale: float, out, lse=None, window: int = 0, chosen=None):
    """q, out [rows][n_heads_q][d]; lse float32 [rows][n_heads_q] or None; chosen int32 [rows][n_heads][n_chosen] or None."""
    st = _lib.call().pages_attend(p._scratch.call, p.k, q, table, lens, starts, max_new, scale, out, lse, window, chosen)
    if st is not None:
        return _check(st, "tq_pages_attend")
    pq, dtype, row, head = _rows(q, "q", p)
    po, _, row_o, head_o = _rows(out, "out", p, q.dtype, q.shape)
    _writable(out, "out")
    n, heads = q.shape[:2]
    _check_heads(heads, p)
    if lse is not None:
        _where(lse, "lse")
        if lse.dtype != torch.float32 or tuple(lse.shape) != (n, heads) or not lse.is_contiguous() or lse.device != p.device:
            raise TurboQuantError(f"lse: expected contiguous float32 {(n, heads)} on {p.device}, got {lse.dtype} {tuple(lse.shape)}")
    n_chosen = 0
    if chosen is not None:
        _where(chosen, "chosen")
        n_chosen = chosen.shape[-1] if chosen.dim() == 3 else 0
        _ints(chosen, "chosen", (n, p.n_heads, n_chosen), p.device)
    b, window = _batch(p, n, table, lens, starts, max_new), _int32(window, "window")
    need = int(_lib.load().tq_pages_attend_workspace_bytes(C.byref(p.c), C.byref(b), heads, n_chosen if chosen is not None else 0, window))
    # (an empty list is a list: its tensor may have no address)
    pc = None if chosen is None else C.c_void_p(chosen.data_ptr() or p.c.k)
    _call(p, "tq_pages_attend", C.byref(b), pq, dtype, row, head, heads, C.c_float(scale), window, pc, n_chosen, po, row_o, head_o,
          None if lse is None else C.c_void_p(lse.data_ptr()), need=need)


def tq_pages_select(p: Pages, q, table, lens, starts, max_new: int, chosen, keep_first: int = 1, keep_last: int = 1):
    """chosen int32 [rows][n_heads][n_chosen] out."""
    st = _lib.call().pages_select(p._scratch.call, p.k, q, table, lens, starts, max_new, chosen, keep_first, keep_last)
    if st is not None:
        return _check(st, "tq_pages_select")
    pq, dtype, row, head = _rows(q, "q", p)
    n, heads = q.shape[:2]
    _check_heads(heads, p)
    _where(chosen, "chosen")
    n_chosen = chosen.shape[-1] if chosen.dim() == 3 else 0
    pc = _ints(chosen, "chosen", (n, p.n_heads, n_chosen), p.device)
    if p.bounds is None:
        raise TurboQuantError("tq_pages_select: the cache has no bounds")
    b, keep_first, keep_last = _batch(p, n, table, lens, starts, max_new), _int32(keep_first, "keep_first"), _int32(keep_last, "keep_last")
    need = int(_lib.load().tq_pages_select_workspace_bytes(C.byref(p.c), C.byref(b)))
    _call(p, "tq_pages_select", C.byref(b), pq, dtype, row, head, heads, keep_first, keep_last, C.c_void_p(pc), n_chosen, need=need)


def _pool(p: Pages):
    if p.refs is None:
        raise TurboQuantError("the cache has no reference counts")


def _pool_bytes(p: Pages, n: int = 0):
    return int(_lib.load().tq_pages_pool_workspace_bytes(C.byref(p.c), n))


def _one(t, what, p: Pages):
    return None if t is None else C.c_void_p(_ints(t, what, (1,), p.device))


def tq_pages_reserve(p: Pages, table, lens, max_new: int, missing=None, starts=None):
    """Pages for the new tokens of every sequence (without starts: the last max_new); missing int32 [1] out: pages that were not there."""
    st = _lib.call().pages_reserve(p._scratch.call, p.k, table, lens, starts, max_new, missing)
    if st is not None:
        return _check(st, "tq_pages_reserve")
    _pool(p)
    b = _batch(p, None, table, lens, starts, max_new)
    _call(p, "tq_pages_reserve", C.byref(b), _one(missing, "missing", p), need=_pool_bytes(p))


def tq_pages_fork(p: Pages, table, lens, parents, children, missing=None):
    """Rows children[i] become copies of rows parents[i]."""
    st = _lib.call().pages_fork(p._scratch.call, p.k, table, lens, parents, children, missing)
    if st is not None:
        return _check(st, "tq_pages_fork")
    _pool(p)
    n = int(parents.shape[0]) if isinstance(parents, torch.Tensor) and parents.dim() == 1 else -1
    pp, pc = _ints(parents, "parents", (n,), p.device), _ints(children, "children", (n,), p.device)
    b = _batch(p, None, table, lens, None, 0)
    _call(p, "tq_pages_fork", C.byref(b), C.c_void_p(pp), C.c_void_p(pc), n, _one(missing, "missing", p), need=_pool_bytes(p, n))


def tq_pages_free(p: Pages, table, lens, rows):
    """Rows give back their pages."""
    st = _lib.call().pages_free(p.c, p.k, table, lens, rows)
    if st is not None:
        return _check(st, "tq_pages_free")
    _pool(p)
    n = int(rows.shape[0]) if isinstance(rows, torch.Tensor) and rows.dim() == 1 else -1
    pr = _ints(rows, "rows", (n,), p.device)
    b = _batch(p, None, table, lens, None, 0)
    _call(p, "tq_pages_free", C.byref(b), C.c_void_p(pr), n)


def tq_pages_compact(p: Pages, table, n_live=None):
    """The pages in use move to the front of the pool; n_live int32 [1] out."""
    st = _lib.call().pages_compact(p._scratch.call, p.k, table, n_live)
    if st is not None:
        return _check(st, "tq_pages_compact")
    _pool(p)
    b = _batch(p, None, table, None, None, 0)
    _call(p, "tq_pages_compact", C.byref(b), _one(n_live, "n_live", p), need=_pool_bytes(p))


def tq_pages_copy(p: Pages, src, dst):
    """Page src[i] to page dst[i]."""
    st = _lib.call().pages_copy(p.c, p.k, src, dst)
    if st is not None:
        return _check(st, "tq_pages_copy")
    n = int(src.shape[0]) if isinstance(src, torch.Tensor) and src.dim() == 1 else -1
    ps, pd = _ints(src, "src", (n,), p.device), _ints(dst, "dst", (n,), p.device)
    _call(p, "tq_pages_copy", C.c_void_p(ps), C.c_void_p(pd), n)
