"""A destination's serving operators on the device: a paged cache of keys and values, the calls
that take, share, move and free its pages, attention over whole prompts (a miss) and attention
of requests that share a cached prefix (a hit, and every decoded token). Marshalling only; the
library does the work.

    pool = PagePool(k, v, refs)                       # k, v [layers, pages, heads, tokens, dim]
    pool.extend(table, None, length)                  # pages for new sequences
    attend_prompt(q, k, v, off, off, scale, out=o)    # a miss: the whole prompt ...
    pool.append(0, k, v, off, length, table)          # ... whose keys and values are kept
    pool.fork(table, parent, length, child)           # a request behind a cached prefix
    attend_shared(q, pool, 0, q_off, group_off, table, length, own_table, own_len, scale, out=o)
    pool.free(table, length)                          # an eviction

Tensors are on the GPU. Offsets, lengths and page tables are int32; a call enqueues kernels on
``stream`` (default: the current one) and returns. Problems that only the device sees set bits
of ``pool.err``, of the workspace's ``err`` or of an ``err`` given (``CR_ERR_*``), and the sequence
concerned is skipped as the library documents. Nothing here is differentiable: tensors that require
a gradient are refused where gradients are recorded.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.CR_BF16, torch.float16: B.CR_F16}
_INT32, _FLOAT32 = torch.int32, torch.float32
_HERE = contextlib.nullcontext()
_raw_stream, _device = B._raw_stream, B._device
_pack_rows, _pack_prompt, _pack_shared, _RANGE = B.ROWS.pack, B.PROMPT_ARGS.pack, B.SHARED_ARGS.pack, (struct.error, OverflowError)


def _dtype(t: torch.Tensor) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise B.CrError(f"bfloat16 or float16 wanted, not {t.dtype}") from None


# The checks below are in every call of a serving loop, whose small calls are bound by the host: each attribute
# of a tensor is looked at once, and what a check refuses is told apart afterwards.

def _rows(t: torch.Tensor):
    """Fields of a cr_rows: [tokens, heads, dim] with any strides of tokens and heads."""
    stride = t.stride()
    if len(stride) != 3 or stride[2] != 1:
        raise B.CrError("rows are [tokens, heads, dim] with dim contiguous")
    if not t.is_cuda:
        raise B.CrError("libcr takes device tensors")
    return t.data_ptr(), stride[0], stride[1]


_grad_on = torch.is_grad_enabled


def _refuse_grad():
    raise B.CrError("the serving calls have no gradient: call them under torch.no_grad(), or detach what requires one")


def _refuse(t, n):
    if t.dtype is not _INT32:
        raise B.CrError(f"offsets, lengths and tables are int32, not {t.dtype}")
    if n is not None and t.numel() != n:
        raise B.CrError(f"{n} entries wanted, not {t.numel()}")
    B._ptr(t)


def _index(t: torch.Tensor, n: Optional[int] = None) -> int:
    """Pointer of an int32 array of n elements (any, if n is None)."""
    if t.dtype is not _INT32 or not t.is_cuda or not t.is_contiguous() or (n is not None and t.numel() != n):
        _refuse(t, n)
    return t.data_ptr()


def _table(t: torch.Tensor, n: int):
    """Pointer and width of a table of n rows."""
    shape = t.shape
    if len(shape) != 2 or shape[0] != n:
        raise B.CrError(f"a table is [{n}, width], not {list(shape)}")
    return _index(t), shape[1]


def _taken_on(stream):
    """Memory for a call is taken from the pool of the stream that it works on: a piece of the current stream's may
    still be written to by what is enqueued there."""
    return _HERE if stream is None else torch.cuda.stream(stream)


def _new_out(q, stream):
    with _taken_on(stream):
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if stream is not None:
        out.record_stream(torch.cuda.current_stream())  # the caller's, where it goes on with it
    return out


class _Memory:
    """Device memory that calls on any stream use: once its owner is dropped, it is not handed out before the
    work enqueued on each of them is done. (Not what a graph captured: its owner has to outlive the graph.)"""

    def __init__(self, *tensors):
        self._memory, self._seen = list(tensors), set()

    def _on(self, stream) -> Optional[int]:
        """Handle of the stream of a call: ``stream``, or the current one."""
        handle = _raw_stream(_device()) if stream is None and _raw_stream else B._stream(stream)
        if handle not in self._seen:
            self._see(handle, stream)
        return handle

    def _see(self, handle, stream):
        if not torch.cuda.is_current_stream_capturing():
            s = torch.cuda.current_stream() if stream is None else stream
            for t in self._memory:
                t.record_stream(s)
            self._seen.add(handle)


class Workspace(_Memory):
    """Device scratch of an attention call and its error word."""

    def __init__(self, nbytes: int, device, err: Optional[torch.Tensor] = None):
        self.buf = torch.empty(max(16, nbytes), dtype=torch.uint8, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device) if err is None else err
        self.args = self.buf.data_ptr(), self.buf.numel(), _index(self.err, 1)
        super().__init__(self.buf, self.err)


class PagePool(_Memory):
    """Handle of a paged cache. ``k``, ``v``: [layers, pages, heads, tokens, dim] (``order``
    "head") or [layers, pages, tokens, heads, dim] ("token"), bfloat16 or float16, equal
    strides; ``refs``: int32 [pages], how many table entries name a page (0 = free)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, refs: torch.Tensor, order: str = "head"):
        if order not in ("head", "token"):
            raise ValueError(f"unknown order {order!r}")
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(4) != 1:
            raise B.CrError("k and v are five-dimensional alike, with dim contiguous")
        if not (k.is_cuda and v.is_cuda):
            raise B.CrError("libcr takes device tensors")
        h, t = (2, 3) if order == "head" else (3, 2)
        self.k, self.v, self.refs, self.order = k, v, refs, order
        self.layers, self.num_pages, self.heads, self.page_tokens, self.dim = k.shape[0], k.shape[1], k.shape[h], k.shape[t], k.shape[4]
        self.err = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.c = B.CrKvCache(_dtype(k), self.heads, self.dim, self.page_tokens, self.num_pages, self.layers, k.data_ptr(),
                             v.data_ptr(), k.stride(0), k.stride(1), k.stride(h), k.stride(t), _index(refs, self.num_pages))
        self._ref, self._err = ctypes.byref(self.c), _index(self.err)
        self._ws = torch.empty(B.cr_pages_workspace_bytes(self.num_pages, 0), dtype=torch.uint8, device=k.device)
        self._ws_for = 0  # sequences that it is known to be large enough for
        super().__init__(k, v, refs, self.err, self._ws)

    @classmethod
    def empty(cls, layers: int, num_pages: int, heads: int, page_tokens: int, dim: int, dtype=torch.bfloat16, device="cuda",
              order: str = "head") -> "PagePool":
        """A new cache, all pages free."""
        shape = (layers, num_pages) + ((heads, page_tokens) if order == "head" else (page_tokens, heads)) + (dim,)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device),
                   torch.zeros(num_pages, dtype=torch.int32, device=device), order)

    def _scratch(self, n: int, stream):
        """The page calls' workspace, kept with the handle: its calls are for one stream at a time. It stays where it
        is until a call has more than about 1.5 sequences per page of the cache; at least doubled then, so that those
        it has outgrown are no more than it."""
        if n > self._ws_for:
            nbytes = B.cr_pages_workspace_bytes(self.num_pages, n)
            if nbytes > self._ws.numel():
                with _taken_on(stream):
                    self._ws = torch.empty(max(nbytes, 2 * self._ws.numel()), dtype=torch.uint8, device=self.k.device)
                self._memory.append(self._ws)  # the smaller one stays: captured graphs may go on using it
                self._seen.clear()
            self._ws_for = n
        return self._ws.data_ptr(), self._ws.numel(), self._err, self._on(stream)

    def pages_of(self, tokens: int) -> int:
        return -(-tokens // self.page_tokens)

    def extend(self, table, len_old, len_new, stream=None):
        """Free pages for sequences that grow from len_old (None: 0) to len_new tokens."""
        n = len_new.numel()
        new, old = _index(len_new), None if len_old is None else _index(len_old, n)
        p, width = _table(table, n)
        B._check(B.load().cr_pages_extend(self._ref, old, new, n, p, width, *self._scratch(n, stream)), "cr_pages_extend")

    def fork(self, table, parent, length, child, stream=None):
        """child[i]: the first length[i] tokens of table[parent[i]], the partial tail copied."""
        n, rows = parent.numel(), table.shape[0]
        (p, width), (c, child_width) = _table(table, rows), _table(child, n)
        B._check(B.load().cr_pages_fork(self._ref, p, rows, width, _index(parent), _index(length, n), n, c, child_width,
                                        *self._scratch(n, stream)), "cr_pages_fork")

    def free(self, table, length, stream=None):
        """Gives the pages of every row's first length tokens back."""
        n = length.numel()
        p, width = _table(table, n)
        B._check(B.load().cr_pages_free(self._ref, p, width, _index(length), n, self._err, self._on(stream)), "cr_pages_free")

    def compact(self, table, length, table_out=None, refs_out=None, stream=None):
        """Moves the live pages to the front and renames the table's entries (in place, if no
        other place is given). Of several tables, each but the last call's gives ``refs_out``
        another place; the last may be None."""
        refs = _index(self.refs if refs_out is None else refs_out, self.num_pages)
        p = lengths = out = None
        rows = width = 0
        if table is not None:
            rows = length.numel()
            p, width = _table(table, rows)
            lengths, out = _index(length), p if table_out is None else _index(table_out, rows * width)
        B._check(B.load().cr_pages_compact(self._ref, p, lengths, rows, width, out, refs, *self._scratch(0, stream)), "cr_pages_compact")

    def copy(self, src, dst, stream=None):
        """Contents of page src[i] to page dst[i], all layers."""
        n = src.numel()
        B._check(B.load().cr_pages_copy(self._ref, _index(src), _index(dst, n), n, self._err, self._on(stream)), "cr_pages_copy")

    def append(self, layer: int, k, v, off, length, table, stream=None):
        """Rows off[i]..off[i+1] of k and v ([total, heads, dim]) become the last tokens of the
        length[i] of sequence i."""
        shape, n, dtype = k.shape, length.numel(), self.k.dtype
        if len(shape) != 3 or shape[1] != self.heads or shape[2] != self.dim or shape != v.shape or k.dtype is not dtype or v.dtype is not dtype:
            raise B.CrError("new keys and values have the cache's heads, dim and type")
        if (k.requires_grad or v.requires_grad) and _grad_on():
            _refuse_grad()
        p, width = _table(table, n)
        B._check(B.load().cr_kv_append(self._ref, layer, _pack_rows(*_rows(k)), _pack_rows(*_rows(v)), shape[0],
                                       _index(off, n + 1), _index(length), n, p, width, self._err, self._on(stream)), "cr_kv_append")


def _check_out(q, shape, out, lse):
    if out.shape != shape or out.dtype is not q.dtype:
        raise B.CrError("out has q's shape and type")
    if lse is not None:
        rows = lse.shape
        if lse.dtype is not _FLOAT32 or len(rows) != 2 or rows[0] != shape[0] or rows[1] != shape[1]:
            raise B.CrError("lse is float32 [tokens, heads]")


def prompt_workspace(q, k, q_off, err: Optional[torch.Tensor] = None) -> Workspace:
    """Scratch for ``attend_prompt`` of tensors of these shapes."""
    (nq, hq, d), (nk, hkv, _) = q.shape, k.shape
    a = B.CrAttnPromptArgs(_dtype(q), hq, hkv, d, q_off.numel() - 1, 1, nq, nk, 1.0)
    return Workspace(B.cr_attn_prompt_workspace_bytes(a), q.device, err)


def attend_prompt(q, k, v, q_off, k_off, scale: float, *, out=None, lse=None, causal: bool = True,
                  ws: Optional[Workspace] = None, err: Optional[torch.Tensor] = None, stream=None):
    """Attention of packed sequences: q [total_q, heads_q, dim], k, v [total_k, heads_kv, dim],
    sequence b at q_off[b]..q_off[b+1] and k_off[b]..k_off[b+1]. Returns out (and fills lse,
    float32 [total_q, heads_q], if given). Problems that only the device sees set bits of ``ws.err`` or,
    where no workspace is given, of ``err`` (int32 [1]); with neither they show in no word."""
    if ws is not None and err is not None:
        raise B.CrError("a workspace has an error word of its own")
    shape, keys, dtype = q.shape, k.shape, q.dtype
    if keys != v.shape or len(keys) != 3 or len(shape) != 3 or keys[2] != shape[2] or k.dtype is not dtype or v.dtype is not dtype:
        raise B.CrError("q, k and v have one type and dim, k and v one shape")
    if (q.requires_grad or k.requires_grad or v.requires_grad) and _grad_on():
        _refuse_grad()
    code = _dtype(q)
    if out is None:
        out = _new_out(q, stream)
    _check_out(q, shape, out, lse)
    n = q_off.numel()
    try:
        a = _pack_prompt(code, shape[1], keys[1], shape[2], n - 1, causal, shape[0], keys[0], scale, *_rows(q), *_rows(k), *_rows(v),
                         *_rows(out), B._ptr(lse) or 0, _index(q_off), _index(k_off, n))
    except _RANGE as e:
        raise B.CrError(f"an argument is out of range: {e}") from None
    if ws is None:
        with _taken_on(stream):
            ws = prompt_workspace(q, k, q_off, err)
    B._check(B.load().cr_attn_prompt(a, *ws.args, ws._on(stream)), "cr_attn_prompt")
    return out


def shared_workspace(q, pool: PagePool, group_off, prefix_table, own_table, err: Optional[torch.Tensor] = None) -> Workspace:
    """Scratch for ``attend_shared`` of tensors of these shapes."""
    batch, own_width = own_table.shape
    a = B.CrAttnSharedArgs(q.shape[1], 0, batch, group_off.numel() - 1, q.shape[0], prefix_table.shape[1], own_width, 1.0)
    return Workspace(B.cr_attn_shared_workspace_bytes(pool.c, a), q.device, pool.err if err is None else err)


def attend_shared(q, pool: PagePool, layer: int, q_off, group_off, prefix_table, prefix_len, own_table, own_len,
                  scale: float, *, out=None, lse=None, ws: Optional[Workspace] = None, stream=None):
    """Attention of requests in groups that share a cached prefix: requests group_off[g] ..
    group_off[g+1] see the prefix_len[g] tokens of prefix_table[g] and, causally, their own
    own_len[r] tokens of own_table[r], the last of which are the queries' (append them first).
    q [total_q, heads_q, dim], request r's at q_off[r]..q_off[r+1]. Returns out. Tables about as
    wide as their longest row keep the GPU busy: the widths stand for the lengths, which only the
    device knows."""
    shape = q.shape
    if q.dtype is not pool.k.dtype or len(shape) != 3 or shape[2] != pool.dim:
        raise B.CrError("q has the cache's type and dim")
    if (q.requires_grad or pool.k.requires_grad or pool.v.requires_grad) and _grad_on():
        _refuse_grad()
    if out is None:
        out = _new_out(q, stream)
    _check_out(q, shape, out, lse)
    batch, groups = own_len.numel(), group_off.numel() - 1
    own, own_width = _table(own_table, batch)
    prefix, prefix_width = _table(prefix_table, groups)
    try:
        a = _pack_shared(shape[1], layer, batch, groups, shape[0], prefix_width, own_width, scale, *_rows(q), *_rows(out),
                         B._ptr(lse) or 0, _index(q_off, batch + 1), _index(group_off), prefix, _index(prefix_len, groups), own, _index(own_len))
    except _RANGE as e:
        raise B.CrError(f"an argument is out of range: {e}") from None
    if ws is None:
        with _taken_on(stream):
            ws = shared_workspace(q, pool, group_off, prefix_table, own_table)
    handle = pool._on(stream)
    if handle not in ws._seen:
        ws._see(handle, stream)
    B._check(B.load().cr_attn_shared(pool._ref, a, *ws.args, handle), "cr_attn_shared")
    return out
