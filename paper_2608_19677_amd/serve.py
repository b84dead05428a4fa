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
of ``pool.err`` or of the workspace's ``err`` (``CR_ERR_*``), and the sequence concerned is
skipped as the library documents.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.CR_BF16, torch.float16: B.CR_F16}


def _dtype(t: torch.Tensor) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise B.CrError(f"bfloat16 or float16 wanted, not {t.dtype}") from None


def _rows(t: torch.Tensor):
    """Fields of a cr_rows: [tokens, heads, dim] with any strides of tokens and heads."""
    stride = t.stride()
    if len(stride) != 3 or stride[2] != 1:
        raise B.CrError("rows are [tokens, heads, dim] with dim contiguous")
    if not t.is_cuda:
        raise B.CrError("libcr takes device tensors")
    return t.data_ptr(), stride[0], stride[1]


def _int32(t: Optional[torch.Tensor], n: Optional[int] = None):
    """An int32 array of n elements (any, if n is None), or None."""
    if t is not None:
        if t.dtype is not torch.int32:
            raise B.CrError(f"offsets, lengths and tables are int32, not {t.dtype}")
        if n is not None and t.numel() != n:
            raise B.CrError(f"{n} entries wanted, not {t.numel()}")
    return t


def _index(t: torch.Tensor, n: Optional[int] = None) -> int:
    """Pointer of such an array."""
    return B._ptr(_int32(t, n))


def _used_on(stream, *tensors):
    """Memory taken here from the current stream's pool and used on another stream."""
    if stream is not None:
        for t in tensors:
            t.record_stream(stream)


class Workspace:
    """Device scratch of an attention call and its error word."""

    def __init__(self, nbytes: int, device, err: Optional[torch.Tensor] = None):
        self.buf = torch.empty(max(16, nbytes), dtype=torch.uint8, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device) if err is None else err


class PagePool:
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
        self._ws: Optional[torch.Tensor] = None

    @classmethod
    def empty(cls, layers: int, num_pages: int, heads: int, page_tokens: int, dim: int, dtype=torch.bfloat16, device="cuda",
              order: str = "head") -> "PagePool":
        """A new cache, all pages free."""
        shape = (layers, num_pages) + ((heads, page_tokens) if order == "head" else (page_tokens, heads)) + (dim,)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device),
                   torch.zeros(num_pages, dtype=torch.int32, device=device), order)

    def _scratch(self, n: int, stream) -> torch.Tensor:
        """The page calls' workspace, kept with the handle: its calls are for one stream at a time."""
        need = B.cr_pages_workspace_bytes(self.num_pages, n)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.k.device)
        _used_on(stream, self._ws)
        return self._ws

    def pages_of(self, tokens: int) -> int:
        return -(-tokens // self.page_tokens)

    def extend(self, table, len_old, len_new, stream=None):
        """Free pages for sequences that grow from len_old (None: 0) to len_new tokens."""
        n = len_new.numel()
        _int32(len_new), _int32(table), _int32(len_old, n)
        _same_rows(table, n)
        B.cr_pages_extend(self.c, len_old, len_new, table, self._scratch(n, stream), self.err, stream)

    def fork(self, table, parent, length, child, stream=None):
        """child[i]: the first length[i] tokens of table[parent[i]], the partial tail copied."""
        n = parent.numel()
        _int32(table), _int32(parent), _int32(length, n), _int32(child)
        _same_rows(table, table.shape[0])
        _same_rows(child, n)
        B.cr_pages_fork(self.c, table, parent, length, child, self._scratch(n, stream), self.err, stream)

    def free(self, table, length, stream=None):
        """Gives the pages of every row's first length tokens back."""
        _int32(table), _int32(length)
        _same_rows(table, length.numel())
        B.cr_pages_free(self.c, table, length, self.err, stream)

    def compact(self, table, length, table_out=None, refs_out=None, stream=None):
        """Moves the live pages to the front and renames the table's entries (in place, if no
        other place is given)."""
        table_out, refs_out = (table if table_out is None else table_out), (self.refs if refs_out is None else refs_out)
        _int32(table), _int32(length), _int32(refs_out, self.num_pages)
        if table is not None:
            _int32(table_out, table.numel())
            _same_rows(table, length.numel())
        B.cr_pages_compact(self.c, table, length, table_out, refs_out, self._scratch(0, stream), self.err, stream)

    def copy(self, src, dst, stream=None):
        """Contents of page src[i] to page dst[i], all layers."""
        _int32(src), _int32(dst, src.numel())
        B.cr_pages_copy(self.c, src, dst, self.err, stream)

    def append(self, layer: int, k, v, off, length, table, stream=None):
        """Rows off[i]..off[i+1] of k and v ([total, heads, dim]) become the last tokens of the
        length[i] of sequence i."""
        if k.shape != v.shape or k.shape[1:] != (self.heads, self.dim) or k.dtype != self.k.dtype or v.dtype != self.k.dtype:
            raise B.CrError("new keys and values have the cache's heads, dim and type")
        _int32(length), _int32(off, length.numel() + 1), _int32(table)
        _same_rows(table, length.numel())
        B.cr_kv_append(self.c, layer, B.CrRows(*_rows(k)), B.CrRows(*_rows(v)), k.shape[0], off, length, table, self.err, stream)


def _same_rows(table, n: int):
    if table.dim() != 2 or table.shape[0] != n:
        raise B.CrError(f"a table is [{n}, width], not {list(table.shape)}")


def _check_out(q, out, lse):
    if out.shape != q.shape or out.dtype != q.dtype:
        raise B.CrError("out has q's shape and type")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != q.shape[:2]):
        raise B.CrError("lse is float32 [tokens, heads]")


def _prompt_args(dtype, q, k, batch, scale, causal, *rest) -> B.CrAttnPromptArgs:
    nq, hq, d = q.shape
    return B.CrAttnPromptArgs(dtype, hq, k.shape[1], d, batch, causal, nq, k.shape[0], scale, *rest)


def prompt_workspace(q, k, q_off, err: Optional[torch.Tensor] = None) -> Workspace:
    """Scratch for ``attend_prompt`` of tensors of these shapes."""
    return Workspace(B.cr_attn_prompt_workspace_bytes(_prompt_args(_dtype(q), q, k, q_off.numel() - 1, 1.0, True)), q.device, err)


def attend_prompt(q, k, v, q_off, k_off, scale: float, *, out=None, lse=None, causal: bool = True,
                  ws: Optional[Workspace] = None, stream=None):
    """Attention of packed sequences: q [total_q, heads_q, dim], k, v [total_k, heads_kv, dim],
    sequence b at q_off[b]..q_off[b+1] and k_off[b]..k_off[b+1]. Returns out (and fills lse,
    float32 [total_q, heads_q], if given)."""
    if k.shape != v.shape or k.shape[2] != q.shape[2] or k.dtype != q.dtype or v.dtype != q.dtype:
        raise B.CrError("q, k and v have one type and dim, k and v one shape")
    dtype = _dtype(q)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        _used_on(stream, out)
    _check_out(q, out, lse)
    n = q_off.numel()
    a = _prompt_args(dtype, q, k, n - 1, scale, causal, _rows(q), _rows(k), _rows(v), _rows(out), B._ptr(lse), _index(q_off),
                     _index(k_off, n))
    if ws is None:
        ws = prompt_workspace(q, k, q_off)
        _used_on(stream, ws.buf, ws.err)
    B.cr_attn_prompt(a, ws.buf, ws.err, stream)
    return out


def _shared_args(q, pool: PagePool, layer, groups, prefix_table, own_table, scale, *rest) -> B.CrAttnSharedArgs:
    batch, own_width = own_table.shape
    return B.CrAttnSharedArgs(q.shape[1], layer, batch, groups, q.shape[0], prefix_table.shape[1], own_width, scale, *rest)


def shared_workspace(q, pool: PagePool, group_off, prefix_table, own_table, err: Optional[torch.Tensor] = None) -> Workspace:
    """Scratch for ``attend_shared`` of tensors of these shapes."""
    a = _shared_args(q, pool, 0, group_off.numel() - 1, prefix_table, own_table, 1.0)
    return Workspace(B.cr_attn_shared_workspace_bytes(pool.c, a), q.device, pool.err if err is None else err)


def attend_shared(q, pool: PagePool, layer: int, q_off, group_off, prefix_table, prefix_len, own_table, own_len,
                  scale: float, *, out=None, lse=None, ws: Optional[Workspace] = None, stream=None):
    """Attention of requests in groups that share a cached prefix: requests group_off[g] ..
    group_off[g+1] see the prefix_len[g] tokens of prefix_table[g] and, causally, their own
    own_len[r] tokens of own_table[r], the last of which are the queries' (append them first).
    q [total_q, heads_q, dim], request r's at q_off[r]..q_off[r+1]. Returns out."""
    if q.dtype != pool.k.dtype or q.dim() != 3 or q.shape[2] != pool.dim:
        raise B.CrError("q has the cache's type and dim")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        _used_on(stream, out)
    _check_out(q, out, lse)
    batch, groups = own_table.shape[0], group_off.numel() - 1
    _same_rows(own_table, batch)
    _same_rows(prefix_table, groups)
    a = _shared_args(q, pool, layer, groups, prefix_table, own_table, scale, _rows(q), _rows(out), B._ptr(lse),
                     _index(q_off, batch + 1), _index(group_off), _index(prefix_table), _index(prefix_len, groups),
                     _index(own_table), _index(own_len, batch))
    if ws is None:
        ws = shared_workspace(q, pool, group_off, prefix_table, own_table)
        _used_on(stream, ws.buf)
    B.cr_attn_shared(pool.c, a, ws.buf, ws.err, stream)
    return out
