"""A destination's serving operators on the device: a paged cache of keys and values, the calls
that take, share, move and free its pages, attention over whole prompts (a miss) and attention
of requests that share a cached prefix (a hit, and every decoded token). The cache holds 16-bit
elements or 8-bit floats with scales, and queries and keys are turned by their positions before they go in.
Marshalling only; the library does the work.

    pool = PagePool(k, v, refs)                       # k, v [layers, pages, heads, tokens, dim]
    pool.extend(table, None, length)                  # pages for new sequences
    attend_prompt(q, k, v, off, off, scale, out=o)    # a miss: the whole prompt ...
    pool.append(0, k, v, off, length, table)          # ... whose keys and values are kept
    pool.fork(table, parent, length, child)           # a request behind a cached prefix
    attend_shared(q, pool, 0, q_off, group_off, table, length, own_table, own_len, scale, out=o)
    pool.free(table, length)                          # an eviction

    pool = QuantPagePool.empty(layers, pages, heads, tokens, dim)   # the same calls on a cache in 8 bits
    pool.read(0, k, v, off, length, table)            # its tokens as 16-bit rows
    rotary = Rotary(dim, base=500000.0)               # positions ...
    rotary.apply(q, k, positions, q_out=q, k_out=k)   # ... of a step's queries and new keys

Tensors are on the GPU. Offsets, lengths and page tables are int32; a call enqueues kernels on
``stream`` (default: the current one) and returns. Problems that only the device sees set bits
of ``pool.err``, of the workspace's ``err`` or of an ``err`` given (``CR_ERR_*``), and the sequence
concerned is skipped as the library documents. Nothing here is differentiable: tensors that require
a gradient are refused where gradients are recorded.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct
from typing import Optional, Sequence

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.CR_BF16, torch.float16: B.CR_F16}
_CODES = {torch.float8_e4m3fn: B.CR_E4M3, torch.float8_e5m2: B.CR_E5M2}
_LAYOUTS = {"half": B.CR_ROTARY_HALF, "pairs": B.CR_ROTARY_PAIRS}
_INT32, _FLOAT32 = torch.int32, torch.float32
_HERE = contextlib.nullcontext()
_raw_stream, _device = B._raw_stream, B._device
_pack_rows, _pack_prompt, _pack_shared, _RANGE = B.ROWS.pack, B.PROMPT_ARGS.pack, B.SHARED_ARGS.pack, (struct.error, OverflowError)
_pack_rotary, _pack_tokens = B.ROTARY_ARGS.pack, B.TOKENS_ARGS.pack


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


def _on_device(self, stream) -> Optional[int]:
    """As _Memory's _on, for memory of one device: the call's launches go to the current one."""
    device = _device()
    if device != self._device:
        raise B.CrError(f"made on cuda:{self._device}, the current device is cuda:{device}")
    handle = _raw_stream(device) if stream is None and _raw_stream else B._stream(stream)
    if handle not in self._seen:
        self._see(handle, stream)
    return handle


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
        strides = self._take(k, v, refs, order)
        self.dtype = k.dtype
        self.c = B.CrKvCache(_dtype(k), self.heads, self.dim, self.page_tokens, self.num_pages, self.layers, k.data_ptr(),
                             v.data_ptr(), *strides, _index(refs, self.num_pages))
        self._ready("cr_pages_", "cr_kv_append", "cr_attn_shared")

    def _take(self, k, v, refs, order):
        """The tensors, and their strides of layers, pages, heads and tokens."""
        if order not in ("head", "token"):
            raise ValueError(f"unknown order {order!r}")
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(4) != 1:
            raise B.CrError("k and v are five-dimensional alike, with dim contiguous")
        if not (k.is_cuda and v.is_cuda):
            raise B.CrError("libcr takes device tensors")
        h, t = (2, 3) if order == "head" else (3, 2)
        self.k, self.v, self.refs, self.order = k, v, refs, order
        self.layers, self.num_pages, self.heads, self.page_tokens, self.dim = k.shape[0], k.shape[1], k.shape[h], k.shape[t], k.shape[4]
        return k.stride(0), k.stride(1), k.stride(h), k.stride(t)

    def _ready(self, pages: str, append: str, attn: str, *held):
        """The library's calls for this cache, and the memory that they use."""
        L = B.load()
        self._extend, self._fork, self._free, self._compact, self._copy = (getattr(L, pages + x) for x in ("extend", "fork", "free", "compact", "copy"))
        self._append, self._attn, self._attn_bytes = getattr(L, append), getattr(L, attn), getattr(B, attn + "_workspace_bytes")
        self.err = torch.zeros(1, dtype=torch.int32, device=self.k.device)
        self._ref, self._err = ctypes.byref(self.c), _index(self.err)
        self._ws = torch.empty(B.cr_pages_workspace_bytes(self.num_pages, 0), dtype=torch.uint8, device=self.k.device)
        self._ws_for = 0  # sequences that it is known to be large enough for
        _Memory.__init__(self, self.k, self.v, self.refs, self.err, self._ws, *held)

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
        B._check(self._extend(self._ref, old, new, n, p, width, *self._scratch(n, stream)), self._extend.__name__)

    def fork(self, table, parent, length, child, stream=None):
        """child[i]: the first length[i] tokens of table[parent[i]], the partial tail copied."""
        n, rows = parent.numel(), table.shape[0]
        (p, width), (c, child_width) = _table(table, rows), _table(child, n)
        B._check(self._fork(self._ref, p, rows, width, _index(parent), _index(length, n), n, c, child_width,
                                        *self._scratch(n, stream)), self._fork.__name__)

    def free(self, table, length, stream=None):
        """Gives the pages of every row's first length tokens back."""
        n = length.numel()
        p, width = _table(table, n)
        B._check(self._free(self._ref, p, width, _index(length), n, self._err, self._on(stream)), self._free.__name__)

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
        B._check(self._compact(self._ref, p, lengths, rows, width, out, refs, *self._scratch(0, stream)), self._compact.__name__)

    def copy(self, src, dst, stream=None):
        """Contents of page src[i] to page dst[i], all layers."""
        n = src.numel()
        B._check(self._copy(self._ref, _index(src), _index(dst, n), n, self._err, self._on(stream)), self._copy.__name__)

    def append(self, layer: int, k, v, off, length, table, stream=None):
        """Rows off[i]..off[i+1] of k and v ([total, heads, dim]) become the last tokens of the
        length[i] of sequence i."""
        shape, n, dtype = k.shape, length.numel(), self.dtype
        if len(shape) != 3 or shape[1] != self.heads or shape[2] != self.dim or shape != v.shape or k.dtype is not dtype or v.dtype is not dtype:
            raise B.CrError("new keys and values have the cache's heads, dim and type")
        if (k.requires_grad or v.requires_grad) and _grad_on():
            _refuse_grad()
        p, width = _table(table, n)
        B._check(self._append(self._ref, layer, _pack_rows(*_rows(k)), _pack_rows(*_rows(v)), shape[0],
                                       _index(off, n + 1), _index(length), n, p, width, self._err, self._on(stream)), self._append.__name__)


class QuantPagePool(PagePool):
    """Handle of a paged cache in 8 bits. ``k``, ``v``: as a PagePool's, float8_e4m3fn or float8_e5m2; ``scale``: uint8
    [layers, pages, heads, page tokens / block tokens, 2], of each block of tokens the exponent + 127 of the power of two
    that its keys' codes, and its values', are multiplied with (1 to 254; a scale of 127 is 1); ``dtype``: the type of queries, new keys and values and outputs.
    All of PagePool's calls and ``attend_shared`` work on it: ``append`` rounds into it, with a block's scale chosen by
    its largest element."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, scale: torch.Tensor, refs: torch.Tensor, dtype=torch.bfloat16, order: str = "head"):
        strides = self._take(k, v, refs, order)
        if k.dtype not in _CODES:
            raise B.CrError(f"float8_e4m3fn or float8_e5m2 wanted, not {k.dtype}")
        if dtype not in _DTYPES:
            raise B.CrError(f"bfloat16 or float16 wanted, not {dtype}")
        blocks = scale.shape[3] if scale.dim() == 5 else 0
        if scale.dtype is not torch.uint8 or blocks == 0 or scale.shape != (self.layers, self.num_pages, self.heads, blocks, 2) or \
                self.page_tokens % blocks or not scale.is_contiguous():
            raise B.CrError("scale is uint8 [layers, pages, heads, page tokens / block tokens, 2], contiguous")
        if not (k.device == v.device == scale.device == refs.device):
            raise B.CrError("codes, scales and refs are on one device")
        self.scale, self.dtype, self.block_tokens = scale, dtype, self.page_tokens // blocks
        self.c = B.CrKvqCache(_DTYPES[dtype], _CODES[k.dtype], self.heads, self.dim, self.page_tokens, self.block_tokens, self.num_pages,
                              self.layers, k.data_ptr(), v.data_ptr(), *strides, scale.data_ptr(), _index(refs, self.num_pages))
        self._device = k.device.index
        self._ready("cr_kvq_", "cr_kvq_append", "cr_kvq_attn", scale)
        self._read = B.load().cr_kvq_read
        self._head = torch.Size((self.heads, self.dim))

    @classmethod
    def empty(cls, layers: int, num_pages: int, heads: int, page_tokens: int, dim: int, dtype=torch.bfloat16, device="cuda",
              order: str = "head", codes=torch.float8_e4m3fn, block_tokens: Optional[int] = None) -> "QuantPagePool":
        """A new cache, all pages free; blocks of 16 tokens (or of a page, if that is smaller) unless given."""
        block = min(16, page_tokens) if block_tokens is None else block_tokens
        if block < 1 or page_tokens % block:
            raise B.CrError(f"a page of {page_tokens} tokens is not whole blocks of {block}")
        shape = (layers, num_pages) + ((heads, page_tokens) if order == "head" else (page_tokens, heads)) + (dim,)
        k, v = (torch.empty(shape, dtype=torch.uint8, device=device).view(codes) for _ in range(2))
        scale = torch.full((layers, num_pages, heads, page_tokens // block, 2), 127, dtype=torch.uint8, device=device)
        return cls(k, v, scale, torch.zeros(num_pages, dtype=torch.int32, device=device), dtype, order)

    _on = _on_device

    def _tokens(self, layer, k, v, off, length, table):
        """A cr_kvq_tokens of rows [total, heads, dim] of both."""
        shape, sk, sv, dtype = k.shape, k.stride(), v.stride(), self.dtype
        if k.dtype is not dtype or v.dtype is not dtype or shape != v.shape or shape[1:] != self._head or sk[2] != 1 or sv[2] != 1:
            raise B.CrError("rows of keys and values have the cache's heads, dim and type, with dim contiguous")
        if not (k.is_cuda and v.is_cuda):
            raise B.CrError("libcr takes device tensors")
        if (k.requires_grad or v.requires_grad) and _grad_on():
            _refuse_grad()
        n = length.numel()
        p, width = _table(table, n)
        try:
            return _pack_tokens(layer, shape[0], n, width, k.data_ptr(), sk[0], sk[1], v.data_ptr(), sv[0], sv[1], _index(off, n + 1), _index(length), p)
        except _RANGE as e:
            raise B.CrError(f"an argument is out of range: {e}") from None

    def append(self, layer: int, k, v, off, length, table, stream=None):
        """Rows off[i]..off[i+1] of k and v ([total, heads, dim]) are rounded into the last tokens of the
        length[i] of sequence i."""
        rc = self._append(self._ref, self._tokens(layer, k, v, off, length, table), self._err, self._on(stream))
        if rc:
            B._check(rc, "cr_kvq_append")

    def read(self, layer: int, k, v, off, length, table, stream=None):
        """The reverse of ``append``: the last tokens of the length[i] of sequence i into rows off[i]..off[i+1] of k and
        v ([total, heads, dim], the cache's dtype, apart from each other; either may be None)."""
        if k is None and v is None:
            raise B.CrError("rows of keys or of values are wanted")
        t = self._tokens(layer, v if k is None else k, k if v is None else v, off, length, table)
        if k is None or v is None:  # the other one's rows have no place
            f = list(B.TOKENS_ARGS.unpack(t))
            f[4 if k is None else 7] = 0
            t = _pack_tokens(*f)
        rc = self._read(self._ref, t, self._err, self._on(stream))
        if rc:
            B._check(rc, "cr_kvq_read")


def rotary_frequencies(rotated: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, length: Optional[int] = None,
                       low: float = 1.0, high: float = 4.0) -> list:
    """Radians per position of each pair i of ``rotated`` / 2: f_i = base^(-2i / rotated), for contexts that are
    ``factor`` times as long as trained with ``scaling``

    * "linear": f_i / factor;
    * "base": base becomes base * factor^(rotated / (rotated - 2)), which divides the last frequency by the factor and keeps the first;
    * "turns": frequencies that make ``high`` turns or more over ``length`` tokens stay, those of ``low`` or fewer are
      divided by the factor, between them the share that stays goes by the turns;
    * "index": the same with the share falling from pair to pair between the two that would make ``high`` and
      ``low`` turns, rounded outwards.
    """
    if scaling not in (None, "linear", "base", "turns", "index"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if rotated < 2 or rotated % 2:
        raise B.CrError(f"pairs of elements turn, not {rotated}")
    by_turns = scaling in ("turns", "index")
    try:
        base, factor = float(base), float(factor)
        if by_turns and length is not None:
            length, low, high = float(length), float(low), float(high)
    except OverflowError:
        raise B.CrError("an argument passes a float's range") from None
    if not (1.0 < base < math.inf and 0.0 < factor < math.inf):
        raise B.CrError("base is above 1 and factor above 0, both finite")
    if by_turns and not (length is not None and 0.0 < length < math.inf and 0.0 < low < high < math.inf):
        raise B.CrError("this scaling goes by the turns over `length` tokens, 0 < low < high, all finite")
    try:
        f = _frequencies(rotated, base, scaling, factor, length, low, high)
    except OverflowError:
        f = [math.inf]
    if not all(math.isfinite(x) for x in f):
        raise B.CrError("frequencies pass a float's range")
    return f


def _frequencies(rotated, base, scaling, factor, length, low, high):
    if scaling == "base":
        if rotated == 2:
            raise B.CrError("one pair alone has no other base")
        try:
            base *= factor ** (rotated / (rotated - 2))
        except OverflowError:
            base = math.inf
        if not 0.0 < base < math.inf:
            raise B.CrError("base and factor pass a float's range")
    f = [base ** (-2.0 * i / rotated) for i in range(rotated // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling in (None, "base"):
        return f
    if scaling == "turns":
        stay = [(length * x / (2.0 * math.pi) - low) / (high - low) for x in f]
    else:
        def pair(turns):
            over = length / (2.0 * math.pi * turns)
            log = math.log(over) if 0.0 < over < math.inf else math.log(length) - math.log(2.0 * math.pi) - math.log(turns)
            return rotated * log / (2.0 * math.log(base))

        a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotated - 1)
        stay = [1.0 - (i - a) / max(b - a, 0.001) for i in range(len(f))]
    stay = [min(1.0, max(0.0, s)) for s in stay]
    return [x * ((1.0 - s) / factor + s) for x, s in zip(f, stay)]


def _float(x) -> float:
    """x, or infinity where it is a whole number beyond a float's range."""
    try:
        return float(x)
    except OverflowError:
        return math.inf


class Rotary(_Memory):
    """Rotary positions for heads of ``dim``: the first ``rotated`` elements (all, if not given) turn, pairs being elements i and
    i + rotated / 2 (``layout`` "half") or 2i and 2i + 1 ("pairs"). Frequencies are rotary_frequencies(...) or given
    (radians per position, one a pair); what turns is also multiplied with ``magnitude``. Far positions lose nothing: angles are exact
    fractions of a turn."""

    def __init__(self, dim: int, rotated: Optional[int] = None, *, base: float = 10000.0, layout: str = "half", scaling: Optional[str] = None,
                 factor: float = 1.0, length: Optional[int] = None, low: float = 1.0, high: float = 4.0, magnitude: float = 1.0,
                 frequencies: Optional[Sequence[float]] = None, device="cuda"):
        if layout not in _LAYOUTS:
            raise ValueError(f"unknown layout {layout!r}")
        self.dim, self.rotated, self.layout, self.magnitude = dim, dim if rotated is None else rotated, layout, _float(magnitude)
        if dim not in (64, 128) or self.rotated not in range(16, dim + 1, 16):
            raise B.CrError("heads are of 64 or 128 elements, of which a multiple of 16 turns")
        if not abs(self.magnitude) <= 3.4e38:
            raise B.CrError("magnitude is finite")
        if frequencies is None:
            frequencies = rotary_frequencies(self.rotated, base, scaling, factor, length, low, high)
        self.frequencies = [_float(f) for f in frequencies]
        if len(self.frequencies) != self.rotated // 2 or not all(math.isfinite(f) for f in self.frequencies):
            raise B.CrError(f"{self.rotated // 2} finite frequencies wanted")
        if any(abs(f) >= 2.0 ** 900 for f in self.frequencies):
            raise B.CrError("frequencies pass a float's range as fractions of a turn")
        turns = [int(round(f / (2.0 * math.pi) * 2.0 ** 64)) % (1 << 64) for f in self.frequencies]  # of 2^64 a turn
        self.freq = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64).to(device)
        if not self.freq.is_cuda:
            raise B.CrError("libcr takes device tensors")
        self._device, self._code = self.freq.device.index, _LAYOUTS[layout]
        self._freq, self._call = self.freq.data_ptr(), B.load().cr_rotary
        super().__init__(self.freq)

    _on = _on_device

    def apply(self, q, k, positions, q_out=None, k_out=None, stream=None):
        """q [tokens, heads, dim] and k [tokens, key heads, dim] (or None) turned by ``positions`` (int32 [tokens]; negative ones
        turn back) into q_out and k_out, new tensors if not given; q and k themselves may be given, other tensors must not overlap
        q or k, nor the two each other (one tensor as q and as k is not turned in place). Returns both."""
        shape, dtype, dim = q.shape, q.dtype, self.dim
        code = _DTYPES.get(dtype)
        if code is None:
            _dtype(q)
        if len(shape) != 3 or shape[2] != dim:
            raise B.CrError("rows are [tokens, heads, dim] with the dim of this handle")
        if q_out is None:
            q_out = _new_out(q, stream)
        elif q_out.shape != shape or q_out.dtype is not dtype:
            raise B.CrError("q_out has q's shape and type")
        if k is None:
            if k_out is not None:
                raise B.CrError("there are no keys to turn")
            heads_k, keys, keys_out = 0, (0, 0, 0), (0, 0, 0)
        else:
            key_shape = k.shape
            if len(key_shape) != 3 or key_shape[0] != shape[0] or key_shape[2] != dim or k.dtype is not dtype:
                raise B.CrError("k has q's tokens, dim and type")
            if k_out is None:
                k_out = _new_out(k, stream)
            elif k_out.shape != key_shape or k_out.dtype is not dtype:
                raise B.CrError("k_out has k's shape and type")
            if k.requires_grad and _grad_on():
                _refuse_grad()
            heads_k, keys = key_shape[1], _rows(k)
            keys_out = keys if k_out is k else _rows(k_out)
        if q.requires_grad and _grad_on():
            _refuse_grad()
        queries = _rows(q)
        try:
            a = _pack_rotary(code, shape[1], heads_k, dim, self.rotated, self._code, shape[0], self.magnitude, *queries, *keys,
                             *(queries if q_out is q else _rows(q_out)), *keys_out, _index(positions, shape[0]), self._freq)
        except _RANGE as e:
            raise B.CrError(f"an argument is out of range: {e}") from None
        rc = self._call(a, self._on(stream))
        if rc:
            B._check(rc, "cr_rotary")
        return q_out, k_out


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
    return Workspace(pool._attn_bytes(pool.c, a), q.device, pool.err if err is None else err)


def attend_shared(q, pool: PagePool, layer: int, q_off, group_off, prefix_table, prefix_len, own_table, own_len,
                  scale: float, *, out=None, lse=None, ws: Optional[Workspace] = None, stream=None):
    """Attention of requests in groups that share a cached prefix: requests group_off[g] ..
    group_off[g+1] see the prefix_len[g] tokens of prefix_table[g] and, causally, their own
    own_len[r] tokens of own_table[r], the last of which are the queries' (append them first).
    q [total_q, heads_q, dim], request r's at q_off[r]..q_off[r+1]. Returns out. Tables about as
    wide as their longest row keep the GPU busy: the widths stand for the lengths, which only the
    device knows."""
    shape = q.shape
    if q.dtype is not pool.dtype or len(shape) != 3 or shape[2] != pool.dim:
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
    B._check(pool._attn(pool._ref, a, *ws.args, handle), pool._attn.__name__)
    return out
