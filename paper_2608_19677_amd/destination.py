"""One destination of a routed stream, run for real: the requests that a plan sends to it go through a
paged cache of W whole prefixes with the serving operators, where the replay only counts them
(Section 3.2: admitted and cold prefixes share each destination's cache, least recent out).

A batch of requests in arrival order:

* a key that is not cached (a miss) takes pages for its prefix, runs prompt attention over it and
  keeps its keys and values; the least recent prefix beyond W goes when the batch is done;
* every request appends its suffix behind the cached prefix and attends to both, the requests of
  one prefix sharing the pass over it; ``samples`` continuations of each are forked from it and
  decode one token;
* the requests' own pages are freed again.

The cache holds 16-bit elements, or 8-bit floats (``codes``: twice the prefixes in the same memory); with ``rotary``
queries and keys are turned by their positions, a request's following its prefix's.

Keys and values come from ``project`` (a model's layer; here a seeded stand-in). The hits and
prefill tokens counted on the way are the replay's statistics of that destination.

  python -m paper_2608_19677_amd.destination [--requests N] [--batch B] [--codes e4m3] [--rotary]
"""
from __future__ import annotations

import argparse
import math
import time
from collections import OrderedDict
from dataclasses import dataclass
from typing import List, Optional

import numpy as np
import torch

from . import binding as B
from . import serve


class Projection:
    """Stand-in for a model's query, key and value projections: values of a prefix depend on its
    key alone, those of other tokens on the request."""

    def __init__(self, heads_q: int, heads_kv: int, dim: int, dtype, device):
        self.heads_q, self.heads_kv, self.dim, self.dtype, self.device = heads_q, heads_kv, dim, dtype, device

    def __call__(self, layer: int, ids, lengths):
        """q, k, v of packed sequences, sequence i with lengths[i] tokens seeded by ids[i]."""
        parts = []
        for i, n in zip(ids, lengths):
            g = torch.Generator(device=self.device).manual_seed(int(i) * 1024 + layer)
            parts.append(torch.randn((int(n), self.heads_q + 2 * self.heads_kv, self.dim), generator=g, device=self.device))
        x = torch.cat(parts).to(self.dtype)
        return x[:, :self.heads_q], x[:, self.heads_q:-self.heads_kv], x[:, -self.heads_kv:]


@dataclass
class Counts:
    """The replay's statistics of a destination."""
    requests: int = 0
    hits: int = 0
    prefill: int = 0
    hit_prefix: int = 0


class Destination:
    """A cache of W prefixes of up to max_prefix tokens and the operators around it."""

    def __init__(self, W: int, max_prefix: int, max_suffix: int, batch: int, *, layers: int = 1, heads_q: int = 64,
                 heads_kv: int = 8, dim: int = 128, page_tokens: int = 16, samples: int = 0, dtype=torch.bfloat16,
                 device="cuda", project=None, codes: Optional[torch.dtype] = None, rotary: Optional[serve.Rotary] = None):
        self.W, self.batch, self.layers, self.samples, self.device = W, batch, layers, samples, device
        self.scale = 1.0 / math.sqrt(dim)
        up = lambda n: -(-n // page_tokens)  # noqa: E731
        self.width, self.own_width = up(max_prefix), up(max_suffix + 1)
        rows = W + batch  # prefixes of a batch stay until it is done
        pages = rows * self.width + batch * (1 + samples) * self.own_width
        self.rotary = rotary
        if codes is None:
            self.pool = serve.PagePool.empty(layers, pages, heads_kv, page_tokens, dim, dtype, device)
        else:
            self.pool = serve.QuantPagePool.empty(layers, pages, heads_kv, page_tokens, dim, dtype, device, codes=codes)
        self.table = torch.full((rows, self.width), -1, dtype=torch.int32, device=device)
        self.rows: List[int] = list(range(rows))       # free rows of the table
        self.length = np.zeros(rows, dtype=np.int64)   # tokens of each row's prefix
        self.slots: "OrderedDict[int, int]" = OrderedDict()  # key -> row, least recent first
        self.project = project or Projection(heads_q, heads_kv, dim, dtype, device)
        self.counts = Counts()
        self.prefilled = None  # the last batch's misses: keys, offsets, outputs of the last layer

    def _i32(self, v):
        return torch.tensor(np.asarray(v, dtype=np.int32), device=self.device)

    @staticmethod
    def _off(lengths):
        return np.concatenate([[0], np.cumsum(lengths)])

    def serve(self, keys, prefix_len, suffix_len, first_id: int = 0):
        """A batch of requests in arrival order: their keys, prefix lengths and suffix lengths. Returns
        per request whether its prefix was cached, and the attention outputs of the last layer:
        [tokens, heads, dim] of the suffixes packed in the order of ``order`` with the offsets, and,
        with ``samples``, of one decoded token per continuation. Raises where a call of the batch reported a
        problem (bits of ``pool.err``)."""
        assert 0 < len(keys) <= self.batch
        hit, row, missed, gone = [], [], [], []
        for k, n in zip(keys, prefix_len):
            k = int(k)
            if k in self.slots:
                self.slots.move_to_end(k)
                self.counts.hits += 1
                self.counts.hit_prefix += int(n)
                hit.append(True)
            else:
                r = self.rows.pop()
                self.length[r] = int(n)
                self.slots[k] = r
                missed.append((k, r))
                self.counts.prefill += int(n)
                hit.append(False)
                if len(self.slots) > self.W:
                    gone.append(self.slots.popitem(last=False)[1])
            row.append(self.slots[k])
        self.counts.requests += len(keys)
        self.counts.prefill += int(np.sum(suffix_len, dtype=np.int64))
        self.prefilled = None
        if missed:
            self._prefill(missed)
        order = np.argsort(np.asarray(row), kind="stable")  # requests of one prefix side by side
        out = self._attend(np.asarray(row)[order], np.asarray(suffix_len)[order], first_id + order)
        for r in gone:
            self.pool.free(self.table[r:r + 1], self._i32([self.length[r]]))
            self.rows.append(r)
        self._check()
        return hit, order, out

    def _positions(self, first, lengths):
        """Positions of packed tokens, lengths[i] of them from first[i] on; None without rotary."""
        if self.rotary is None:
            return None
        return self._i32(np.concatenate([np.arange(n) + a for a, n in zip(first, lengths)]))

    def _project(self, layer, ids, lengths, positions):
        q, k, v = self.project(layer, ids, lengths)
        if positions is not None:
            q, k = self.rotary.apply(q, k, positions)
        return q, k, v

    def _check(self):
        bits = int(self.pool.err.item())
        if bits:
            raise B.CrError(f"a call on the cache reported {bits:#x}")

    def _prefill(self, missed):
        rows = torch.tensor([r for _, r in missed], device=self.device)
        lengths = self.length[[r for _, r in missed]]
        table = torch.full((len(missed), self.width), -1, dtype=torch.int32, device=self.device)
        n, off = self._i32(lengths), self._i32(self._off(lengths))
        self.pool.extend(table, None, n)
        out, pos = None, self._positions(np.zeros(len(lengths), dtype=np.int64), lengths)
        for layer in range(self.layers):
            q, k, v = self._project(layer, [key for key, _ in missed], lengths, pos)
            out = serve.attend_prompt(q, k, v, off, off, self.scale, err=self.pool.err)
            self.pool.append(layer, k, v, off, n, table)
        self.table[rows] = table
        self.prefilled = [key for key, _ in missed], off, out

    def _attend(self, row, suffix, ids):
        starts = np.flatnonzero(np.concatenate([[True], row[1:] != row[:-1]]))
        groups = self._i32(np.concatenate([starts, [len(row)]]))
        prefixes, plen = self.table[torch.from_numpy(row[starts]).to(self.device)], self._i32(self.length[row[starts]])
        own = torch.full((len(row), self.own_width), -1, dtype=torch.int32, device=self.device)
        n, off = self._i32(suffix), self._i32(self._off(suffix))
        self.pool.extend(own, None, n)
        out = decoded = None
        before = self.length[row]  # tokens of each request's prefix
        pos = self._positions(before, suffix)
        for layer in range(self.layers):
            q, k, v = self._project(layer, [1 << 40 | int(i) for i in ids], suffix, pos)
            self.pool.append(layer, k, v, off, n, own)
            out = serve.attend_shared(q, self.pool, layer, off, groups, prefixes, plen, own, n, self.scale)
        if self.samples:
            decoded = self._decode(starts, prefixes, plen, own, n, suffix, ids, before + suffix)
        self.pool.free(own, n)
        return out, off, decoded

    def _decode(self, starts, prefixes, plen, own, n, suffix, ids, at):
        """One token of ``samples`` continuations of every request, at position at[r]."""
        s = self.samples
        parent, length = self._i32(np.repeat(np.arange(len(suffix)), s)), self._i32(np.repeat(suffix, s))
        child = torch.empty((len(suffix) * s, self.own_width), dtype=torch.int32, device=self.device)
        self.pool.fork(own, parent, length, child)
        self.pool.extend(child, length, length + 1)
        ones = self._i32(np.arange(len(suffix) * s + 1))
        groups = self._i32(np.concatenate([starts, [len(suffix)]]) * s)
        one = np.ones(len(suffix) * s, dtype=np.int64)
        out, pos = None, self._positions(np.repeat(at, s), one)
        for layer in range(self.layers):
            q, k, v = self._project(layer, [2 << 40 | int(i) * s + j for i in ids for j in range(s)], one, pos)
            self.pool.append(layer, k, v, ones, length + 1, child)
            out = serve.attend_shared(q, self.pool, layer, ones, groups, prefixes, plen, child, length + 1, self.scale)
        self.pool.free(child, length + 1)
        return out

    def compact(self):
        """The cached prefixes' pages to the front of the cache."""
        n = np.zeros(len(self.length), dtype=np.int64)
        for r in self.slots.values():
            n[r] = self.length[r]
        self.pool.compact(self.table, self._i32(n))
        self._check()


def main():
    from . import workload
    from .pipeline import Pipeline

    ap = argparse.ArgumentParser(description="serve one destination's share of the tiny workload")
    ap.add_argument("--requests", type=int, default=256, help="requests of the destination to serve")
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--codes", choices=("e4m3", "e5m2"), help="hold the cache in these 8-bit floats")
    ap.add_argument("--rotary", action="store_true", help="turn queries and keys by their positions")
    a = ap.parse_args()
    wl = workload.tiny(n=20_000)
    pipe = Pipeline(wl)
    pipe.step()
    dest = pipe.host()["dest"][0]
    mine = np.flatnonzero(dest == 0)[:a.requests]
    keys, suffix = wl.keys[mine], wl.suffix[mine].astype(np.int64)
    plen = wl.prefix_len[keys].astype(np.int64)
    codes = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, None: None}[a.codes]
    d = Destination(wl.candidates[0].W, int(plen.max()), int(suffix.max()), a.batch, samples=2, codes=codes,
                    rotary=serve.Rotary(128) if a.rotary else None)
    t0 = time.perf_counter()
    for b in range(0, len(mine), a.batch):
        e = min(len(mine), b + a.batch)
        d.serve(keys[b:e], plen[b:e], suffix[b:e], first_id=b)
    d.compact()
    torch.cuda.synchronize()
    spent = time.perf_counter() - t0
    c = d.counts
    print(f"destination 0: {c.requests} requests, {c.hits} hits, {c.prefill} tokens prefilled, {c.hit_prefix} taken from the cache, "
          f"errors {int(d.pool.err.item()):#x}, {spent * 1e3:.0f} ms with the stand-in projections")


if __name__ == "__main__":
    main()
