"""Operators of a destination's prefix cache, as a serving loop calls them.

Kinds of case (``kind``):

* ``prompt``  attention over whole packed prompts (requests whose prefix is not cached);
* ``shared``  new keys and values appended to a paged cache, then attention of requests in
              groups that share a prefix (a decoded token each, or the suffix of a hit);
* ``fork``    children of cached sequences: full pages shared, the partial tail copied, and
              the children freed again;
* ``compact`` the live pages of a fragmented cache moved to its front, tables renamed.

Lengths follow the prefixes and suffixes of ``paper_2608_19677_amd/workload.py`` (lognormal
prefixes around 2,000 and 3,000 tokens, suffixes of 50 to 400) or are generic; a case's
lengths come from its ``shape`` number, the values of its tensors from the seed.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
SUFFIX = (50, 400)


def _case(name, kind, **kw):
    c = dict(kind=kind, dtype="bf16", hq=32, hkv=8, d=128, page=16, order="head", shape=1)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # A single short prompt on one request's own: the smallest call, launch and latency.
        _case("prompt_short", "prompt", seqs=1, median=37, sigma=0.0, cap=37, ctx=0),
        # Sixteen-bit floats, small heads, one key head per query head, ragged short chat turns.
        _case("prompt_turns_f16", "prompt", dtype="f16", hq=20, hkv=20, d=64, seqs=24, median=300, sigma=0.6, cap=1021, ctx=0),
        # Misses of one destination's batch: prefixes around 2,000 tokens.
        _case("prompt_misses", "prompt", hq=64, seqs=8, median=2000, sigma=0.5, cap=5003, ctx=0),
        # One long document, the largest call.
        _case("prompt_long", "prompt", hq=64, seqs=1, median=16384, sigma=0.0, cap=16384, ctx=0),
        # The first tokens of three requests behind a short common instruction.
        _case("shared_small", "shared", hq=16, hkv=2, groups=1, reqs=3, median=130, sigma=0.0, cap=130, own_lo=1, own_hi=40, ql_lo=1, ql_hi=1),
        # A decode step of one hot prefix: 64 requests with suffixes of 50 to 400.
        _case("shared_hot", "shared", hq=64, groups=1, reqs=64, median=2000, sigma=0.0, cap=2000, own_lo=50, own_hi=400, ql_lo=1, ql_hi=1),
        # A decode step of a whole destination: many prefixes, uneven groups, tokens before heads in a page.
        _case("shared_mixed_f16", "shared", dtype="f16", hq=48, hkv=8, d=64, page=32, order="token", groups=48, reqs=256, median=2000, sigma=0.5, cap=6007, own_lo=1, own_hi=700, ql_lo=1, ql_hi=1),
        # Suffixes of cache hits: each request brings 50 to 400 new tokens behind its prefix.
        _case("shared_hits", "shared", groups=5, reqs=24, median=3000, sigma=0.7, cap=9001, own_lo=50, own_hi=400, ql_lo=400, ql_hi=400),
        # 128 requests on one very long document, decoding.
        _case("shared_document", "shared", hq=64, groups=1, reqs=128, median=65536, sigma=0.0, cap=65536, own_lo=50, own_hi=2000, ql_lo=1, ql_hi=1),
        # Four samples of one request, one layer: launch and latency.
        _case("fork_small", "fork", layers=1, pages=512, parents=1, children=4, median=200, sigma=0.0, cap=200),
        # Every request of a busy destination forked from its prefix, all layers.
        _case("fork_serve", "fork", layers=32, pages=700, page=32, parents=8, children=192, median=2000, sigma=0.5, cap=2500),
        # A fragmented cache after evictions.
        _case("compact_half", "compact", layers=2, pages=6000, live=0.5, rows=90, width=40),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "shared", "shared", "fork", "compact"])
    hkv = rng.choice([1, 2, 4, 5, 8])
    kw = dict(dtype=rng.choice(["bf16", "f16"]), d=rng.choice([64, 128]), hkv=hkv, hq=hkv * rng.choice([1, 2, 3, 4, 6, 8]),
              page=rng.choice([8, 16, 32, 64, 128]), order=rng.choice(["head", "token"]), shape=rng.randrange(1 << 20))
    if kind == "prompt":
        seqs = _log_int(rng, 1, 32)
        # the plain form's padded scores stay below those of the largest listed case
        top = int(math.sqrt(64 * 16384 ** 2 / (seqs * kw["hq"])))
        cap = _log_int(rng, 20, min(16384, top))
        ctx = rng.choice([0, 0, _log_int(rng, 1, max(2, cap // 2))])
        cap = max(8, cap - ctx)
        return _case(None, kind, seqs=seqs, median=max(1, int(cap * rng.uniform(0.3, 1.0))), sigma=rng.choice([0.0, 0.5, 0.7]), cap=cap, ctx=ctx, **kw)
    if kind == "shared":
        groups = _log_int(rng, 1, 48)
        reqs = max(groups, _log_int(rng, 1, 256))
        cap = _log_int(rng, 60, 65536 // groups)
        own_hi = _log_int(rng, 1, 1500)
        ql = rng.choice([1, 1, _log_int(rng, 2, 200)])
        if ql > 1:
            reqs, groups, cap = min(reqs, 24), min(groups, 5), min(cap, 9001)
        return _case(None, kind, groups=groups, reqs=max(reqs, groups), median=max(1, int(cap * rng.uniform(0.3, 1.0))), sigma=rng.choice([0.0, 0.5]), cap=cap,
                     own_lo=rng.randint(1, own_hi), own_hi=own_hi, ql_lo=1 if rng.random() < 0.5 else ql, ql_hi=ql, **kw)
    token = kw["page"] * kw["hkv"] * kw["d"] * 4  # bytes of a page of keys and values, one layer
    layers = _log_int(rng, 1, 32)
    pages = _log_int(rng, 40, max(41, min(20000, (1 << 30) // (token * layers))))
    if kind == "fork":
        children = _log_int(rng, 1, max(1, min(400, pages // 3)))
        cap = _log_int(rng, 1, max(1, pages // 3 * kw["page"]))
        return _case(None, kind, layers=layers, pages=pages, parents=max(1, min(8, children, pages // 3 * kw["page"] // cap)), children=children,
                     median=max(1, int(cap * rng.uniform(0.3, 1.0))), sigma=0.5, cap=cap, **kw)
    return _case(None, kind, layers=layers, pages=pages, live=rng.uniform(0.05, 0.95), rows=_log_int(rng, 1, 200), width=_log_int(rng, 1, 100), **kw)


# ---------------------------------------------------------------------------
# Lengths: from the case alone.
# ---------------------------------------------------------------------------

def _lengths(r, n, c):
    return [max(1, min(c["cap"], round(c["median"] * math.exp(c["sigma"] * r.gauss(0, 1))))) for _ in range(n)]


def _prompt_lens(c):
    r = random.Random(c["shape"])
    q = _lengths(r, c["seqs"], c)
    return q, [n + (r.randint(0, c["ctx"]) if c["ctx"] else 0) for n in q]


def _shared_lens(c):
    r = random.Random(c["shape"])
    prefix = _lengths(r, c["groups"], c)
    cuts = sorted(r.sample(range(1, c["reqs"]), c["groups"] - 1)) if c["groups"] > 1 else []
    group_off = [0] + cuts + [c["reqs"]]
    own_len = [r.randint(c["own_lo"], c["own_hi"]) for _ in range(c["reqs"])]
    q_len = [min(o, r.randint(c["ql_lo"], c["ql_hi"])) for o in own_len]
    return prefix, group_off, own_len, q_len


def _fork_lens(c):
    r = random.Random(c["shape"])
    plen = _lengths(r, c["parents"], c)
    parent = sorted(r.randrange(c["parents"]) for _ in range(c["children"]))
    # a child starts at its parent's end, or behind some of its tokens
    return plen, parent, [plen[p] if r.random() < 0.7 else r.randint(0, plen[p]) for p in parent]


def _cum(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def _up(a, b):
    return -(-a // b)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32).to(DEV)


# ---------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dtype)


def _pool(c, g, layers, pages):
    h, p, d = c["hkv"], c["page"], c["d"]
    shape = (layers, pages, h, p, d) if c["order"] == "head" else (layers, pages, p, h, d)
    return _randn(g, shape, DTYPES[c["dtype"]]), _randn(g, shape, DTYPES[c["dtype"]])


def _handle(st, c):
    from paper_2608_19677_amd.serve import PagePool
    st.pool = PagePool(st.k, st.v, st.refs, order=c["order"])


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = SimpleNamespace(case=c, scale=1.0 / math.sqrt(c["d"]))
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "prompt":
        q_len, k_len = _prompt_lens(c)
        st.max_q, st.max_k = max(q_len), max(k_len)
        st.q_off, st.k_off = _i32(_cum(q_len)), _i32(_cum(k_len))
        nq, nk = sum(q_len), sum(k_len)
        # attention sharper than that of unit vectors: some rows lean on few keys
        st.q = _randn(g, (nq, c["hq"], c["d"]), dt, 1.5)
        kv = _randn(g, (nk, 2, c["hkv"], c["d"]), dt)  # one projection's output: strided halves
        st.k, st.v = kv[:, 0], kv[:, 1]
        st.out = torch.empty_like(st.q)
        st.lse = torch.empty((nq, c["hq"]), dtype=torch.float32, device=DEV)
        if own:  # the workspace that a serving loop keeps
            from paper_2608_19677_amd import serve
            st.ws = serve.prompt_workspace(st.q, st.k, st.q_off)
        return st
    if c["kind"] == "shared":
        prefix, group_off, own_len, q_len = _shared_lens(c)
        pg = c["page"]
        np_, no = [_up(x, pg) for x in prefix], [_up(x, pg) for x in own_len]
        pages = sum(np_) + sum(no) + 5
        ids = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)  # pages lie anywhere
        st.prefix_table, at = _tables(ids, np_, 0)
        st.own_table, at = _tables(ids, no, at)
        st.refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
        st.refs[ids[:at].long()] = 1
        st.k, st.v = _pool(c, g, 1, pages)
        st.max_prefix, st.max_own, st.max_q = max(prefix), max(own_len), max(q_len)
        st.max_group = max(sum(q_len[a:b]) for a, b in zip(group_off, group_off[1:]))
        st.prefix_len, st.own_len = _i32(prefix), _i32(own_len)
        st.group_off, st.q_off = _i32(group_off), _i32(_cum(q_len))
        nq = sum(q_len)
        st.q = _randn(g, (nq, c["hq"], c["d"]), dt, 1.5)
        st.k_new, st.v_new = _randn(g, (nq, c["hkv"], c["d"]), dt), _randn(g, (nq, c["hkv"], c["d"]), dt)
        st.out = torch.empty_like(st.q)
        st.lse = torch.empty((nq, c["hq"]), dtype=torch.float32, device=DEV)
        if own:  # the cache's handle and the workspace that a serving loop keeps
            from paper_2608_19677_amd import serve
            _handle(st, c)
            st.ws = serve.shared_workspace(st.q, st.pool, st.group_off, st.prefix_table, st.own_table)
        return st
    if c["kind"] == "fork":
        plen, parent, clen = _fork_lens(c)
        n = [_up(x, c["page"]) for x in plen]
        ids = torch.randperm(c["pages"], generator=g, device=DEV).to(torch.int32)
        st.table, at = _tables(ids, n, 0)
        st.refs = torch.zeros(c["pages"], dtype=torch.int32, device=DEV)
        st.refs[ids[:at].long()] = 1
        st.k, st.v = _pool(c, g, c["layers"], c["pages"])
        st.parent, st.length = _i32(parent), _i32(clen)
        st.child = torch.empty((len(parent), st.table.shape[1] + 1), dtype=torch.int32, device=DEV)
    else:
        live = max(1, round(c["pages"] * c["live"]))
        ids = torch.randperm(c["pages"], generator=g, device=DEV)[:live].to(torch.int32)
        st.table = ids[torch.randint(live, (c["rows"], c["width"]), generator=g, device=DEV)]
        st.length = torch.randint(0, c["width"] * c["page"] + 1, (c["rows"],), generator=g, device=DEV).to(torch.int32)
        st.refs = torch.zeros(c["pages"], dtype=torch.int32, device=DEV)
        st.refs[ids.long()] = 1 + torch.randint(3, (live,), generator=g, device=DEV).to(torch.int32)
        st.k, st.v = _pool(c, g, c["layers"], c["pages"])
        st.table_out, st.refs_out = torch.empty_like(st.table), torch.empty_like(st.refs)
    if own:  # the cache's handle
        _handle(st, c)
    return st


def _tables(ids, counts, at):
    """Rows of page ids taken from ids[at:], -1 behind each row's pages."""
    t = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32, device=DEV)
    for i, n in enumerate(counts):
        t[i, :n] = ids[at:at + n]
        at += n
    return t, at


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------

def run(st):
    return (_run_own if own else _run_plain)[st.case["kind"]](st)


def _own_prompt(st):
    from paper_2608_19677_amd import serve
    serve.attend_prompt(st.q, st.k, st.v, st.q_off, st.k_off, st.scale, out=st.out, lse=st.lse, ws=st.ws)
    return {"out": st.out, "lse": st.lse}


def _own_shared(st):
    from paper_2608_19677_amd import serve
    st.pool.append(0, st.k_new, st.v_new, st.q_off, st.own_len, st.own_table)
    serve.attend_shared(st.q, st.pool, 0, st.q_off, st.group_off, st.prefix_table, st.prefix_len, st.own_table, st.own_len, st.scale, out=st.out, lse=st.lse, ws=st.ws)
    return {"out": st.out, "lse": st.lse, "k": st.k, "v": st.v}


def _own_fork(st):
    st.pool.fork(st.table, st.parent, st.length, st.child)
    st.pool.free(st.child, st.length)
    return {"child": st.child, "refs": st.refs, "k": st.k, "v": st.v}


def _own_compact(st):
    st.pool.compact(st.table, st.length, table_out=st.table_out, refs_out=st.refs_out)
    return {"table": st.table_out, "refs": st.refs_out, "k": st.k, "v": st.v}


_run_own = {"prompt": _own_prompt, "shared": _own_shared, "fork": _own_fork, "compact": _own_compact}


def _softmax_parts(s, mask, v):
    """Scores (..., rows, keys), mask broadcastable to them, values (..., keys, d): the values
    weighed by the masked softmax, and the log of its sum (rows without a key: 0 and -inf)."""
    s.masked_fill_(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (m + total.log()).squeeze(-1)


def _rows(x, off, n):
    """Packed rows (tokens, ...) padded to (sequences, n, ...) in 32 bits."""
    at = off[:-1, None].long() + torch.arange(n, device=DEV)
    return x[at.clamp(max=x.shape[0] - 1)].float()


def _by_head(q, hkv):
    """(B, n, Hq, D) to (B, Hkv, G n, D), rows of one key head's query heads together."""
    b, n, hq, d = q.shape
    return q.reshape(b, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, hq // hkv * n, d)


def _by_token(o, n):
    """(B, Hkv, G n, ...) back to (B, n, Hq, ...)."""
    b, h, gn = o.shape[:3]
    o = o.reshape(b, h, gn // n, n, *o.shape[3:])
    return o.permute(0, 3, 1, 2, *range(4, o.dim())).reshape(b, n, h * (gn // n), *o.shape[4:])


def _place(off, n):
    """Of each packed row: its sequence and its place there."""
    t = torch.arange(n, device=DEV)
    b = torch.searchsorted(off[1:].long(), t, right=True)
    return b, t - off.long()[b]


def _plain_prompt(st):
    hkv, n, m = st.case["hkv"], st.max_q, st.max_k
    q = _by_head(_rows(st.q, st.q_off, n), hkv)
    k, v = (_rows(x, st.k_off, m).permute(0, 2, 1, 3) for x in (st.k, st.v))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st.scale)
    nq, nk = (x.diff().long()[:, None, None] for x in (st.q_off, st.k_off))
    i, j = torch.arange(n, device=DEV)[None, :, None], torch.arange(m, device=DEV)[None, None, :]
    mask = (j < nk) & (j <= i + nk - nq)
    o, lse = _softmax_parts(s.view(s.shape[0], hkv, -1, n, m), mask[:, None, None], v.unsqueeze(2))
    b, i = _place(st.q_off, st.q.shape[0])
    o, lse = _by_token(o.flatten(2, 3), n), _by_token(lse.flatten(2, 3), n)
    return {"out": o[b, i].to(st.q.dtype), "lse": lse[b, i]}


def _paged(x, table, n, order):
    """The first n tokens of each row of pages, layer 0: (rows, Hkv, n, D) in 32 bits."""
    t = x[0][table.clamp(min=0).long()]
    t = t if order == "token" else t.transpose(2, 3)
    return t.flatten(1, 2)[:, :n].float().transpose(1, 2)


def _plain_shared(st):
    c, hkv, n = st.case, st.case["hkv"], st.max_q
    b, i = _place(st.q_off, st.q.shape[0])
    nq = st.q_off.diff().long()
    pos = (st.own_len.long() - nq)[b] + i
    page, slot = st.own_table[b, pos // c["page"]].long(), pos % c["page"]
    # the new tokens into their pages
    for x, new in ((st.k, st.k_new), (st.v, st.v_new)):
        (x[0] if c["order"] == "token" else x[0].transpose(1, 2))[page, slot] = new
    # every group's prefix, for all rows of the group
    tok_off = st.q_off[st.group_off.long()]
    mg = st.max_group
    q = _by_head(_rows(st.q, tok_off, mg), hkv)
    k, v = (_paged(x, st.prefix_table, st.max_prefix, c["order"]) for x in (st.k, st.v))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st.scale)
    mask = torch.arange(st.max_prefix, device=DEV) < st.prefix_len.long()[:, None]
    o1, lse1 = _softmax_parts(s, mask[:, None, None], v)
    g, at = _place(tok_off, st.q.shape[0])
    o1, lse1 = _by_token(o1, mg)[g, at], _by_token(lse1, mg)[g, at]
    # every request's own tokens
    q = _by_head(_rows(st.q, st.q_off, n), hkv)
    k, v = (_paged(x, st.own_table, st.max_own, c["order"]) for x in (st.k, st.v))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st.scale)
    j, row = torch.arange(st.max_own, device=DEV), torch.arange(n, device=DEV)
    mask = j <= (row + (st.own_len.long() - nq)[:, None])[:, :, None]
    o2, lse2 = _softmax_parts(s.view(s.shape[0], hkv, -1, n, st.max_own), mask[:, None, None], v.unsqueeze(2))
    o2, lse2 = _by_token(o2.flatten(2, 3), n)[b, i], _by_token(lse2.flatten(2, 3), n)[b, i]
    lse = torch.logaddexp(lse1, lse2)
    o = o1 * (lse1 - lse).exp()[..., None] + o2 * (lse2 - lse).exp()[..., None]
    return {"out": o.to(st.q.dtype), "lse": lse, "k": st.k, "v": st.v}


def _plain_fork(st):
    pg = st.case["page"]
    n = st.length.long()
    full, tail = n // pg, n % pg
    need = tail > 0
    rows = st.table.long()[st.parent.long()]
    free = torch.sort((st.refs > 0).to(torch.int8), stable=True).indices  # free pages, lowest first
    new = free[(need.long().cumsum(0) - 1).clamp(min=0)]
    src = rows.gather(1, full[:, None].clamp(max=rows.shape[1] - 1)).squeeze(1)
    new = torch.where(need, new, src.clamp(min=0))
    col = torch.arange(st.child.shape[1], device=DEV)
    rows = torch.nn.functional.pad(rows, (0, 1), value=-1)
    child = torch.where(col < full[:, None], rows, torch.where((col == full[:, None]) & need[:, None], new[:, None], -1))
    used = (child >= 0).to(torch.int32).flatten()
    at = child.clamp(min=0).flatten()
    st.refs.scatter_add_(0, at, used)
    st.child.copy_(child)
    tok = torch.arange(pg, device=DEV) < tail[:, None]
    tok = tok[:, None, :, None] if st.case["order"] == "head" else tok[:, :, None, None]
    src = src.clamp(min=0)
    for x in (st.k, st.v):
        x[:, new] = torch.where(tok, x[:, src], x[:, new])
    st.refs.scatter_add_(0, at, -used)
    return {"child": st.child, "refs": st.refs, "k": st.k, "v": st.v}


def _plain_compact(st):
    live = st.refs > 0
    n = live.sum()
    ids = torch.arange(st.refs.shape[0], device=DEV)
    src, dst = (live & (ids >= n)).nonzero()[:, 0], (~live & (ids < n)).nonzero()[:, 0]
    name = ids.clone()
    name[src] = dst
    st.refs_out.copy_(st.refs)
    st.refs_out[dst] = st.refs[src]
    st.refs_out[src] = 0
    used = torch.arange(st.table.shape[1], device=DEV) * st.case["page"] < st.length[:, None]
    st.table_out.copy_(torch.where(used, name[st.table.long()], st.table))
    for x in (st.k, st.v):
        x[:, dst] = x[:, src]
    return {"table": st.table_out, "refs": st.refs_out, "k": st.k, "v": st.v}


_run_plain = {"prompt": _plain_prompt, "shared": _plain_shared, "fork": _plain_fork, "compact": _plain_compact}


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it should give.
# ---------------------------------------------------------------------------

def work(case):
    c = case
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "prompt":
        q_len, k_len = _prompt_lens(c)
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q_len, k_len))
        return {"bytes": sum(q_len) * hq * (4 * d + 4) + sum(k_len) * hkv * 4 * d, "flops": 4 * d * hq * pairs}
    if c["kind"] == "shared":
        prefix, group_off, own_len, q_len = _shared_lens(c)
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q_len, own_len))
        for p, a, b in zip(prefix, group_off, group_off[1:]):
            pairs += p * sum(q_len[a:b])
        kv = sum(prefix) + sum(own_len) + sum(q_len)  # the new tokens are read beside the cache
        return {"bytes": sum(q_len) * hq * (4 * d + 4) + kv * hkv * 4 * d + 4 * (_up(sum(prefix), c["page"]) + _up(sum(own_len), c["page"])), "flops": 4 * d * hq * pairs}
    if c["kind"] == "fork":
        plen, _, clen = _fork_lens(c)
        tails = sum(n % c["page"] for n in clen) * hkv * d * 4 * c["layers"]
        entries = sum(_up(n, c["page"]) for n in clen)
        return {"bytes": 2 * tails + 4 * 4 * entries + 4 * c["pages"], "flops": 0}
    live = max(1, round(c["pages"] * c["live"]))
    moved = live * (c["pages"] - live) / c["pages"]  # expected of scattered pages
    return {"bytes": 2 * moved * c["page"] * hkv * d * 4 * c["layers"] + 8 * c["pages"] + 8 * c["rows"] * c["width"], "flops": 0}


def exact(case, seed):
    if case["kind"] not in ("prompt", "shared"):
        return None  # copies and whole numbers: nothing computed
    st = prepare(case, seed)
    c, group = case, case["hq"] // case["hkv"]
    outs, lses = [], []

    def head(q, parts):
        """One head's rows (float64) over parts of (keys, values, limit of each row)."""
        s = [torch.where(torch.arange(k.shape[0], device=DEV) < lim[:, None], (q @ k.t().contiguous()) * st.scale, -math.inf) for k, _, lim in parts]
        s = torch.cat(s, 1)
        lse = torch.logsumexp(s, 1)
        return torch.nan_to_num(torch.exp(s - lse[:, None]), nan=0.0) @ torch.cat([v for _, v, _ in parts]), lse

    if c["kind"] == "prompt":
        q_len, k_len = _prompt_lens(c)
        if c["hq"] * sum(n * m for n, m in zip(q_len, k_len)) > 2e10:
            return None
        seqs = []
        for a, n, b, m in zip(_cum(q_len), q_len, _cum(k_len), k_len):
            lim = torch.arange(n, device=DEV) + m - n + 1
            seqs.append((st.q[a:a + n], [(st.k[b:b + m], st.v[b:b + m], lim)]))
    else:
        prefix, group_off, own_len, q_len = _shared_lens(c)
        if c["hq"] * sum(sum(q_len[a:b]) * p for p, a, b in zip(prefix, group_off, group_off[1:])) > 2e10:
            return None

        def tokens(x, row, n):
            p = x[0][row[:_up(n, c["page"])].long()]
            return (p.transpose(1, 2) if c["order"] == "head" else p).reshape(-1, c["hkv"], c["d"])[:n]

        off, seqs = _cum(q_len), []
        for g, (a, b) in enumerate(zip(group_off, group_off[1:])):
            pk, pv = (tokens(x, st.prefix_table[g], prefix[g]) for x in (st.k, st.v))
            for r in range(a, b):
                n, m = q_len[r], own_len[r]
                ok, ov = (torch.cat([tokens(x, st.own_table[r], m)[:m - n], new[off[r]:off[r] + n]]) for x, new in ((st.k, st.k_new), (st.v, st.v_new)))
                all_of = torch.full((n,), prefix[g], device=DEV)
                seqs.append((st.q[off[r]:off[r] + n], [(pk, pv, all_of), (ok, ov, torch.arange(n, device=DEV) + m - n + 1)]))
    for q, parts in seqs:
        o, l = torch.empty(q.shape, dtype=torch.float64, device=DEV), torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
        for h in range(c["hkv"]):
            heads = q[:, h * group:(h + 1) * group].double().transpose(0, 1).reshape(-1, c["d"])
            got = head(heads, [(k[:, h].double(), v[:, h].double(), lim.repeat(group)) for k, v, lim in parts])
            o[:, h * group:(h + 1) * group] = got[0].reshape(group, -1, c["d"]).transpose(0, 1)
            l[:, h * group:(h + 1) * group] = got[1].reshape(group, -1).t()
        outs.append(o)
        lses.append(l)
    got = {"out": torch.cat(outs), "lse": torch.cat(lses)}
    return got if c["kind"] == "prompt" else {**got, "k": None, "v": None}
