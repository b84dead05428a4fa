"""Prompt attention and shared-prefix attention against their 64-bit statement, where they can go
wrong: lengths of none and one, rows without a key, odd head groups, strides, pages that end inside a
tile, stale bits behind every sequence's end, few rows on long keys, streams and captured graphs."""
import math

import numpy as np
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _cum(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(int).tolist()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


PROMPTS = [
    # dtype, heads, key heads, dim, query lengths, key lengths, causal
    ("bf16", 8, 1, 128, [1], [1], True),
    ("bf16", 4, 4, 64, [0, 1, 0, 2, 65, 0], [0, 1, 3, 2, 65, 0], True),
    ("f16", 8, 2, 128, [33, 64, 127, 128, 129], [33, 64, 127, 128, 129], True),
    ("f16", 6, 2, 64, [31, 100, 5], [200, 100, 69], True),
    ("bf16", 7, 1, 128, [50, 3, 40], [20, 3, 0], True),     # rows that see no key
    ("bf16", 5, 5, 128, [50, 17, 4], [70, 1, 0], False),
    ("bf16", 20, 4, 64, [200, 1], [200, 1], False),
    ("f16", 3, 3, 128, [257], [513], True),
    ("bf16", 8, 2, 128, [3], [5000], True),                # few rows, keys split over workgroups
    ("f16", 2, 1, 64, [1, 2], [3001, 0], True),
    ("bf16", 64, 8, 128, [1] * 70, [9] * 70, True),        # more sequences than lanes
]


@pytest.mark.parametrize("case", PROMPTS, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-{len(c[4])}seq-{max(c[5])}" for c in PROMPTS])
@pytest.mark.parametrize("strided", [False, True])
def test_prompt(case, strided):
    name, hq, hkv, d, ql, kl, causal = case
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[name]
    say(f"[case] prompt {case} strided={strided}")
    g = _gen(hash((hq, hkv, d, sum(ql), sum(kl))) % 1000)
    nq, nk = sum(ql), sum(kl)
    if strided:  # one projection's rows [tokens, heads of q, k and v]; heads before tokens in the output
        q = _randn(g, nq, hq + 3, d, dtype=dt, scale=1.5)[:, 1:hq + 1]
        kv = _randn(g, nk, 2, hkv, d, dtype=dt)
        k, v = kv[:, 0], kv[:, 1]
        out = torch.empty(hq, nq, d, dtype=dt, device="cuda").transpose(0, 1)
    else:
        q, k, v = _randn(g, nq, hq, d, dtype=dt, scale=1.5), _randn(g, nk, hkv, d, dtype=dt), _randn(g, nk, hkv, d, dtype=dt)
        out = torch.full((nq, hq, d), math.nan, dtype=dt, device="cuda")
    lse = torch.full((nq, hq), math.nan, device="cuda")
    scale = 1 / math.sqrt(d)
    ws = serve.prompt_workspace(q, k, _i32(_cum(ql)))
    serve.attend_prompt(q, k, v, _i32(_cum(ql)), _i32(_cum(kl)), scale, out=out, lse=lse, causal=causal, ws=ws)
    assert int(ws.err.item()) == 0
    ref = so.flat(so.prompt(q, k, v, _cum(ql), _cum(kl), scale, causal))
    so.check(out.reshape(-1, d), lse.reshape(-1), ref, dt, str(case))
    again = serve.attend_prompt(q, k, v, _i32(_cum(ql)), _i32(_cum(kl)), scale, causal=causal)
    assert torch.equal(again, out)


def test_prompt_largest_scores_first_and_last():
    """The running maximum falls from its first key, rises to its last, and jumps in between."""
    n, d = 700, 128
    for seed, order in enumerate(("down", "up", "jump")):
        g = _gen(40 + seed)
        q, k, v = (_randn(g, n, 1, d, dtype=torch.bfloat16) for _ in range(3))
        ramp = torch.linspace(0, 6, n, device="cuda")[:, None, None]
        ramp = {"down": ramp.flip(0), "up": ramp, "jump": (torch.arange(n, device="cuda")[:, None, None] % 97 == 96) * 6.0}[order]
        k = (k + ramp * q.float().mean(0, keepdim=True) * 8).to(torch.bfloat16)
        say(f"[case] prompt scores {order}")
        off = [0, n]
        lse = torch.empty(n, 1, device="cuda")
        out = serve.attend_prompt(q, k, v, _i32(off), _i32(off), 0.5, lse=lse)
        so.check(out.reshape(-1, d), lse.reshape(-1), so.flat(so.prompt(q, k, v, off, off, 0.5, True)), torch.bfloat16, order)


def test_prompt_other_sequences_never_reach_a_row():
    ql = [70, 64, 1, 130]
    off = _cum(ql)
    g = _gen(5)
    q, k, v = (_randn(g, sum(ql), 4, 128, dtype=torch.bfloat16) for _ in range(3))
    clean = serve.attend_prompt(q, k, v, _i32(off), _i32(off), 0.1)
    for bad in (math.nan, math.inf, -math.inf, torch.finfo(torch.bfloat16).min):
        k2, v2 = k.clone(), v.clone()
        for b in (0, 2):
            k2[off[b]:off[b + 1]], v2[off[b]:off[b + 1]] = bad, bad
        say(f"[case] prompt with {bad} in other sequences")
        got = serve.attend_prompt(q, k2, v2, _i32(off), _i32(off), 0.1)
        for b in (1, 3):
            assert torch.equal(got[off[b]:off[b + 1]], clean[off[b]:off[b + 1]])


SHARED = [
    # dtype, heads, key heads, dim, page, order, prefix lengths, requests per group, own lengths, query lengths
    ("bf16", 8, 1, 128, 16, "head", [130], [3], [1, 7, 40], [1, 1, 1]),
    ("f16", 16, 2, 64, 32, "token", [65, 0, 1], [2, 1, 3], [5, 9, 1, 64, 65, 33], [1] * 6),
    ("bf16", 4, 4, 128, 1, "head", [77], [2], [3, 18], [3, 2]),
    ("bf16", 6, 2, 64, 8, "token", [200, 63], [0, 4], [10, 20, 100, 3], [10, 1, 37, 3]),
    ("f16", 7, 1, 128, 128, "head", [500, 3], [1, 1], [130, 0], [130, 0]),
    ("bf16", 8, 8, 128, 64, "head", [0], [2], [4, 2], [4, 5]),   # no prefix; a query before its first own token
    ("bf16", 16, 2, 128, 16, "token", [3000], [40], [17 * (i % 5) + 1 for i in range(40)], [1] * 40),
    ("f16", 32, 4, 64, 16, "head", [10] * 70, [1] * 70, [2] * 70, [1] * 70),
    ("bf16", 8, 1, 128, 16, "head", [40], [1], [4000], [2]),
]


def _paged_case(case, seed, poison=math.nan):
    name, hq, hkv, d, pg, order, prefix, per, own, ql = case
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[name]
    g = _gen(seed)
    up = lambda n: -(-n // pg)  # noqa: E731
    need = [up(n) for n in prefix] + [up(n) for n in own]
    pages = sum(need) + 3
    pool = serve.PagePool.empty(2, pages, hkv, pg, d, dt, order=order)
    pool.k.fill_(poison), pool.v.fill_(poison)
    ids = torch.randperm(pages, generator=g, device="cuda").tolist()
    width = max(need) + 1
    rows, kv, at = [], [], 0
    for n, m in zip(prefix + own, need):
        rows.append(ids[at:at + m] + [-1] * (width - m))
        at += m
        kv.append((_randn(g, n, hkv, d, dtype=dt), _randn(g, n, hkv, d, dtype=dt)))
    ng = len(prefix)
    tab = _i32(rows)
    # all tokens but the queries' are in the cache already
    done = list(prefix) + [max(0, n - q) for n, q in zip(own, ql)]
    for i, n in enumerate(done):
        if n:
            pool.append(1, kv[i][0][:n], kv[i][1][:n], _i32([0, n]), _i32([n]), tab[i:i + 1])
    new = [min(n, q) for n, q in zip(own, ql)]
    kn = torch.cat([x[0][len(x[0]) - m:] for x, m in zip(kv[ng:], new)])
    vn = torch.cat([x[1][len(x[1]) - m:] for x, m in zip(kv[ng:], new)])
    pool.append(1, kn, vn, _i32(_cum(new)), _i32(own), tab[ng:])
    q = _randn(g, sum(ql), hq, d, dtype=dt, scale=1.5)
    return pool, q, tab[:ng], tab[ng:], kv[:ng], kv[ng:], _cum(ql), _cum(per), dt


@pytest.mark.parametrize("case", SHARED, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{c[5]}-{max(c[6])}-{len(c[8])}req" for c in SHARED])
def test_shared(case):
    say(f"[case] shared {case}")
    prefix, own = case[6], case[8]
    pool, q, ptab, otab, pkv, okv, q_off, g_off, dt = _paged_case(case, 11)
    d, scale = case[3], 1 / math.sqrt(case[3])
    args = (q, pool, 1, _i32(q_off), _i32(g_off), ptab, _i32(prefix), otab, _i32(own), scale)
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    out = torch.full_like(q, math.nan)
    serve.attend_shared(*args, out=out, lse=lse)
    assert int(pool.err.item()) == 0
    ref = so.shared(q, [tuple(map(so.f64, x)) for x in pkv], [tuple(map(so.f64, x)) for x in okv], q_off, g_off, scale)
    so.check(out.reshape(-1, d), lse.reshape(-1), so.flat(ref), dt, str(case))
    assert torch.equal(serve.attend_shared(*args), out)
    # no layer but its own was written
    assert torch.isnan(pool.k[0].float()).all() and torch.isnan(pool.v[0].float()).all()


@pytest.mark.parametrize("bad", [0.0, math.inf, -math.inf, torch.finfo(torch.bfloat16).min])
def test_shared_stale_bits_never_reach_a_row(bad):
    case = SHARED[0][:6] + ([77, 16], [2, 1], [3, 18, 16], [1, 2, 1])
    say(f"[case] shared with {bad} behind the ends")
    runs = []
    for poison in (math.nan, bad):
        pool, q, ptab, otab, _, _, q_off, g_off, _ = _paged_case(case, 12, poison)
        runs.append(serve.attend_shared(q, pool, 1, _i32(q_off), _i32(g_off), ptab, _i32(case[6]), otab, _i32(case[8]), 0.1))
    assert torch.isfinite(runs[0].float()).all() and torch.equal(*runs)


def test_shared_equals_prompt_over_the_whole_sequence():
    """One request with everything in its own pages, all rows, is a prompt."""
    n, hq, hkv, d = 150, 8, 2, 128
    case = ("bf16", hq, hkv, d, 16, "head", [0], [1], [n], [n])
    pool, q, ptab, otab, _, okv, q_off, g_off, dt = _paged_case(case, 13)
    say("[case] shared = prompt")
    got = serve.attend_shared(q, pool, 1, _i32(q_off), _i32(g_off), ptab, _i32([0]), otab, _i32([n]), 0.09)
    k, v = okv[0]
    want = serve.attend_prompt(q, k, v, _i32([0, n]), _i32([0, n]), 0.09)
    assert (got.float() - want.float()).abs().max() <= 2 * so.UNIT[dt] * want.float().abs().max()


def test_append_places_tokens():
    """The pool holds exactly the appended rows at their places and is untouched elsewhere."""
    for order in ("head", "token"):
        pool = serve.PagePool.empty(3, 40, 2, 8, 64, torch.float16, order=order)
        pool.k.fill_(7), pool.v.fill_(9)
        lens, new = [17, 8, 3, 25], [17, 1, 0, 9]
        g = _gen(3)
        tab = _i32(torch.randperm(40, generator=g, device="cuda").tolist()).reshape(4, 10)
        kv = _randn(g, sum(new), 2, 2, 64, dtype=torch.float16)
        k, v = kv[:, 0], kv[:, 1]
        want_k, want_v = pool.k.cpu().clone(), pool.v.cpu().clone()
        say(f"[case] append {order}")
        pool.append(2, k, v, _i32(_cum(new)), _i32(lens), tab)
        at = 0
        for i, (n, m) in enumerate(zip(lens, new)):
            for p in range(n - m, n):
                page, t = int(tab[i, p // 8]), p % 8
                for want, x in ((want_k, k), (want_v, v)):
                    (want[2, page, :, t] if order == "head" else want[2, page, t]).copy_(x[at].cpu())
                at += 1
        assert torch.equal(pool.k.cpu(), want_k) and torch.equal(pool.v.cpu(), want_v) and int(pool.err.item()) == 0


def test_data_errors_set_bits_and_spare_the_others():
    g = _gen(9)
    q, k, v = (_randn(g, 60, 4, 64, dtype=torch.bfloat16) for _ in range(3))
    good = serve.attend_prompt(q, k, v, _i32([0, 20, 40, 60]), _i32([0, 20, 40, 60]), 0.1)
    ws = serve.prompt_workspace(q, k, _i32([0, 20, 40, 60]))
    say("[case] key offsets past the end")
    got = serve.attend_prompt(q, k, v, _i32([0, 20, 40, 60]), _i32([0, 20, 40, 61]), 0.1, ws=ws)
    assert int(ws.err.item()) == B.CR_ERR_SEQ and torch.equal(got[:40], good[:40])
    case = SHARED[0][:6] + ([40], [2], [20, 20], [1, 1])
    pool, q, ptab, otab, _, _, q_off, g_off, _ = _paged_case(case, 14)
    args = lambda pt, pl, ot, ol: serve.attend_shared(q, pool, 1, _i32(q_off), _i32(g_off), pt, _i32(pl), ot, _i32(ol), 0.1)  # noqa: E731
    good = args(ptab, [40], otab, [20, 20])
    assert int(pool.err.item()) == 0
    say("[case] a length past its table")
    got = args(ptab, [40], otab, [20, 4000])
    assert int(pool.err.item()) == B.CR_ERR_SEQ and torch.equal(got[:1], good[:1])
    pool.err.zero_()
    bad = otab.clone()
    bad[1, 0] = pool.num_pages
    say("[case] a page out of range")
    got = args(ptab, [40], bad, [20, 20])
    assert int(pool.err.item()) == B.CR_ERR_PAGE and torch.equal(got[:1], good[:1])


def test_calls_on_another_stream_and_in_a_graph():
    case = SHARED[6]
    pool, q, ptab, otab, _, _, q_off, g_off, _ = _paged_case(case, 15)
    plen, olen, qo, go = _i32(case[6]), _i32(case[8]), _i32(q_off), _i32(g_off)
    ws = serve.shared_workspace(q, pool, go, ptab, otab)
    out = torch.empty_like(q)
    want = serve.attend_shared(q, pool, 1, qo, go, ptab, plen, otab, olen, 0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    say("[case] shared on a side stream")
    got = serve.attend_shared(q, pool, 1, qo, go, ptab, plen, otab, olen, 0.1, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    say("[case] shared in a graph")
    with torch.cuda.graph(graph):
        serve.attend_shared(q, pool, 1, qo, go, ptab, plen, otab, olen, 0.1, out=out, ws=ws)
    for i in range(3):
        q.mul_(-1)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, serve.attend_shared(q, pool, 1, qo, go, ptab, plen, otab, olen, 0.1))
