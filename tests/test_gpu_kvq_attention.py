"""Attention over the 8-bit cache against 64 bits on what its codes stand for, in every form of the call: few rows and tiles,
prefixes read once or again, pages that end inside a tile, blocks of one token to 128, stale codes and scales behind
every end, values that are not finite, streams and captured graphs."""
import math

import numpy as np
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import kvq_oracle as ko
import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


CASES = {
    # type, code, heads, key heads, dim, page, block, order, prefix lengths, requests per group, own lengths, query lengths
    "one": ("bf16", "e4m3", 8, 1, 128, 16, 16, "head", [130], [3], [1, 7, 40], [1, 1, 1]),
    "uneven": ("f16", "e5m2", 16, 2, 64, 32, 8, "token", [65, 0, 1], [2, 1, 3], [5, 9, 1, 64, 65, 33], [1] * 6),
    "page-a-token": ("bf16", "e5m2", 4, 4, 128, 1, 1, "head", [77], [2], [3, 18], [3, 2]),
    "empty-group": ("bf16", "e4m3", 6, 2, 64, 8, 4, "token", [200, 63], [0, 4], [10, 20, 100, 3], [10, 1, 37, 3]),
    "no-keys": ("f16", "e4m3", 7, 1, 128, 128, 64, "head", [500, 3], [1, 1], [130, 0], [130, 0]),
    "before-own": ("bf16", "e4m3", 8, 8, 128, 64, 1, "head", [0], [2], [4, 2], [4, 5]),
    "decode": ("bf16", "e4m3", 16, 2, 128, 16, 16, "token", [3000], [40], [17 * (i % 5) + 1 for i in range(40)], [1] * 40),
    "many": ("f16", "e4m3", 32, 4, 64, 16, 16, "head", [10] * 70, [1] * 70, [2] * 70, [1] * 70),
    "long-own": ("bf16", "e5m2", 8, 1, 128, 16, 2, "head", [40], [1], [4000], [2]),
    "pairs": ("f16", "e4m3", 8, 2, 128, 1, 1, "head", [50], [2], [30, 16], [14, 16]),
    "tiles": ("bf16", "e4m3", 8, 2, 128, 16, 8, "head", [70, 300], [2, 1], [60, 40, 90], [60, 40, 33]),
    "tiles-64": ("f16", "e5m2", 8, 8, 64, 2, 2, "token", [1500], [2], [300, 290], [300, 290]),
    "whole": ("bf16", "e4m3", 32, 8, 128, 32, 32, "head", [77], [2], [150, 100], [150, 80]),
    "whole-wide": ("f16", "e4m3", 64, 8, 128, 16, 16, "token", [2500, 900], [2, 3], [400, 333, 100, 257, 64], [400, 300, 100, 257, 1]),
    "whole-wide-64": ("bf16", "e5m2", 32, 32, 64, 128, 128, "head", [1300], [2], [700, 690], [700, 690]),
    "group-wide": ("bf16", "e4m3", 64, 8, 128, 64, 64, "head", [5000], [50], [20] * 50, [1] * 50),
}


def _setup(case, seed, plant=None, stale=0):
    """A pool with everything appended, and what its codes stand for. plant(k, v): changes to the packed rows of
    all prefixes, then all own tokens. What no token lies in holds NaN codes, or `stale`."""
    name, code, hq, hkv, d, pg, block, order, prefix, per, own, ql = case
    dt, g = ko.DT[name], _gen(seed)
    lens = prefix + own
    need = [-(-n // pg) for n in lens]
    pages = sum(need) + 2
    pool = serve.QuantPagePool.empty(2, pages, hkv, pg, d, dt, order=order, codes=ko.CODES[code], block_tokens=block)
    pool.k.view(torch.uint8).fill_(0x7F - stale), pool.v.view(torch.uint8).fill_(0xFF - stale), pool.scale.fill_(255 - 100 * stale)
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    for i, m in enumerate(need):
        table[i, :m] = ids[sum(need[:i]):sum(need[:i]) + m]
    n = sum(lens)
    # heads and tokens of several sizes, so that scales differ
    size = torch.exp2(torch.randint(-3, 3, (n, hkv, 1), generator=g, device="cuda").float() / 2)
    k, v = (_randn(g, n, hkv, d, dtype=torch.float32).mul_(size).to(dt) for _ in range(2))
    if plant:
        plant(k, v)
    off, length = _i32(_cum(lens)), _i32(lens)
    pool.append(1, k, v, off, length, table)
    back = torch.empty_like(k), torch.empty_like(v)
    pool.read(1, *back, off, length, table)
    assert int(pool.err.item()) == 0
    q = _randn(g, sum(ql), hq, d, dtype=dt, scale=1.5)
    ng = len(prefix)
    args = (q, pool, 1, _i32(_cum(ql)), _i32(_cum(per)), table[:ng], _i32(prefix), table[ng:], _i32(own), 1 / math.sqrt(d))
    return pool, args, back, dt


def _reference(case, args, back):
    prefix, per, own, ql = case[8:]
    at, pre, seqs, qo, group = _cum(prefix + own), len(prefix), [], _cum(ql), _cum(per)
    for x in range(pre):
        pk, pv = (t[at[x]:at[x + 1]] for t in back)
        for r in range(group[x], group[x + 1]):
            ok, ov = (t[at[pre + r]:at[pre + r + 1]] for t in back)
            lim = (torch.arange(ql[r], device="cuda") + own[r] - ql[r] + 1).clamp(min=0)
            if ql[r]:
                seqs.append((qo[r], ql[r], [(pk, pv, torch.full((ql[r],), prefix[x], device="cuda")), (ok, ov, lim)]))
    return so.many(args[0], seqs, case[3], args[-1])


@pytest.mark.parametrize("name", CASES)
def test_attention(name):
    case = CASES[name]
    say(f"[case] 8-bit attention {name}")
    pool, args, back, dt = _setup(case, 21)
    q, d = args[0], case[4]
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    out = torch.full_like(q, math.nan)
    serve.attend_shared(*args, out=out, lse=lse)
    assert int(pool.err.item()) == 0
    so.check(out.reshape(-1, d), lse.reshape(-1), _reference(case, args, back), dt, name)
    ws = serve.shared_workspace(q, pool, args[4], args[5], args[7])
    assert torch.equal(serve.attend_shared(*args, ws=ws), out)
    # other codes behind the ends, other scales of blocks without tokens
    assert torch.equal(serve.attend_shared(*_setup(case, 21, stale=1)[1]), out)
    # strided queries, heads before tokens in the output
    wide = torch.empty(q.shape[0], q.shape[1] + 2, d, dtype=dt, device="cuda")
    wide[:, 1:-1].copy_(q)
    o = torch.empty(q.shape[1], q.shape[0], d, dtype=dt, device="cuda").transpose(0, 1)
    serve.attend_shared(wide[:, 1:-1], *args[1:], out=o)
    assert torch.equal(o, out)


PLACES = {  # keys that are not finite: of the prefixes and own tokens in their order
    "one": [129, 130, 137, 150], "uneven": [64, 66, 80, 242], "pairs": [49, 55, 70, 79, 83, 95], "tiles": [3, 69, 369, 400, 429, 470, 559],
    "tiles-64": [1499, 1500, 1700, 1799, 1800, 2089], "whole": [76, 77, 150, 226, 300], "whole-wide": [2499, 3399, 3500, 3799, 4000, 4553],
    "whole-wide-64": [1299, 1300, 1700, 1999, 2010, 2689], "decode": [2999, 3000, 3010], "long-own": [39, 4038, 4039],
}


@pytest.mark.parametrize("name", PLACES)
def test_not_finite(name):
    """A NaN or infinity among the values reaches the rows that see its token, and no others: those are what they are with 0
    in its place, bit for bit."""
    case = CASES[name]
    code, hq, hkv = case[1], case[2], case[3]
    prefix, per, own, ql = case[8:]
    n = sum(prefix) + sum(own)
    bad = torch.zeros(n, hkv, case[4], dtype=torch.bool, device="cuda")
    for i, t in enumerate(PLACES[name]):
        for h in {0, hkv - 1}:
            bad[t, h, 3 * i:3 * i + 2] = True
    say(f"[case] 8-bit attention {name}, values that are not finite")

    def plant(value):
        def do(k, v):
            v.masked_fill_(bad, value)
        return do

    clean = serve.attend_shared(*_setup(case, 5, plant(0.0))[1])
    at, pre, qo, group, g = _cum(prefix + own), len(prefix), _cum(ql), _cum(per), hq // hkv
    hit = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    for x in range(pre):
        for r in range(group[x], group[x + 1]):
            seen_prefix = bad[at[x]:at[x + 1]].any(0)
            mine = bad[at[pre + r]:at[pre + r + 1]]
            for t in range(ql[r]):
                lim = max(0, own[r] - ql[r] + t + 1)
                hit[qo[r] + t] = (seen_prefix | mine[:lim].any(0)).repeat_interleave(g, 0)
    assert bool(hit.any()) and not bool(hit.all())
    for value in (math.nan, math.inf) if code == "e5m2" else (math.nan,):
        out = serve.attend_shared(*_setup(case, 5, plant(value))[1])
        assert torch.equal(out[~hit], clean[~hit])
        assert not bool(torch.isfinite(out[hit].float()).any())


@pytest.mark.parametrize("name", ["one", "pairs", "tiles", "whole", "whole-wide-64"])
def test_keys_not_finite(name):
    """A key that is not finite makes the rows that see it so; the others do not change."""
    case = CASES[name]
    prefix, per, own, ql = case[8:]
    t = sum(prefix) + own[0] - 1 - (ql[0] > 1) * (ql[0] // 2)  # among the first request's own
    say(f"[case] 8-bit attention {name}, a key that is not finite")

    def plant(k, v):
        k[t] = math.nan

    def zero(k, v):
        k[t] = 0

    clean, out = (serve.attend_shared(*_setup(case, 6, x)[1]) for x in (zero, plant))
    hit = torch.zeros(clean.shape[0], dtype=torch.bool, device="cuda")
    for r in range(ql[0]):
        hit[r] = own[0] - ql[0] + r + 1 > t - sum(prefix)
    assert torch.equal(out[~hit], clean[~hit]) and bool(torch.isnan(out[hit].float()).all())


def test_largest_scales():
    """Codes at the ends of the types: keys and values as large and as small as their scales allow."""
    say("[case] 8-bit attention, large and small scales")
    for name, code, big in (("bf16", "e4m3", 2.0 ** 100), ("bf16", "e5m2", 2.0 ** -110), ("f16", "e4m3", 2.0 ** 14), ("f16", "e5m2", 2.0 ** -12)):
        case = (name, code, 4, 2, 64, 16, 16, "head", [90], [2], [30, 5], [3, 1])

        def plant(k, v):
            v.mul_(big / v.float().abs().amax()).to(v.dtype)

        pool, args, back, dt = _setup(case, 8, plant)
        out = serve.attend_shared(*args)
        o, _, mag, reach = _reference(case, args, back)
        # as serve_oracle.check, relative to the values' size; below 2^-14 float16 rounds to multiples of 2^-24
        tol = so.UNIT[dt] * (mag + np.abs(o)) * 1.02 + 2.0 ** -14 * mag + 2.0 ** -18 * reach[:, None] * mag + (2.0 ** -25 if name == "f16" else 0)
        if name == "f16":
            tol = tol + 2.0 ** -24 * mag  # weights below 2^-14 of the largest
        assert np.all(np.abs(so.f64(out).reshape(o.shape) - o) <= tol), (name, code)


def test_device_side_problems():
    case = CASES["one"][:8] + ([40], [2], [20, 20], [1, 1])
    pool, args, _, _ = _setup(case, 14)
    good = serve.attend_shared(*args)
    assert int(pool.err.item()) == 0
    say("[case] 8-bit attention, a length past its table")
    long = list(args)
    long[8] = _i32([20, 4000])
    got = serve.attend_shared(*long)
    assert int(pool.err.item()) == B.CR_ERR_SEQ and torch.equal(got[:1], good[:1])
    pool.err.zero_()
    bad = list(args)
    bad[7] = args[7].clone()
    bad[7][1, 0] = pool.num_pages
    say("[case] 8-bit attention, a page out of range")
    got = serve.attend_shared(*bad)
    assert int(pool.err.item()) == B.CR_ERR_PAGE and torch.equal(got[:1], good[:1])


def test_offsets_past_32_bits():
    """Pages whose codes and scales lie beyond 2^32 bytes and 2^31 pairs of scales."""
    hkv, d, pt, n = 8, 64, 1024, 2500
    say("[case] 8-bit attention, offsets past 32 bits")
    pages = (1 << 32) // (hkv * d * pt) + 30
    g = _gen(4)
    k, v = _randn(g, n, hkv, d, dtype=torch.bfloat16), _randn(g, n, hkv, d, dtype=torch.bfloat16)
    q = _randn(g, 3, 16, d, dtype=torch.bfloat16)
    out = []
    for count, ids in ((pages, [pages - 1, pages - 9, 1]), (3, [0, 1, 2])):
        pool = serve.QuantPagePool.empty(1, count, hkv, pt, d, block_tokens=1)
        table = _i32([ids])
        pool.append(0, k, v, _i32([0, n]), _i32([n]), table)
        out.append(serve.attend_shared(q, pool, 0, _i32([0, 3]), _i32([0, 1]), table, _i32([0]), table, _i32([n]), 0.125))
        assert int(pool.err.item()) == 0
    assert torch.equal(*out) and bool(out[0].isfinite().all())


def test_a_step_captured_and_on_another_stream():
    """Positions, append and attention as a decode step runs them: captured and replayed on other inputs with eager work
    between, and on a stream of its own, against the eager result."""
    say("[case] 8-bit step, captured")
    name, code, hq, hkv, d, pg, block, order, prefix, per, own, ql = case = CASES["decode"]
    pool, args, _, dt = _setup(case, 3)
    q, qo, go, ptab, plen, otab, olen, scale = args[0], args[3], args[4], args[5], args[6], args[7], args[8], args[9]
    n, g = q.shape[0], _gen(77)
    rot = serve.Rotary(d, layout="half")
    k, v = _randn(g, n, hkv, d, dtype=dt), _randn(g, n, hkv, d, dtype=dt)
    pos = olen + prefix[0] - 1
    q_turned, k_turned, out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    ws = serve.shared_workspace(q, pool, go, ptab, otab)

    def step(out, ws=None, stream=None):
        rot.apply(q, k, pos, q_turned, k_turned, stream=stream)
        pool.append(1, k_turned, v, qo, olen, otab, stream=stream)
        return serve.attend_shared(q_turned, pool, 1, qo, go, ptab, plen, otab, olen, scale, out=out, ws=ws, stream=stream)

    step(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    codes = pool.k.view(torch.uint8), pool.v.view(torch.uint8), pool.scale
    side = torch.cuda.Stream()
    for i in range(4):
        q.copy_(_randn(g, *q.shape, dtype=dt, scale=1.5))
        k.copy_(_randn(g, *k.shape, dtype=dt, scale=2.0 ** i))
        before = [t.clone() for t in codes]
        graph.replay()
        torch.cuda.synchronize()
        got, after = out.clone(), [t.clone() for t in codes]
        for t, x in zip(codes, before):
            t.copy_(x)
        assert torch.equal(step(None), got) and all(torch.equal(*x) for x in zip(codes, after))
        for t, x in zip(codes, before):
            t.copy_(x)
        side.wait_stream(torch.cuda.current_stream())
        other = step(None, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(other, got) and all(torch.equal(*x) for x in zip(codes, after))
    assert int(pool.err.item()) == 0
