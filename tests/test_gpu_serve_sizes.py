"""The attention calls at the sizes that take each of their forms: tiles of 256 and of 128 rows, few rows with
shares that end inside sequences, keys split over workgroups and joined, more sequences than a block looks at
at once, and offsets past 32 bits."""
import math

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


PROMPTS = [
    # dtype, heads, key heads, dim, query lengths, key lengths, causal
    ("bf16", 64, 8, 128, [1100, 1], [1100, 1], True),             # tiles of 256 rows
    ("f16", 32, 32, 64, [1300], [1300], True),                    # the same, one query head per key head
    ("bf16", 16, 2, 64, [700, 250], [1500, 2333], True),          # 256 rows, keys split
    ("f16", 24, 8, 128, [300], [2500], False),
    ("bf16", 4, 4, 128, [333, 64, 129], [333, 64, 129], True),    # tiles of 128 rows
    ("f16", 8, 1, 64, [20], [20000], True),                       # few blocks, many parts
    ("bf16", 2, 2, 128, [1], [70001], False),                     # one row
    ("f16", 64, 8, 64, [8], [9000], True),                        # 64 rows a key head by pairs
    ("bf16", 8, 8, 64, [1] * 700, [i % 97 for i in range(700)], True),
    ("f16", 16, 1, 128, [3] * 300, [(i * 37) % 500 for i in range(300)], True),
]


@pytest.mark.parametrize("case", PROMPTS, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-{len(c[4])}seq-{max(c[5])}" for c in PROMPTS])
def test_prompt(case):
    name, hq, hkv, d, ql, kl, causal = case
    dt, g, scale = DT[name], _gen(sum(ql) + sum(kl)), 1 / math.sqrt(d)
    q, k, v = (_randn(g, n, h, d, dtype=dt, scale=x) for n, h, x in ((sum(ql), hq, 1.5), (sum(kl), hkv, 1.0), (sum(kl), hkv, 1.0)))
    qo, ko = _cum(ql), _cum(kl)
    say(f"[case] prompt {case[:4]} {len(ql)} sequences")
    lse = torch.empty(q.shape[:2], device="cuda")
    ws = serve.prompt_workspace(q, k, _i32(qo))
    out = serve.attend_prompt(q, k, v, _i32(qo), _i32(ko), scale, lse=lse, causal=causal, ws=ws)
    assert int(ws.err.item()) == 0
    seqs = []
    for a, n, b, m in zip(qo, ql, ko, kl):
        lim = torch.arange(n, device="cuda") + m - n + 1 if causal else torch.full((n,), m, device="cuda")
        seqs.append((a, n, [(k[b:b + m], v[b:b + m], lim)]))
    so.check(out.reshape(-1, d), lse.reshape(-1), so.many(q, seqs, hkv, scale), dt, str(case[:4]))
    assert torch.equal(out, serve.attend_prompt(q, k, v, _i32(qo), _i32(ko), scale, causal=causal))


SHARED = [
    # dtype, heads, key heads, dim, page, order, prefix lengths, requests per group, own lengths, query lengths
    ("bf16", 64, 8, 128, 16, "head", [1500], [40], [70 + i for i in range(40)], [1] * 40),      # wide prefix, few own rows
    ("f16", 64, 8, 64, 8, "token", [6000], [200], [1 + i % 9 for i in range(200)], [1] * 200),  # 256-row prefix tiles
    ("bf16", 32, 8, 128, 32, "token", [2100, 700], [3, 2], [350, 80, 200, 33, 400], [350, 80, 200, 33, 390]),  # prefix read again
    ("f16", 8, 2, 64, 4, "head", [333, 1, 0], [1, 1, 1], [64, 65, 70], [64, 65, 60]),
    ("bf16", 16, 2, 64, 16, "head", [900], [4], [60, 40, 30, 20], [12, 10, 8, 9]),               # own tiles of 128 rows
    ("f16", 8, 8, 128, 2, "token", [40 + i for i in range(300)], [1] * 300, [1 + i % 5 for i in range(300)], [1] * 300),
    ("bf16", 6, 1, 128, 64, "head", [5000, 3], [9, 300], [5] * 309, [1] * 309),                  # a group of 1,800 rows
    ("f16", 40, 1, 64, 16, "token", [3000], [2], [2000, 7], [2, 1]),
    ("bf16", 8, 1, 64, 128, "head", [100], [1], [50000], [4]),
]


def _shared(case, poison):
    name, hq, hkv, d, pg, order, prefix, per, own, ql = case
    dt, g = DT[name], _gen(len(own))
    need = [-(-n // pg) for n in prefix + own]
    pages, width = sum(need) + 2, max(need)
    pool = serve.PagePool.empty(1, pages, hkv, pg, d, dt, order=order)
    pool.k.fill_(poison), pool.v.fill_(poison)
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table, at, kv = torch.full((len(need), width), -1, dtype=torch.int32, device="cuda"), 0, []
    for i, (n, m) in enumerate(zip(prefix + own, need)):
        table[i, :m] = ids[at:at + m]
        at += m
        kv.append((_randn(g, n, hkv, d, dtype=dt), _randn(g, n, hkv, d, dtype=dt)))
    lens = prefix + own
    pool.append(0, torch.cat([x[0] for x in kv]), torch.cat([x[1] for x in kv]), _i32(_cum(lens)), _i32(lens), table)
    q = _randn(g, sum(ql), hq, d, dtype=dt, scale=1.5)
    return pool, q, table[:len(prefix)].contiguous(), table[len(prefix):].contiguous(), kv


@pytest.mark.parametrize("case", SHARED, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-{c[5]}-{max(c[6])}-{len(c[8])}req" for c in SHARED])
def test_shared(case):
    name, hq, hkv, d, pg, order, prefix, per, own, ql = case
    dt, scale = DT[name], 1 / math.sqrt(d)
    pool, q, ptab, otab, kv = _shared(case, math.nan)
    go, qo = _cum(per), _cum(ql)
    lse = torch.empty(q.shape[:2], device="cuda")
    say(f"[case] shared {case[:6]} {len(prefix)} groups {len(own)} requests")
    args = (q, pool, 0, _i32(qo), _i32(go), ptab, _i32(prefix), otab, _i32(own), scale)
    out = serve.attend_shared(*args, lse=lse)
    assert int(pool.err.item()) == 0
    seqs = []
    for x, (a, b) in enumerate(zip(go, go[1:])):
        for r in range(a, b):
            n = ql[r]
            (pk, pv), (ok, ov) = kv[x], kv[len(prefix) + r]
            seqs.append((qo[r], n, [(pk, pv, torch.full((n,), prefix[x], device="cuda")), (ok, ov, torch.arange(n, device="cuda") + own[r] - n + 1)]))
    so.check(out.reshape(-1, d), lse.reshape(-1), so.many(q, seqs, hkv, scale), dt, str(case[:6]))
    assert torch.equal(out, serve.attend_shared(*args))


def test_prompt_keys_past_32_bits():
    """Keys and values of 2^32 elements and more: the last sequence's rows lie beyond."""
    n, hkv, d, last = 4_400_000, 8, 128, 3001
    k, v = (torch.empty(n, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert (n - last) * hkv * d > 1 << 32
    g = _gen(3)
    for x in (k, v):
        x[n - last:] = _randn(g, last, hkv, d, dtype=torch.bfloat16)
    q = _randn(g, 40, 16, d, dtype=torch.bfloat16)
    say("[case] prompt past 2^32 elements")
    out = serve.attend_prompt(q, k, v, _i32([0, 0, 40]), _i32([0, n - last, n]), 0.09)
    ref = so.many(q, [(0, 40, [(k[n - last:], v[n - last:], torch.arange(40, device="cuda") + last - 39)])], hkv, 0.09)
    so.check(out.reshape(-1, d), None, ref, torch.bfloat16)


def test_cache_past_32_bits():
    """Pages whose places lie beyond 2^32 elements: append, attend, fork and compact there."""
    pages, pt, hkv, d = 40_000, 128, 8, 128
    pool = serve.PagePool.empty(1, pages, hkv, pt, d)
    assert (pages - 10) * pt * hkv * d > 1 << 32
    g = _gen(4)
    table = _i32([[pages - 1, pages - 7, pages - 3]])
    pool.refs[table.long().flatten()] = 1
    n = 300
    k, v = (_randn(g, n, hkv, d, dtype=torch.bfloat16) for _ in range(2))
    say("[case] cache past 2^32 elements")
    pool.append(0, k, v, _i32([0, n]), _i32([n]), table)
    q = _randn(g, 2, 16, d, dtype=torch.bfloat16)
    child = torch.empty(1, 3, dtype=torch.int32, device="cuda")
    pool.refs[:pages - 9] += 1  # what is free lies at the end
    pool.fork(table, _i32([0]), _i32([290]), child)
    assert child.tolist() == [[pages - 1, pages - 7, pages - 9]]
    args = (_i32([0, 1, 2]), _i32([0, 1, 2]), torch.cat([table, child]), _i32([n, 290]), _i32([[0], [0]]), _i32([0, 0]), 0.09)
    out = serve.attend_shared(q, pool, 0, *args)
    rows = [(i, 1, [(k[:m], v[:m], torch.full((1,), m, device="cuda"))]) for i, m in enumerate((n, 290))]
    ref = so.many(q, rows, hkv, 0.09)
    so.check(out.reshape(-1, d), None, ref, torch.bfloat16)
    pool.refs[:pages - 9] -= 1
    both = torch.cat([table, child])
    pool.compact(both, _i32([n, 290]))
    assert both.tolist() == [[3, 1, 2], [3, 1, 0]] and int(pool.err.item()) == 0
    out = serve.attend_shared(q, pool, 0, *args[:2], both, *args[3:])
    so.check(out.reshape(-1, d), None, ref, torch.bfloat16)


def test_offsets_that_do_not_cover_are_reported():
    g = _gen(6)
    q, k = _randn(g, 30, 4, 64, dtype=torch.bfloat16), _randn(g, 30, 4, 64, dtype=torch.bfloat16)
    for qo in ([0, 10, 29], [1, 10, 30], [0, 31, 30]):
        ws = serve.prompt_workspace(q, k, _i32(qo))
        say(f"[case] prompt offsets {qo}")
        serve.attend_prompt(q, k, k, _i32(qo), _i32([0, 10, 30]), 0.1, ws=ws)
        assert int(ws.err.item()) == B.CR_ERR_SEQ
    case = ("bf16", 4, 4, 64, 16, "head", [20, 30], [2, 2], [40, 40, 40, 40], [40, 40, 40, 40])
    for ql in ([40] * 4, [1] * 4):  # the prefix read again, and joined
        pool, q, ptab, otab, _ = _shared(case[:9] + (ql,), 0.0)
        for go in ([0, 2, 3], [1, 2, 4], [0, 5, 4]):
            pool.err.zero_()
            say(f"[case] groups {go}, {ql[0]} queries")
            serve.attend_shared(q, pool, 0, _i32(_cum(ql)), _i32(go), ptab, _i32([20, 30]), otab, _i32([40] * 4), 0.1)
            assert int(pool.err.item()) == B.CR_ERR_SEQ


def test_offsets_out_of_order_stop_the_call():
    """Rows counted again and again by offsets that go back: more units than 32 bits hold, none is worked on."""
    n, total_k = 4096, 65536
    q = torch.zeros(32768, 8, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(total_k, 1, 64, dtype=torch.bfloat16, device="cuda")
    qo, ko = [32768 * (i % 2) for i in range(n + 1)], [total_k * (i % 2) for i in range(n + 1)]
    ws = serve.prompt_workspace(q, k, _i32(qo))
    say("[case] prompt offsets out of order, 4,096 sequences")
    serve.attend_prompt(q, k, k, _i32(qo), _i32(ko), 0.1, ws=ws)
    assert int(ws.err.item()) == B.CR_ERR_SEQ


def test_many_small_weights_in_sixteen_bit_floats():
    """60,000 keys of weight 2^-26 beside one of 1: below what a 16-bit float near 1 resolves, together 2^-10.
    The weights are exact, the output's rounding is 2^-11 of it, the scores' (26 in 24 bits) 2^-19."""
    n, d = 60001, 64
    q = torch.zeros(1, 1, d, dtype=torch.float16, device="cuda")
    k = torch.zeros(n, 1, d, dtype=torch.float16, device="cuda")
    v = torch.ones(n, 1, d, dtype=torch.float16, device="cuda")
    q[..., 0], k[0, 0, 0], v[0] = 1.0, 26.0, 0.0
    rest = (n - 1) * 2.0 ** -26
    for rows in (1, 300):  # few rows, and tiles of rows
        say(f"[case] small weights, {rows} rows")
        out = serve.attend_prompt(q.expand(rows, 1, d).contiguous(), k, v, _i32([0, rows]), _i32([0, n]), math.log(2.0), causal=False)
        assert (out.double() / (rest / (1 + rest)) - 1).abs().max() <= 2.0 ** -10


def test_offsets_out_of_order_write_nothing():
    """Few rows: query offsets that go back stop the call whether the sequence's key offsets fit or not."""
    g = _gen(12)
    q, k = _randn(g, 30, 4, 64, dtype=torch.bfloat16), _randn(g, 50, 4, 64, dtype=torch.bfloat16)
    for ko in ([0, 10, 20, 50], [0, 10, 60, 50], [0, 10, 5, 50]):
        qo = [0, 20, 10, 30]
        ws = serve.prompt_workspace(q, k, _i32(qo))
        out = torch.full_like(q, 7.0)
        say(f"[case] prompt offsets {qo}, keys {ko}")
        serve.attend_prompt(q, k, k, _i32(qo), _i32(ko), 0.1, out=out, ws=ws)
        assert int(ws.err.item()) == B.CR_ERR_SEQ and bool((out == 7.0).all())
