"""Calls of several rounds of blocks, whose sequences are taken by falling numbers of keys: equal and empty
sequences, as many sequences as a wavefront has lanes and one more, prefixes of groups, own tokens, whole requests."""
import math

import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say
from test_gpu_serve_sizes import DT, _cum, _gen, _i32, _randn, _shared

pytestmark = pytest.mark.gpu

PROMPTS = [
    # dtype, heads, key heads, dim, query lengths, key lengths, causal
    ("f16", 20, 20, 64, [300, 1, 0, 300, 77, 140, 300, 513], [300, 1, 0, 300, 500, 140, 300, 513], True),
    ("bf16", 32, 32, 64, [(i * 37) % 90 + 40 for i in range(64)], [(i * 37) % 90 + 40 for i in range(64)], True),
    ("bf16", 32, 32, 64, [(i * 37) % 90 + 40 for i in range(65)], [(i * 37) % 90 + 40 for i in range(65)], True),
    ("f16", 16, 16, 128, [700, 700, 700], [1400, 20, 1400], True),          # rows that see no key in the middle one
    ("bf16", 64, 8, 128, [400, 0, 700, 300], [1500, 900, 1100, 0], False),  # tiles of 256 rows
]


@pytest.mark.parametrize("case", PROMPTS, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-{len(c[4])}seq-{max(c[5])}" for c in PROMPTS])
def test_prompt(case):
    name, hq, hkv, d, ql, kl, causal = case
    dt, g, scale = DT[name], _gen(sum(ql) + 7 * sum(kl)), 1 / math.sqrt(d)
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


SHARED = [
    # dtype, heads, key heads, dim, page, order, prefix lengths, requests per group, own lengths, query lengths
    ("bf16", 32, 8, 128, 16, "head", [1500, 0, 700, 1500], [3, 2, 0, 9], [100 + 20 * i for i in range(14)], [100 + 20 * i for i in range(14)]),
    ("f16", 32, 16, 64, 32, "token", [130, 700, 65], [8, 40, 16], [40 + i for i in range(64)], [40 + i % 9 for i in range(64)]),
    ("bf16", 16, 16, 64, 16, "head", [600, 200, 0, 900], [90, 110, 130, 90], [3] * 420, [1] * 420),  # prefixes of many rows
    ("bf16", 128, 128, 64, 16, "head", [600, 200, 0, 900], [7, 9, 5, 7], [30] * 28, [10] * 28),      # the same, more blocks than a round
]


@pytest.mark.parametrize("case", SHARED, ids=[f"{c[0]}-{c[1]}x{c[2]}x{c[3]}-{len(c[8])}req" for c in SHARED])
def test_shared(case):
    name, hq, hkv, d, pg, order, prefix, per, own, ql = case
    dt, scale = DT[name], 1 / math.sqrt(d)
    pool, q, ptab, otab, kv = _shared(case, math.nan)
    go, qo = _cum(per), _cum(ql)
    lse = torch.empty(q.shape[:2], device="cuda")
    say(f"[case] shared {case[:6]} {len(prefix)} groups {len(own)} requests")
    out = serve.attend_shared(q, pool, 0, _i32(qo), _i32(go), ptab, _i32(prefix), otab, _i32(own), scale, lse=lse)
    assert int(pool.err.item()) == 0
    seqs = []
    for x, (a, b) in enumerate(zip(go, go[1:])):
        for r in range(a, b):
            n = ql[r]
            (pk, pv), (ok, ov) = kv[x], kv[len(prefix) + r]
            seqs.append((qo[r], n, [(pk, pv, torch.full((n,), prefix[x], device="cuda")), (ok, ov, torch.arange(n, device="cuda") + own[r] - n + 1)]))
    so.check(out.reshape(-1, d), lse.reshape(-1), so.many(q, seqs, hkv, scale), dt, str(case[:6]))


def test_offsets_that_do_not_fit_are_reported():
    """The others keep their results; empty sequences report too."""
    g = _gen(8)
    ql = [300, 0, 700, 400]
    qo, n = _cum(ql), sum(ql)
    q, k = _randn(g, n, 32, 64, dtype=torch.bfloat16), _randn(g, n, 32, 64, dtype=torch.bfloat16)
    want = serve.attend_prompt(q, k, k, _i32(qo), _i32(qo), 0.1)
    for ko, good in (([0, 300, n + 1, 1000, 1400], slice(0, 300)), ([0, 300, 300, 1000, 1401], slice(0, 1000))):
        ws = serve.prompt_workspace(q, k, _i32(qo))
        say(f"[case] key offsets {ko}")
        out = serve.attend_prompt(q, k, k, _i32(qo), _i32(ko), 0.1, ws=ws)
        assert int(ws.err.item()) == B.CR_ERR_SEQ and torch.equal(out[good], want[good])
    for bad in ([1, 300, 300, 1000, 1400], [0, 300, 300, 1000, 1399], [0, 0, 1500, 1000, 1400]):
        ws = serve.prompt_workspace(q, k, _i32(qo))
        say(f"[case] query offsets {bad}")
        serve.attend_prompt(q, k, k, _i32(bad), _i32(qo), 0.1, ws=ws)
        assert int(ws.err.item()) == B.CR_ERR_SEQ
