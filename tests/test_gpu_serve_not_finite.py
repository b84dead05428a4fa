"""Values that are not finite reach the rows that see them, and no others: rows before them in the same sequence
are what they are with 0 in their place, bit for bit, in every form of both calls."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _cum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _plant(v, places):
    """A NaN, +inf and -inf at the keys, in key head 0 (the last one too), at elements 0, 1 and 2 on."""
    bad = torch.zeros(v.shape, dtype=torch.bool, device="cuda")
    for i, t in enumerate(places):
        for h in {0, v.shape[1] - 1}:
            v[t, h, 3 * i % v.shape[2]], v[t, h, 3 * i % v.shape[2] + 1] = math.nan, (math.inf if i % 2 else -math.inf)
            bad[t, h, 3 * i % v.shape[2]:3 * i % v.shape[2] + 2] = True
    return bad


def _check(out, clean, hit):
    """hit: elements of outputs whose row sees a value there that is not finite."""
    assert torch.equal(out[~hit], clean[~hit])
    assert not bool(torch.isfinite(out[hit].float()).any())


def _hits(bad, q_off, k_off, group, causal, shape):
    hit = torch.zeros(shape, dtype=torch.bool, device="cuda")
    for a, e, b, f in zip(q_off, q_off[1:], k_off, k_off[1:]):
        seen = torch.cat([torch.zeros_like(bad[b:b + 1]), bad[b:f].cummax(0).values]) if f > b else torch.zeros_like(bad[:1])
        lim = (torch.arange(e - a, device="cuda") + (f - b) - (e - a) + 1).clamp(0, f - b) if causal else torch.full((e - a,), f - b, device="cuda")
        hit[a:e] = seen[lim].repeat_interleave(group, 1)
    return hit


PROMPTS = {
    # type, heads, key heads, dim, query lengths, key lengths, causal, keys that are not finite
    "few": ("bf16", 4, 4, 64, [40, 9], [40, 30], True, [0, 17, 39, 45, 69]),
    "few-pairs": ("f16", 8, 2, 128, [14, 16], [300, 16], True, [290, 293, 299, 305, 315]),
    "few-split": ("bf16", 2, 1, 128, [20], [5000], True, [100, 4981, 4990, 4999]),
    "tiles": ("f16", 8, 2, 128, [90, 33, 150], [90, 60, 150], True, [0, 40, 63, 64, 89, 120, 149, 160, 280, 299]),
    "tiles-64": ("bf16", 6, 6, 64, [333, 200], [333, 10], True, [5, 127, 128, 200, 332, 333, 342]),
    "tiles-split": ("bf16", 2, 2, 64, [200], [5000], True, [10, 4800, 4900, 4950, 4999]),
    "tiles-ends": ("f16", 8, 2, 64, [100, 70], [77, 101], False, [76, 77, 177]),
    "wide": ("bf16", 64, 8, 128, [1201, 3], [1201, 3], True, [0, 31, 500, 511, 900, 1199, 1200, 1203]),
    "wide-64": ("f16", 32, 32, 64, [1300], [1333], True, [40, 700, 1100, 1200, 1330]),
    "sorted": ("f16", 20, 20, 64, [300, 77, 140, 513], [300, 500, 140, 513], True, [7, 299, 450, 799, 801, 1000, 1400]),
}


@pytest.mark.parametrize("form", PROMPTS)
def test_prompt(form):
    name, hq, hkv, d, ql, kl, causal, places = PROMPTS[form]
    g, dt = _gen(len(places)), DT[name]
    q, k, v = _randn(g, sum(ql), hq, d, dtype=dt), _randn(g, sum(kl), hkv, d, dtype=dt), _randn(g, sum(kl), hkv, d, dtype=dt)
    qo, ko = _cum(ql), _cum(kl)
    bad = _plant(v, places)
    args = (_i32(qo), _i32(ko), 1 / math.sqrt(d))
    clean = serve.attend_prompt(q, k, torch.where(bad, 0, v), *args, causal=causal)
    say(f"[case] prompt, {form}, values that are not finite")
    _check(serve.attend_prompt(q, k, v, *args, causal=causal), clean, _hits(bad, qo, ko, hq // hkv, causal, q.shape))


SHARED = {
    # type, heads, key heads, dim, page, prefix, own lengths, query lengths, keys: of the prefix, then of all own tokens
    "few": ("bf16", 4, 4, 64, 8, 0, [40, 12], [40, 9], [], [3, 31, 39, 41, 51]),
    "few-pairs": ("f16", 8, 2, 128, 1, 50, [30, 16], [14, 16], [49], [5, 20, 29, 33, 45]),
    "tiles": ("bf16", 8, 2, 128, 16, 70, [60, 40], [60, 40], [3, 69], [0, 30, 59, 60, 99]),
    "whole": ("bf16", 32, 8, 128, 32, 77, [150, 100], [150, 80], [76], [0, 60, 149, 150, 249]),
    "whole-64": ("f16", 8, 8, 64, 2, 1500, [700, 690], [700, 690], [1, 1499], [0, 500, 699, 700, 1300, 1389]),
    "decode": ("f16", 16, 2, 64, 16, 90, [3, 500], [1, 1], [89], [2, 3, 400]),
}


@pytest.mark.parametrize("form", SHARED)
def test_shared(form):
    name, hq, hkv, d, pt, prefix, own, ql, in_prefix, in_own = SHARED[form]
    g, dt = _gen(len(in_own)), DT[name]
    need = [-(-n // pt) for n in [prefix] + own]
    pool = serve.PagePool.empty(1, sum(need) + 1, hkv, pt, d, dt)
    table = torch.full((3, max(need)), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(sum(need) + 1, generator=g, device="cuda").to(torch.int32)
    for i, m in enumerate(need):
        table[i, :m] = ids[sum(need[:i]):sum(need[:i]) + m]
    n, lens = prefix + sum(own), [prefix] + own
    k, v = _randn(g, n, hkv, d, dtype=dt), _randn(g, n, hkv, d, dtype=dt)
    bad = _plant(v, in_prefix + [prefix + x for x in in_own])
    q, off, qo = _randn(g, sum(ql), hq, d, dtype=dt), _i32(_cum(lens)), _cum(ql)
    args = (q, pool, 0, _i32(qo), _i32([0, 2]), table[:1], _i32([prefix]), table[1:], _i32(own), 1 / math.sqrt(d))
    pool.append(0, k, torch.where(bad, 0, v), off, _i32(lens), table)
    clean = serve.attend_shared(*args)
    pool.append(0, k, v, off, _i32(lens), table)
    say(f"[case] shared, {form}, values that are not finite")
    out = serve.attend_shared(*args)
    ko = [x + prefix for x in _cum(own)]
    hit = _hits(bad[prefix:], qo, _cum(own), hq // hkv, True, q.shape) | bad[:prefix].any(0).repeat_interleave(hq // hkv, 0)[None]
    assert ko[-1] == n and int(pool.err.item()) == 0
    _check(out, clean, hit)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("form", ["few", "few-split", "tiles", "tiles-64", "wide", "sorted"])
def test_prompt_keys(form, bad):
    """A key that is not finite makes the rows that see it so; the rows before it do not change."""
    name, hq, hkv, d, ql, kl, causal, places = PROMPTS[form]
    g, dt = _gen(len(places)), DT[name]
    q, k, v = _randn(g, sum(ql), hq, d, dtype=dt), _randn(g, sum(kl), hkv, d, dtype=dt), _randn(g, sum(kl), hkv, d, dtype=dt)
    qo, ko = _cum(ql), _cum(kl)
    args = (_i32(qo), _i32(ko), 1 / math.sqrt(d))
    clean = serve.attend_prompt(q, k, v, *args)
    at = torch.zeros(v.shape, dtype=torch.bool, device="cuda")
    at[places[2]] = True
    hit = _hits(at, qo, ko, hq // hkv, True, q.shape)
    k[places[2]] = bad
    say(f"[case] prompt, {form}, a key of {bad}")
    out = serve.attend_prompt(q, k, v, *args)
    assert torch.equal(out[~hit], clean[~hit]) and bool(torch.isnan(out[hit].float()).all())
