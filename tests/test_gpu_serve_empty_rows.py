"""Rows that see no key give 0 and -inf in every form, whatever the values that they do not see hold."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


FORMS = {  # heads, key heads, dim, queries, keys: the last `keys` queries see some
    "few": (4, 4, 64, 40, 30),
    "few-split": (2, 1, 128, 30, 5),
    "tiles": (8, 2, 128, 90, 60),
    "tiles-64": (8, 8, 64, 200, 3),
    "wide": (64, 8, 128, 1200, 1100),
    "wide-part": (64, 8, 128, 1201, 1098),
}


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("form", FORMS)
def test_prompt(form, bad):
    hq, hkv, d, nq, nk = FORMS[form]
    g = torch.Generator(device="cuda").manual_seed(nq)
    q = torch.randn(nq, hq, d, generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(nk, hkv, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    args = (_i32([0, nq]), _i32([0, nk]), 1 / math.sqrt(d))
    clean = serve.attend_prompt(q, k, v, *args)
    v[:] = bad
    lse = torch.empty(nq, hq, device="cuda")
    say(f"[case] prompt rows without a key, {form}, values {bad}")
    out = serve.attend_prompt(q, k, v, *args, lse=lse)
    none = nq - nk
    assert bool((out[:none] == 0).all()) and bool((clean[:none] == 0).all()) and bool((lse[:none] == -math.inf).all())
    assert not bool(torch.isfinite(out[none:].float()).any())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("hq,hkv,nq,nk", [(4, 4, 8, 5), (8, 2, 60, 40), (8, 1, 300, 270)], ids=["few", "tiles", "whole"])
def test_shared(hq, hkv, nq, nk, bad):
    """No prefix, and more queries than own tokens."""
    d = 64
    g = torch.Generator(device="cuda").manual_seed(nq)
    q = torch.randn(nq, hq, d, generator=g, device="cuda").to(torch.bfloat16)
    pages = -(-nk // 16)
    pool = serve.PagePool.empty(1, pages, hkv, 16, d)
    pool.k.normal_(generator=g)
    pool.v.fill_(bad)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    lse = torch.empty(nq, hq, device="cuda")
    say(f"[case] shared rows without a key, {nq} queries, values {bad}")
    out = serve.attend_shared(q, pool, 0, _i32([0, nq]), _i32([0, 1]), torch.empty((1, 0), dtype=torch.int32, device="cuda"), _i32([0]),
                              table, _i32([nk]), 0.125, lse=lse)
    none = nq - nk
    assert bool((out[:none] == 0).all()) and bool((lse[:none] == -math.inf).all()) and int(pool.err.item()) == 0
    assert not bool(torch.isfinite(out[none:].float()).any())
