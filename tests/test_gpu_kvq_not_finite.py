"""Values that are not finite among keys that only some rows of a wavefront see, in elements all over the head: few rows over codes have
a head's elements in an order of their own, for heads of 64 another one than for 128."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

from cr_check import say
from test_gpu_kvq_attention import _cum, _setup

pytestmark = pytest.mark.gpu

NOT_FINITE = {
    # as CASES of test_gpu_kvq_attention.py, then keys that are not finite: of the prefixes and own tokens in their order
    "beside-tiles": (("bf16", "e4m3", 8, 2, 64, 16, 16, "head", [50], [3], [30, 16, 200], [7, 12, 15]), [49, 75, 79, 85, 95, 281, 290, 295]),
    "few": (("f16", "e5m2", 4, 4, 64, 8, 4, "token", [40, 0, 300], [1, 2, 1], [33, 20, 64, 500], [30, 9, 17, 24]),
            [39, 345, 372, 385, 392, 440, 456, 930, 940, 956]),
    "cut": (("bf16", "e5m2", 2, 2, 64, 16, 2, "head", [10], [1], [40000], [32]), [39979, 39990, 39999, 40009]),
    "many-tiles": (("f16", "e4m3", 6, 2, 64, 32, 32, "token", [70] * 3, [1] * 3, [400, 333, 290], [10, 7, 3]), [69, 601, 605, 609, 938, 942, 1232]),
    "pairs": (("bf16", "e5m2", 8, 2, 128, 8, 8, "head", [50], [2], [30, 400], [14, 16]), [49, 66, 70, 79, 465, 470, 479]),
}


@pytest.mark.parametrize("name", NOT_FINITE)
def test_not_finite(name):
    """NaNs and infinities in elements all over the head reach the elements of the rows that see their tokens, and no others: those are what
    they are with 0 in their place, bit for bit."""
    case, places = NOT_FINITE[name]
    code, hq, hkv, d = case[1:5]
    prefix, per, own, ql = case[8:]
    bad = torch.zeros(sum(prefix) + sum(own), hkv, d, dtype=torch.bool, device="cuda")
    for i, t in enumerate(places):
        for h in {0, hkv - 1}:
            for j in range(d // 8):
                bad[t, h, (5 * i + 3 * h + 9 * j) % d] = True
    say(f"[case] 8-bit attention {name}, values that are not finite all over the head")

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
                hit[qo[r] + t] = (seen_prefix | mine[:max(0, own[r] - ql[r] + t + 1)].any(0)).repeat_interleave(g, 0)
    assert bool(hit.any()) and not bool(hit.all())
    for value in (math.nan, math.inf, -math.inf) if code == "e5m2" else (math.nan,):
        out = serve.attend_shared(*_setup(case, 5, plant(value))[1])
        assert torch.equal(out[~hit], clean[~hit])
        assert not bool(torch.isfinite(out[hit].float()).any())
