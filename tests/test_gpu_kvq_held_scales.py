"""Scales that a cache brings along: new tokens of a block are rounded under any that a byte holds, the largest too."""
import numpy as np
import pytest
import torch

from paper_2608_19677_amd import serve

import kvq_oracle as ko
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("name,code", [("bf16", "e4m3"), ("bf16", "e5m2"), ("f16", "e4m3"), ("f16", "e5m2")])
@pytest.mark.parametrize("stored", [1, 247, 248, 253, 254])
def test_tokens_behind_a_given_scale(name, code, stored):
    """Tokens in a block whose tokens from before have a scale of 2^(stored - 127): codes are x 2^-e with the block's e where it is
    the larger one, bit for bit, values that are not finite among them, and read back they are c 2^e rounded to the type."""
    say(f"[case] 8-bit append of {name} behind a scale of {stored}, {code}")
    dt, g, heads, d, had, new = ko.DT[name], _gen(stored), 2, 64, 5, 9
    pool = serve.QuantPagePool.empty(1, 3, heads, 16, d, dt, codes=ko.CODES[code])
    pool.scale.fill_(stored)
    for t in (pool.k, pool.v):  # codes of 0 to 1.5
        t.copy_((torch.randint(0, 4, t.shape, generator=g, device="cuda").float() / 2).to(t.dtype))
    size = torch.exp2(torch.randint(105, 128, (new, heads, d), generator=g, device="cuda").float() if name == "bf16"
                      else torch.randint(-14, 15, (new, heads, d), generator=g, device="cuda").float())
    rows = [((torch.rand(size.shape, generator=g, device="cuda") + 1) * size).to(dt).clamp(-torch.finfo(dt).max, torch.finfo(dt).max) for _ in range(2)]
    rows[1][2, 1, 3], rows[1][3, 0, 4], rows[0][0, 0, 0] = float("inf"), float("nan"), -torch.finfo(dt).max
    table, off, length = _i32([[2]]), _i32([0, new]), _i32([had + new])
    want = ko.Cache(pool)
    pool.append(0, *rows, off, length, table)
    want.append([x.double().cpu().numpy() for x in rows], [0, new], [had + new], [[2]])
    got = ko.Cache(pool)
    for j in range(2):
        assert np.array_equal(got.exps[j], want.exps[j])
        assert np.array_equal(got.codes[j], want.codes[j], equal_nan=True)
    back = [torch.empty(had + new, heads, d, dtype=dt, device="cuda") for _ in range(2)]
    pool.read(0, *back, _i32([0, had + new]), length, table)
    for j in range(2):
        ref = torch.from_numpy(want.tokens(j, [2], had + new)).to(dt)
        same = (back[j].cpu() == ref) | (back[j].cpu().isnan() & ref.isnan())
        assert bool(same.all())
    assert int(pool.err.item()) == 0
    if stored == 254 and name == "bf16":  # large elements have codes of their own under the largest scale
        assert len(np.unique(got.codes[0][2, had:had + new])) > 3
