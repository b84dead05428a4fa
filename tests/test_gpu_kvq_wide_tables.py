"""Attention over the 8-bit cache with tables much wider than their rows, as a destination that serves any length passes them: shares and slots
come from the widths, the results from the lengths."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say
from test_gpu_kvq_attention import CASES, _reference, _setup

pytestmark = pytest.mark.gpu


def _wider(table, tokens, page):
    out = torch.full((table.shape[0], max(table.shape[1], tokens // page)), -1, dtype=torch.int32, device="cuda")
    out[:, :table.shape[1]] = table
    return out


@pytest.mark.parametrize("prefix_tokens,own_tokens", [(4096, 4096), (131072, 131072), (0, 1 << 20), (1 << 20, 0)])
@pytest.mark.parametrize("name", CASES)
def test_wide_tables(name, prefix_tokens, own_tokens):
    case = CASES[name]
    say(f"[case] 8-bit attention {name}, tables for {prefix_tokens} and {own_tokens} tokens")
    pool, args, back, dt = _setup(case, 31)
    args = list(args)
    args[5], args[7] = _wider(args[5], prefix_tokens, case[5]), _wider(args[7], own_tokens, case[5])
    q, d = args[0], case[4]
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    out = serve.attend_shared(*args, out=torch.full_like(q, math.nan), lse=lse)
    assert int(pool.err.item()) == 0
    so.check(out.reshape(-1, d), lse.reshape(-1), _reference(case, args, back), dt, name)
    assert torch.equal(serve.attend_shared(*args), out)
