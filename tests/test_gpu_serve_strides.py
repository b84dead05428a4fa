"""Keys and values whose rows lie up to 2^31 elements apart: products of rows and strides need 64 bits from the second
row on."""
import math

import pytest
import torch

from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

# rows of a wavefront lie 2^32 elements apart and more from 2^32 / 7 (heads of 64) and 2^32 / 3 (heads of 128)
FAR = {64: 613_566_760, 128: 1_431_655_768}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.fixture()
def space():
    """Memory for 33 rows of FAR[128] elements (66 of FAR[64]); only the rows are ever touched."""
    n = 33 * FAR[128]
    if torch.cuda.mem_get_info()[0] < 2 * n + (8 << 30):
        pytest.skip("not enough free memory")
    buf = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    yield buf
    del buf
    torch.cuda.empty_cache()


def _far(space, n, d, seed):
    """Keys and values [n, 1, d] at the stride, side by side, and a copy of each."""
    s = FAR[d]
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for at in (0, d):
        x = space.as_strided((n, 1, d), (s, d, 1), at)
        x.copy_(torch.randn((n, 1, d), generator=g, device="cuda").to(torch.bfloat16))
        out += [x, x.contiguous()]
    return out


@pytest.mark.parametrize("d,rows,keys", [(64, 1, 64), (64, 150, 65), (128, 2, 33)], ids=["few", "tiles", "dim128"])
def test_prompt(space, d, rows, keys):
    say(f"[case] prompt keys {FAR[d]} elements apart, {rows} rows")
    k, k0, v, v0 = _far(space, keys, d, rows)
    q = torch.randn(rows, 4, d, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(torch.bfloat16)
    scale = 1 / math.sqrt(d)
    got = serve.attend_prompt(q, k, v, _i32([0, rows]), _i32([0, keys]), scale, causal=False)
    near = serve.attend_prompt(q, k0, v0, _i32([0, rows]), _i32([0, keys]), scale, causal=False)
    assert torch.equal(got, near)
    ref = so.many(q, [(0, rows, [(k0, v0, torch.full((rows,), keys, device="cuda"))])], 1, scale)
    so.check(got.reshape(-1, d), None, ref, torch.bfloat16)


@pytest.mark.parametrize("rows", [1, 150], ids=["few", "tiles"])
def test_pages(space, rows):
    """One page of 64 tokens."""
    d, n = 64, 64
    say(f"[case] cached tokens {FAR[d]} elements apart, {rows} rows")
    k, k0, v, v0 = _far(space, n, d, 3)
    pages = lambda x: x.as_strided((1, 1, 1, 64, d), (0, 0, 0, FAR[d], 1))  # noqa: E731
    pool = serve.PagePool(pages(k), pages(v), _i32([1]))
    q = torch.randn(rows, 4, d, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(torch.bfloat16)
    args = (_i32([0, rows]), _i32([0, 1]), _i32([[0]]), _i32([n]), torch.empty((1, 0), dtype=torch.int32, device="cuda"), _i32([0]), 0.125)
    got = serve.attend_shared(q, pool, 0, *args)
    assert int(pool.err.item()) == 0
    ref = so.many(q, [(0, rows, [(k0, v0, torch.full((rows,), n, device="cuda"))])], 1, 0.125)
    so.check(got.reshape(-1, d), None, ref, torch.bfloat16)
