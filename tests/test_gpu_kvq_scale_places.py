"""Scales whose places pass 32 bits."""
import pytest
import torch

from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_scales_past_32_bits(d):
    """A cache whose pages are close together in memory and have a scale for every token of a head: pages whose pairs of scales lie
    beyond the 2^32nd. Writing, reading, attention of few rows and by tiles, and page copies are those of a small cache, and attention
    is that of the tokens read back."""
    say(f"[case] 8-bit calls, scales past 32 bits, heads of {d}")
    heads, pt, n, g = 8, 128, 300, _gen(d)
    pages = (1 << 22) + 20000
    page = heads * pt * d  # bytes; 16 apart: pages 8,192 apart do not overlap

    def close(count, apart):
        strides = (0, apart, pt * d, d, 1)
        return [torch.zeros(count * apart + page, dtype=torch.uint8, device="cuda").as_strided((1, count, heads, pt, d), strides).view(torch.float8_e4m3fn)
                for _ in range(2)]

    k, v = _randn(g, n, heads, d, dtype=torch.bfloat16), _randn(g, n, heads, d, dtype=torch.bfloat16, scale=9.0)
    few, many = (_randn(g, m, 16, d, dtype=torch.bfloat16, scale=1.5) for m in (3, 200))
    zero, off, length = _i32([0]), _i32([0, n]), _i32([n])
    runs = []
    for count, apart, ids, to in ((pages, 16, [pages - 1, pages - 9000, 17], pages - 18000), (4, page, [0, 1, 2], 3)):
        scale = torch.empty(1, count, heads, pt, 2, dtype=torch.uint8, device="cuda")
        pool = serve.QuantPagePool(*close(count, apart), scale, torch.zeros(count, dtype=torch.int32, device="cuda"))
        assert pool.block_tokens == 1 and (count < 5 or min(ids[:2] + [to]) * heads * pt >= 1 << 32)
        table = _i32([ids])
        pool.append(0, k, v, off, length, table)
        back = torch.empty_like(k), torch.empty_like(v)
        pool.read(0, *back, off, length, table)
        outs = [serve.attend_shared(q, pool, 0, _i32([0, len(q)]), _i32([0, 1]), table, zero, table, length, 0.125) for q in (few, many)]
        outs.append(serve.attend_shared(few, pool, 0, _i32([0, 3]), _i32([0, 1]), table, length, table[:, :0].contiguous(), zero, 0.125))
        pool.copy(table[0, 1:2].contiguous(), _i32([to]))
        held = [scale[0, x].clone() for x in ids[:2] + [to]] + [pool.k[0, x].view(torch.uint8).clone() for x in ids[:2] + [to]]
        assert torch.equal(held[1], held[2]) and torch.equal(held[4], held[5]) and int(pool.err.item()) == 0
        runs.append([*back, *outs, *held])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    back = runs[0][:2]
    for q, out in zip((few, many), runs[0][2:4]):
        lim = torch.arange(len(q), device="cuda") + n - len(q) + 1
        so.check(out.reshape(-1, d), None, so.many(q, [(0, len(q), [(*back, lim)])], heads, 0.125), torch.bfloat16)
