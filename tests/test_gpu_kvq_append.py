"""New tokens rounded into the 8-bit cache and read back, against the 64-bit statement: codes, scales and what was there
before, bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2608_19677_amd import serve

import kvq_oracle as ko
from cr_check import say

pytestmark = pytest.mark.gpu


def _cum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, n, heads, d, dt, spread=0.0):
    """Rows of random sizes: a token's and a head's by powers of two."""
    x = torch.randn((n, heads, d), generator=g, device="cuda")
    if spread:
        x = x * torch.exp2(torch.randint(-int(spread), int(spread) + 1, (n, heads, 1), generator=g, device="cuda").float())
    return x.to(dt)


def _pool(g, layers, pages, heads, pt, d, dt, code, order, block):
    pool = serve.QuantPagePool.empty(layers, pages, heads, pt, d, dt, order=order, codes=ko.CODES[code], block_tokens=block)
    for t in (pool.k, pool.v):  # what earlier calls left: any finite code
        c = torch.randint(0, 120, t.shape, generator=g, device="cuda", dtype=torch.uint8)
        t.view(torch.uint8).copy_(c)
    pool.scale.copy_(torch.randint(100, 140, pool.scale.shape, generator=g, device="cuda", dtype=torch.uint8))
    return pool


def _table(g, pages, need, width=None):
    """Rows of distinct pages anywhere, -1 behind them."""
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    t = torch.full((len(need), width or max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        t[i, :n] = ids[at:at + n]
        at += n
    return t


def _same(pool, want, layer=0):
    got = ko.Cache(pool, layer)
    for j in range(2):
        assert np.array_equal(got.exps[j], want.exps[j])
        assert np.array_equal(got.codes[j], want.codes[j], equal_nan=True)


CASES = [
    # type, code, heads, dim, page, block, order, tokens before, new tokens
    ("bf16", "e4m3", 1, 128, 16, 16, "head", [0], [1]),
    ("bf16", "e4m3", 2, 128, 16, 16, "head", [0, 5, 16, 15, 31, 3], [40, 1, 1, 2, 0, 13]),
    ("f16", "e5m2", 3, 64, 32, 8, "token", [7, 0, 1, 8], [1, 9, 30, 65]),
    ("bf16", "e5m2", 2, 128, 8, 1, "token", [3, 0, 8], [6, 1, 17]),            # a scale for each token
    ("f16", "e4m3", 5, 64, 4, 2, "head", [1, 2, 0, 9, 3], [1, 1, 5, 8, 0]),    # pages smaller than a wave's rows
    ("f16", "e4m3", 1, 128, 1, 1, "head", [0, 2], [3, 5]),                    # a page per token
    ("bf16", "e4m3", 2, 128, 256, 128, "head", [100, 0, 129], [60, 300, 1]),   # more rows than registers hold
    ("f16", "e5m2", 2, 64, 128, 128, "token", [127, 1], [2, 200]),
    ("bf16", "e4m3", 4, 64, 1024, 64, "head", [1000, 63], [40, 1]),
    ("f16", "e4m3", 8, 128, 16, 4, "token", list(range(70)), [1 + i % 3 for i in range(70)]),  # more sequences than lanes
]


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-p{c[4]}b{c[5]}{c[6][0]}" for c in CASES])
def test_append_and_read(case):
    name, code, heads, d, pt, block, order, had, new = case
    dt, g = ko.DT[name], _gen(pt + block + len(had))
    say(f"[case] 8-bit append {case}")
    length = [a + b for a, b in zip(had, new)]
    need = [-(-n // pt) for n in length]
    pool = _pool(g, 2, sum(need) + 3, heads, pt, d, dt, code, order, block)
    other = pool.k[0].view(torch.uint8).clone(), pool.scale[0].clone()
    table = _table(g, sum(need) + 3, need, max(need) + 2)
    k, v = _rows(g, sum(new), heads, d, dt, 9), _rows(g, sum(new), heads, d, dt, 2)
    want = ko.Cache(pool, 1)
    off = _cum(new)
    pool.append(1, k, v, _i32(off), _i32(length), table)
    want.append([x.double().cpu().numpy() for x in (k, v)], off, length, table.tolist())
    _same(pool, want, 1)
    assert torch.equal(other[0], pool.k[0].view(torch.uint8)) and torch.equal(other[1], pool.scale[0])  # the other layer
    # read back: all tokens, then those of the middle into strided rows
    ro = _cum(length)
    back = [torch.full((ro[-1] + 2, heads, d), math.nan, dtype=dt, device="cuda") for _ in range(2)]
    pool.read(1, back[0][:ro[-1]], back[1][:ro[-1]], _i32(ro), _i32(length), table)
    for j in range(2):
        ref = np.concatenate([want.tokens(j, row, n) for row, n in zip(table.tolist(), length)])
        ref = torch.from_numpy(ref).to(dt)
        assert torch.equal(back[j][:ro[-1]].cpu(), ref) and bool(back[j][ro[-1]:].isnan().all())
    part = [n // 2 for n in length]
    end = [n - n // 3 for n in length]
    part = [min(p, e) for p, e in zip(part, end)]
    po = _cum(part)
    if po[-1]:
        both = torch.full((po[-1], 3, heads, d), math.nan, dtype=dt, device="cuda")
        pool.read(1, both[:, 0], both[:, 2], _i32(po), _i32(end), table)
        for i, (p, e) in enumerate(zip(part, end)):
            for j in range(2):
                assert torch.equal(both[po[i]:po[i + 1], 2 * j], back[j][ro[i] + e - p:ro[i] + e])
        assert bool(both[:, 1].isnan().all())
        only = torch.full((po[-1], heads, d), math.nan, dtype=dt, device="cuda")
        pool.read(1, None, only, _i32(po), _i32(end), table)
        assert torch.equal(only, both[:, 2])
    assert int(pool.err.item()) == 0


@pytest.mark.parametrize("name,code", [("bf16", "e4m3"), ("bf16", "e5m2"), ("f16", "e4m3"), ("f16", "e5m2")])
def test_every_element(name, code):
    """Every value of the element type, in blocks of one and of 16 tokens: the largest and smallest, subnormals, NaN and
    infinities, alone and beside others."""
    dt, d = ko.DT[name], 128
    say(f"[case] every {name} as {code}")
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dt).view(512, 1, d).cuda()
    perm = torch.randperm(65536, generator=torch.Generator().manual_seed(3))
    y = x.flatten()[perm.cuda()].view(512, 1, d).contiguous()
    for block, rows in ((1, x), (16, x), (16, y)):
        pool = serve.QuantPagePool.empty(1, 32, 1, 16, d, dt, codes=ko.CODES[code], block_tokens=block)
        table = torch.arange(32, dtype=torch.int32, device="cuda")[None]
        off, length = _i32([0, 512]), _i32([512])
        pool.k.view(torch.uint8).zero_(), pool.v.view(torch.uint8).zero_()
        want = ko.Cache(pool)
        pool.append(0, rows, rows, off, length, table)
        r = rows.double().cpu().numpy()
        want.append([r, r], [0, 512], [512], table.tolist())
        _same(pool, want)
        back = torch.empty_like(rows)
        pool.read(0, back, None, off, length, table)
        ref = torch.from_numpy(want.tokens(0, table[0].tolist(), 512)).to(dt)
        same = (back.cpu() == ref) | (back.cpu().isnan() & ref.isnan())
        assert bool(same.all())
        finite = rows.isfinite()
        assert bool(back[finite].isfinite().all()) and not bool(back[~finite].isfinite().any())


def test_token_by_token():
    """A decode's tokens one at a time: growing scales move the codes there; and one at a time gives the scales of all at once."""
    dt, heads, d, pt, n = torch.bfloat16, 3, 128, 16, 37
    say("[case] 8-bit append, token by token")
    g = _gen(5)
    k, v = _rows(g, n, heads, d, dt, 6), _rows(g, n, heads, d, dt, 6)
    table = _table(g, 4, [3])
    for code in ("e4m3", "e5m2"):
        pool, whole = (serve.QuantPagePool.empty(1, 4, heads, pt, d, dt, codes=ko.CODES[code]) for _ in range(2))
        for p in (pool, whole):
            p.k.view(torch.uint8).zero_(), p.v.view(torch.uint8).zero_()
        want = ko.Cache(pool)
        for t in range(n):
            pool.append(0, k[t:t + 1], v[t:t + 1], _i32([0, 1]), _i32([t + 1]), table)
            want.append([x[t:t + 1].double().cpu().numpy() for x in (k, v)], [0, 1], [t + 1], table.tolist())
        _same(pool, want)
        whole.append(0, k, v, _i32([0, n]), _i32([n]), table)
        assert torch.equal(whole.scale, pool.scale)
        # again over the last tokens: the scales stay, the codes are the new tokens'
        pool.append(0, k[20:30] / 64, v[20:30] / 64, _i32([0, 10]), _i32([30]), table)
        want.append([(x[20:30] / 64).double().cpu().numpy() for x in (k, v)], [0, 10], [30], table.tolist())
        _same(pool, want)


def test_device_side_problems():
    """What only the device sees: bits of the error word; the sequences concerned are skipped, the others served."""
    dt, heads, d, pt = torch.bfloat16, 2, 64, 16
    say("[case] 8-bit append and read, sequences that do not fit")
    g = _gen(9)
    k, v = _rows(g, 12, heads, d, dt), _rows(g, 12, heads, d, dt)
    good = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32, device="cuda")

    def call(off, length, table, served):
        pool = _pool(g, 1, 6, heads, pt, d, dt, "e4m3", "head", 16)
        want = ko.Cache(pool)  # with the served sequences' tokens only
        for i in served:
            part = [x[off[i]:off[i + 1]].double().cpu().numpy() for x in (k, v)]
            want.append(part, [0, off[i + 1] - off[i]], [length[i]], table[i:i + 1].tolist())
        pool.append(0, k, v, _i32(off), _i32(length), table)
        bits = int(pool.err.item())
        _same(pool, want)
        pool.err.zero_()
        out = torch.full((12, heads, d), 7.0, dtype=dt, device="cuda")
        pool.read(0, out, None, _i32(off), _i32(length), table)
        assert int(pool.err.item()) == bits
        for i in range(3):
            a, e = off[i], off[i + 1]
            if i in served:
                ref = want.tokens(0, table[i].tolist(), length[i])[length[i] - (e - a):]
                assert np.array_equal(out[a:e].double().cpu().numpy(), ref)
            elif a <= e <= 12:
                assert bool((out[a:e] == 7).all())
        return bits

    from paper_2608_19677_amd import binding as B
    assert call([0, 4, 8, 12], [4, 8, 20], good, [0, 1, 2]) == 0
    assert call([0, 4, 8, 12], [4, 3, 20], good, [0, 2]) == B.CR_ERR_SEQ      # fewer tokens than rows
    assert call([0, 4, 8, 12], [4, 33, 20], good, [0, 2]) == B.CR_ERR_SEQ     # beyond the table
    assert call([0, 4, 8, 13], [4, 8, 20], good, [0, 1]) == B.CR_ERR_SEQ      # beyond the rows
    assert call([0, 4, 8, 11], [4, 8, 20], good, [0, 1, 2]) == B.CR_ERR_SEQ   # rows of no sequence
    assert call([1, 4, 8, 12], [4, 8, 20], good, [0, 1, 2]) == B.CR_ERR_SEQ
    bad = good.clone()
    bad[1, 0], bad[2, 1] = 6, -1
    assert call([0, 4, 8, 12], [4, 8, 4], bad, [0, 2]) == B.CR_ERR_PAGE
    pool = _pool(g, 1, 6, heads, pt, d, dt, "e4m3", "head", 16)
    pool.append(0, k, v, _i32([0, 8, 4, 12]), _i32([8, 8, 8]), good)          # out of order
    assert int(pool.err.item()) == B.CR_ERR_SEQ


def test_offsets_past_32_bits():
    """Pages whose codes lie beyond 2^32 bytes."""
    dt, heads, d, pt = torch.bfloat16, 8, 128, 128
    say("[case] 8-bit append and read, offsets past 32 bits")
    pages = (1 << 32) // (heads * d * pt) + 40
    pool = serve.QuantPagePool.empty(1, pages, heads, pt, d, dt, block_tokens=1)
    g = _gen(2)
    table = _i32([[pages - 1, 3, pages - 7]])
    k, v = _rows(g, 300, heads, d, dt), _rows(g, 300, heads, d, dt)
    pool.append(0, k, v, _i32([0, 300]), _i32([300]), table)
    small = serve.QuantPagePool.empty(1, 3, heads, pt, d, dt, block_tokens=1)
    here = _i32([[0, 1, 2]])
    small.append(0, k, v, _i32([0, 300]), _i32([300]), here)
    out = [[torch.empty_like(k), torch.empty_like(k)] for _ in range(2)]
    for p, t, o in ((pool, table, out[0]), (small, here, out[1])):
        p.read(0, o[0], o[1], _i32([0, 300]), _i32([300]), t)
        assert int(p.err.item()) == 0
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    assert bool(((out[0][0] - k).abs() <= 2.0 ** -4 * k.abs() + 2.0 ** -10 * 2.0 ** -8 * k.abs().amax(2, keepdim=True) * 2).all())
