"""Page calls on the 8-bit cache: tables and counts are the 16-bit cache's, and codes and scales go with their pages, in
every layer."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import kvq_oracle as ko
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _pools(g, pages, pt, heads, d, layers, block, order, code="e4m3"):
    """An 8-bit cache of random contents and a 16-bit one of the same pages."""
    pool = serve.QuantPagePool.empty(layers, pages, heads, pt, d, order=order, codes=ko.CODES[code], block_tokens=block)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    pool.scale.copy_(torch.randint(0, 256, pool.scale.shape, generator=g, device="cuda", dtype=torch.uint8))
    plain = serve.PagePool.empty(layers, pages, heads, pt, 64, order=order)
    plain.k.zero_(), plain.v.zero_()
    return pool, plain


def _contents(pool):
    """[layers, pages, heads, tokens, ...] of codes, and scales [layers, pages, heads, tokens, 2]."""
    k, v = ((t if pool.order == "head" else t.transpose(2, 3)).view(torch.uint8).clone() for t in (pool.k, pool.v))
    return k, v, pool.scale.repeat_interleave(pool.block_tokens, 3)


SHAPES = [
    # pages, page tokens, heads, dim, layers, block, order
    (40, 16, 2, 128, 3, 16, "head"),
    (33, 8, 3, 64, 2, 2, "token"),
    (25, 1, 1, 64, 2, 1, "head"),
    (20, 128, 5, 128, 2, 32, "token"),
    (17000, 4, 1, 64, 1, 4, "head"),   # more pages than one block looks at
    (64, 256, 8, 128, 4, 128, "head"),  # tails of many pieces
]


@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_page_calls(shape):
    pages, pt, heads, d, layers, block, order = shape
    say(f"[case] 8-bit page calls {shape}")
    g = _gen(pages)
    pool, plain = _pools(g, pages, pt, heads, d, layers, block, order)
    lens = [pt * 3 - (pt > 1), 1, pt * 2, max(1, pt // 2)]
    width = 5
    tables = [torch.full((4, width), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    for p, t in zip((pool, plain), tables):
        p.refs[2:7:2] = 1  # taken by others: pages lie apart
        p.extend(t, None, _i32(lens))
    assert torch.equal(*tables) and torch.equal(pool.refs, plain.refs)
    table = tables[0]
    before = _contents(pool)
    parent = [0, 0, 1, 3, 2, 0]
    length = [lens[0], max(0, lens[0] - pt // 2 - 1), 1, lens[3], lens[2] - 1, 0]
    child = [torch.full((6, width), 99, dtype=torch.int32, device="cuda") for _ in range(2)]
    for p, c in zip((pool, plain), child):
        p.fork(table, _i32(parent), _i32(length), c)
    assert torch.equal(*child) and torch.equal(pool.refs, plain.refs)
    after = _contents(pool)
    touched = torch.zeros(pages, pt, dtype=torch.bool, device="cuda")
    for i, (p, n) in enumerate(zip(parent, length)):
        for tok in range(n):
            src, dst = int(table[p, tok // pt]), int(child[0][i, tok // pt])
            s = tok % pt
            assert (src == dst) == (tok // pt < n // pt)
            touched[dst, s] |= src != dst
            for a, b in zip(before, after):
                assert torch.equal(a[:, src, :, s], b[:, dst, :, s]), (i, tok)
    # nothing else: codes by tokens, scales by blocks of them
    kept = ~touched
    for a, b in zip(before[:2], after[:2]):
        assert torch.equal(a.transpose(2, 3)[:, kept], b.transpose(2, 3)[:, kept])
    blocks = ~touched.view(pages, pt // block, block).any(2)
    for a, b in ((before[2], after[2]),):
        a, b = (x[:, :, :, ::block].transpose(2, 3)[:, blocks] for x in (a, b))
        assert torch.equal(a, b)
    # growing a child, freeing the parents, and moving what lives to the front
    for p, c in zip((pool, plain), child):
        p.extend(c, _i32(length), _i32([n + 2 for n in length]))
        p.free(table, _i32(lens))
    assert torch.equal(*child) and torch.equal(pool.refs, plain.refs)
    length = [n + 2 for n in length]
    moved = []
    for p, c in zip((pool, plain), child):
        out = torch.empty_like(c)
        p.compact(c, _i32(length), table_out=out)
        moved.append(out)
    assert torch.equal(*moved) and torch.equal(pool.refs, plain.refs)
    last = _contents(pool)
    for i, n in enumerate(length):
        for j in range(-(-n // pt)):
            for a, b in zip(after, last):
                assert torch.equal(a[:, int(child[0][i, j])], b[:, int(moved[0][i, j])])
    src, dst = [int(moved[0][0, 0]), 3], [pages - 1, pages - 2]
    pool.copy(_i32(src), _i32(dst))
    end = _contents(pool)
    for s, t in zip(src, dst):
        for a, b in zip(last, end):
            assert torch.equal(a[:, s], b[:, t])
    assert int(pool.err.item()) == 0 and int(plain.err.item()) == 0


def test_many_sequences_by_many_blocks():
    say("[case] 8-bit fork by many blocks")
    g = _gen(3)
    pool, plain = _pools(g, 9000, 8, 2, 64, 2, 8, "token", "e5m2")
    lens = torch.randint(1, 40, (1200,), generator=g, device="cuda").to(torch.int32)
    table = torch.full((1200, 5), -1, dtype=torch.int32, device="cuda")
    other = table.clone()
    pool.extend(table, None, lens), plain.extend(other, None, lens)
    parent = torch.arange(1200, dtype=torch.int32, device="cuda").flip(0).contiguous()
    length = (lens[parent.long()] - 1).clamp(min=0)
    child, child2 = torch.empty_like(table), torch.empty_like(table)
    before = _contents(pool)
    pool.fork(table, parent, length, child), plain.fork(other, parent, length, child2)
    assert torch.equal(child, child2) and torch.equal(pool.refs, plain.refs) and int(pool.err.item()) == 0
    after = _contents(pool)
    tok = torch.arange(40, device="cuda")
    i, t = (tok < length[:, None]).nonzero(as_tuple=True)
    src, dst = table[parent.long()[i], t // 8].long(), child[i, t // 8].long()
    for a, b in zip(before, after):
        assert torch.equal(a.transpose(2, 3)[:, src, t % 8], b.transpose(2, 3)[:, dst, t % 8])


def test_strided_planes():
    """Keys and values side by side in one buffer, rows apart."""
    say("[case] 8-bit page copy, strided")
    g = _gen(5)
    both = torch.randint(0, 120, (2, 12, 3, 16, 3, 64), generator=g, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = torch.randint(1, 250, (2, 12, 3, 4, 2), generator=g, device="cuda", dtype=torch.uint8)
    pool = serve.QuantPagePool(both[..., 0, :], both[..., 2, :], scale, torch.zeros(12, dtype=torch.int32, device="cuda"))
    assert pool.block_tokens == 4
    before, scales = both.view(torch.uint8).clone(), scale.clone()
    pool.copy(_i32([1, 2]), _i32([11, 7]))
    want = before.clone()
    for s, t in ((1, 11), (2, 7)):
        want[:, t, ..., 0, :], want[:, t, ..., 2, :] = before[:, s, ..., 0, :], before[:, s, ..., 2, :]
        scales[:, t] = scales[:, s]
    assert torch.equal(both.view(torch.uint8), want) and torch.equal(scale, scales)


def test_binding():
    """The binding's functions of the 8-bit cache's calls against the handle."""
    say("[case] 8-bit calls through the binding")
    g = _gen(6)
    runs = []
    for direct in (False, True):
        g.manual_seed(6)
        pool, _ = _pools(g, 30, 16, 2, 128, 1, 16, "head")
        pool.k.view(torch.uint8).zero_(), pool.v.view(torch.uint8).zero_(), pool.scale.fill_(127)
        k, v, q = (torch.randn((n, h, 128), generator=g, device="cuda").to(torch.bfloat16) for n, h in ((40, 2), (40, 2), (4, 8)))
        table, child = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), torch.empty((2, 4), dtype=torch.int32, device="cuda")
        off, length, out = _i32([0, 33, 40]), _i32([33, 7]), torch.empty_like(q)
        back = torch.empty_like(k)
        qo, go, none = _i32([0, 3, 4]), _i32([0, 2]), _i32([0])
        parent, at = _i32([0, 1]), _i32([20, 7])
        if direct:
            rows = lambda t: B.CrRows(t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
            ws = torch.empty(B.cr_pages_workspace_bytes(30, 2), dtype=torch.uint8, device="cuda")
            B.cr_kvq_extend(pool.c, None, length, table, ws, pool.err)
            B.cr_kvq_append(pool.c, B.CrKvqTokens(0, 40, 2, 4, rows(k), rows(v), off.data_ptr(), length.data_ptr(), table.data_ptr()), pool.err)
            B.cr_kvq_fork(pool.c, table, parent, at, child, ws, pool.err)
            B.cr_kvq_free(pool.c, table, length, pool.err)
            B.cr_kvq_compact(pool.c, child, at, child, pool.refs, ws, pool.err)
            B.cr_kvq_copy(pool.c, _i32([0]), _i32([29]), pool.err)
            some = _i32([0, 20, 27])
            B.cr_kvq_read(pool.c, B.CrKvqTokens(0, 27, 2, 4, rows(back), B.CrRows(), some.data_ptr(), at.data_ptr(), child.data_ptr()), pool.err)
            a = B.CrAttnSharedArgs(8, 0, 2, 1, 4, 4, 4, 0.1, rows(q), rows(out), None, qo.data_ptr(), go.data_ptr(), child.data_ptr(),
                                   none.data_ptr(), child.data_ptr(), at.data_ptr())
            ws = torch.empty(B.cr_kvq_attn_workspace_bytes(pool.c, a), dtype=torch.uint8, device="cuda")
            B.cr_kvq_attn(pool.c, a, ws, pool.err)
        else:
            pool.extend(table, None, length)
            pool.append(0, k, v, off, length, table)
            pool.fork(table, parent, at, child)
            pool.free(table, length)
            pool.compact(child, at)
            pool.copy(_i32([0]), _i32([29]))
            pool.read(0, back[:27], None, _i32([0, 20, 27]), at, child)
            serve.attend_shared(q, pool, 0, qo, go, child[:1], none, child, at, 0.1, out=out)
        assert int(pool.err.item()) == 0
        runs.append((table, child, pool.refs, pool.k.view(torch.uint8), pool.v.view(torch.uint8), pool.scale, back[:27], out))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
