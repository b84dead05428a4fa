"""Page calls of the cache against a one-page-at-a-time statement: tables, counts and contents."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(layers, pages, heads, pt, dim, order, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pool = serve.PagePool.empty(layers, pages, heads, pt, dim, dtype, order=order)
    pool.k.copy_(torch.randn(pool.k.shape, generator=g, device="cuda"))
    pool.v.copy_(torch.randn(pool.v.shape, generator=g, device="cuda"))
    return pool, g


def _tables(g, pages, lens, pt, extra=2):
    ids = torch.randperm(pages, generator=g, device="cuda").tolist()
    need = [-(-n // pt) for n in lens]
    width, at, rows = max(need + [0]) + extra, 0, []
    for m in need:
        rows.append(ids[at:at + m] + [-1] * (width - m))
        at += m
    refs = [0] * pages
    for p in ids[:at]:
        refs[p] = 1
    return rows, refs


def _tail(x, order):
    return x if order == "head" else x.transpose(2, 3)


CACHES = [(1, 40, 1, 16, 64, "head"), (3, 200, 5, 4, 128, "token"), (2, 9000, 1, 1, 64, "head"), (2, 90, 2, 128, 64, "token")]


@pytest.mark.parametrize("geom", CACHES, ids=[f"L{c[0]}-N{c[1]}-H{c[2]}-T{c[3]}-{c[5]}" for c in CACHES])
def test_extend_fork_free(geom):
    layers, pages, heads, pt, dim, order = geom
    pool, g = _pool(layers, pages, heads, pt, dim, order, 1)
    lens = [3 * pt + 1, 0, 2 * pt, 1, pt]
    rows, refs = _tables(g, pages, lens, pt)
    pool.refs.copy_(_i32(refs))
    ref = so.Pages(refs, pt)
    say(f"[case] extend {geom}")
    table = _i32(rows)
    grown = [n + d for n, d in zip(lens, (1, pt + 1, 0, 2 * pt, 1))]
    pool.extend(table, _i32(lens), _i32(grown))
    want, ok = ref.extend(rows, lens, grown)
    assert ok and table.tolist() == want and pool.refs.tolist() == ref.refs
    say(f"[case] fork {geom}")
    parent = [0, 0, 2, 3, 3, 4, 1, 0]
    length = [grown[0], pt, 2 * pt, 1, 0, grown[4], grown[1], 2 * pt + 1 if pt > 1 else 2]
    child = torch.full((len(parent), table.shape[1]), -7, dtype=torch.int32, device="cuda")
    before = pool.k.cpu().clone(), pool.v.cpu().clone()
    pool.fork(table, _i32(parent), _i32(length), child)
    crow, copies, ok = ref.fork(want, parent, length, table.shape[1])
    assert ok and child.tolist() == crow and pool.refs.tolist() == ref.refs
    for x, y in zip((pool.k, pool.v), before):
        for s, d, n in copies:
            _tail(y, order)[:, d, :, :n] = _tail(y, order)[:, s, :, :n]
        assert torch.equal(x.cpu(), y)
    say(f"[case] free {geom}")
    pool.free(table, _i32(grown))
    ref.free(want, grown)
    assert pool.refs.tolist() == ref.refs
    pool.free(child, _i32(length))
    ref.free(crow, length)
    assert pool.refs.tolist() == ref.refs == [0] * pages and int(pool.err.item()) == 0


@pytest.mark.parametrize("pages,live", [(1, 1), (1, 0), (50, 25), (50, 50), (4097, 2000), (9001, 8999), (9001, 3), (70000, 30000)])
@pytest.mark.parametrize("inplace", [False, True])
def test_compact(pages, live, inplace):
    pool, g = _pool(2, pages, 1, 2, 64, "head", 2)
    ids = torch.randperm(pages, generator=g, device="cuda")[:live]
    pool.refs[ids] = 1 + torch.arange(live, device="cuda", dtype=torch.int32) % 3
    rows, width = 7, 11
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    lens = [0, 1, 2, 3, 21, 22, 10] if live else [0] * rows
    if live:
        table[:] = ids[torch.randint(live, (rows, width), generator=g, device="cuda")].to(torch.int32)
    ref = so.Pages(pool.refs.tolist(), 2)
    want, moves = ref.compact(table.tolist(), lens)
    wk, wv = pool.k.cpu().clone(), pool.v.cpu().clone()
    for x in (wk, wv):
        if moves:
            s, d = (torch.tensor([m[i] for m in moves]) for i in (0, 1))
            x[:, d] = x[:, s]
    out = table if inplace else torch.empty_like(table)
    counts = pool.refs if inplace else torch.full_like(pool.refs, -5)
    say(f"[case] compact {pages} pages {live} live in place {inplace}")
    pool.compact(table, _i32(lens), table_out=out, refs_out=counts)
    assert out.tolist() == want and counts.tolist() == ref.refs and int(pool.err.item()) == 0
    assert torch.equal(pool.k.cpu(), wk) and torch.equal(pool.v.cpu(), wv)


def test_compact_without_tables_and_copy():
    pool, g = _pool(2, 33, 3, 4, 64, "token", 3)
    before = pool.k.cpu().clone()
    src, dst = [4, 9, 4, 32], [0, 1, 2, 3]
    say("[case] copy")
    pool.copy(_i32(src), _i32(dst))
    before[:, dst] = before[:, src]
    assert torch.equal(pool.k.cpu(), before)
    pool.refs[[32, 5]] = 2
    say("[case] compact without tables")
    pool.compact(None, None)
    before[:, [0, 1]] = before[:, [5, 32]]
    assert pool.refs.tolist() == [2, 2] + [0] * 31 and torch.equal(pool.k.cpu(), before)


def test_strided_pool_fork_and_compact():
    """Pages inside a larger buffer: gaps between heads and tokens stay as they are."""
    big = torch.randn(2, 20, 3, 8, 192, device="cuda").to(torch.float16)
    vig = torch.randn(2, 20, 3, 8, 192, device="cuda").to(torch.float16)
    pool = serve.PagePool(big[..., :64], vig[..., :64], torch.zeros(20, dtype=torch.int32, device="cuda"))
    pool.refs[[3, 17, 18]] = 1
    table = _i32([[17, 3, 18]])
    child = torch.empty(2, 4, dtype=torch.int32, device="cuda")
    want = big.cpu().clone()
    say("[case] fork and compact in a strided pool")
    pool.fork(table, _i32([0, 0]), _i32([19, 9]), child)
    assert child.tolist() == [[17, 3, 0, -1], [17, 1, -1, -1]]
    want[:, 0, :, :3, :64] = want[:, 18, :, :3, :64]
    want[:, 1, :, :1, :64] = want[:, 3, :, :1, :64]
    assert torch.equal(big.cpu(), want)
    pool.compact(child, _i32([19, 9]))
    assert child.tolist() == [[2, 3, 0, -1], [2, 1, -1, -1]] and pool.refs.tolist()[:6] == [1, 1, 3, 2, 1, 0]
    want[:, 2, ..., :64], want[:, 4, ..., :64] = want[:, 17, ..., :64].clone(), want[:, 18, ..., :64].clone()
    assert torch.equal(big.cpu(), want)


def test_errors_leave_the_rest_right():
    pool, g = _pool(1, 10, 1, 4, 64, "head", 4)
    pool.refs[:6] = 1
    table = _i32([[0, 1, 2], [3, 4, 5]])
    before = pool.refs.tolist()

    def bit():
        v = int(pool.err.item())
        pool.err.zero_()
        return v

    say("[case] more pages than are free")
    big = torch.full((1, 9), -1, dtype=torch.int32, device="cuda")
    pool.extend(big, None, _i32([20]))
    assert bit() == B.CR_ERR_PAGES_OUT and big.tolist() == [[-1] * 9] and pool.refs.tolist() == before
    child = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    pool.fork(table, _i32([0, 0, 1, 1, 1]), _i32([9, 1, 1, 1, 5]), child)
    assert bit() == B.CR_ERR_PAGES_OUT and child.tolist() == [[-1] * 3] * 5 and pool.refs.tolist() == before
    say("[case] lengths and rows that do not fit")
    pool.extend(big, _i32([8]), _i32([4]))
    assert bit() == B.CR_ERR_SEQ and pool.refs.tolist() == before
    child = torch.zeros(3, 3, dtype=torch.int32, device="cuda")
    pool.fork(table, _i32([2, 0, 1]), _i32([1, 13, 5]), child)
    assert bit() == B.CR_ERR_SEQ and child.tolist() == [[-1] * 3, [-1] * 3, [3, 6, -1]]
    pool.free(child, _i32([0, 0, 5]))
    assert pool.refs.tolist() == before and bit() == 0
    say("[case] freed more often than named")
    pool.free(_i32([[0, 0, 99], [0, 1, 2]]), _i32([12, 13]))
    assert bit() == B.CR_ERR_PAGE | B.CR_ERR_SEQ and pool.refs.tolist() == [0] + before[1:]
    say("[case] entries that name no live page")
    child = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    pool.fork(_i32([[9, 1, 50]]), _i32([0]), _i32([12]), child)
    assert bit() == B.CR_ERR_PAGE and child.tolist() == [[-1, 1, -1]]
    out = torch.empty_like(table)
    pool.compact(table, _i32([12, 13]), table_out=out)
    assert bit() == B.CR_ERR_PAGE | B.CR_ERR_SEQ
    assert out.tolist() == [[0, 1, 2], [3, 4, 5]] and pool.refs.tolist() == [1, 2, 1, 1, 1] + [0] * 5
    pool.copy(_i32([0, 10]), _i32([9, 8]))
    assert bit() == B.CR_ERR_PAGE and torch.equal(pool.k[:, 0], pool.k[:, 9])


def test_page_calls_in_a_graph():
    pool, g = _pool(2, 64, 2, 8, 64, "head", 6)
    pool.refs[:4] = 1
    table, parent, length = _i32([[0, 1, 2, 3]]), _i32([0] * 6), _i32([29, 8, 0, 17, 32, 1])
    child = torch.empty(6, 4, dtype=torch.int32, device="cuda")
    pool.fork(table, parent, length, child)
    want, refs = child.tolist(), pool.refs.tolist()
    pool.free(child, length)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("[case] fork and free in a graph")
    with torch.cuda.graph(graph):
        pool.fork(table, parent, length, child)
    for _ in range(3):
        child.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert child.tolist() == want and pool.refs.tolist() == refs
        pool.free(child, length)
        assert pool.refs.tolist() == [1] * 4 + [0] * 60
