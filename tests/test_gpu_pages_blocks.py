"""Page calls of caches too large for one block: free pages in several chunks of 4,096, sequences in several
rounds of 256, and every error that the calls of small caches report."""
import pytest
import torch

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

import serve_oracle as so
from cr_check import say

pytestmark = pytest.mark.gpu

PAGES = 20_000  # from 16,385 on the calls take many blocks


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(pages, pt=4, layers=1, heads=1, dim=64):
    pool = serve.PagePool.empty(layers, pages, heads, pt, dim)
    # page p of layer l holds 1 + (p + l) % 251 in k and its negative in v: exact in 16 bits
    mark = 1 + (torch.arange(pages, device="cuda")[None] + torch.arange(layers, device="cuda")[:, None]) % 251
    pool.k.copy_(mark[:, :, None, None, None].expand(pool.k.shape))
    pool.v.copy_(-pool.k)
    return pool


def _err(pool):
    v = int(pool.err.item())
    pool.err.zero_()
    return v


@pytest.mark.parametrize("pages", [10, PAGES])
def test_fork_of_a_tail_in_a_free_page(pages):
    """A tail's entry that names a free page, one out of range or CR_NO_PAGE is copied from nowhere, whatever the size
    of the cache and whether that page is handed out meanwhile; the other children are served."""
    pool = _pool(pages)
    pool.refs[2] = 1
    # the free pages are taken by id: 0, 1, 3, 4. Rows 0 and 1 have their tails in pages 0 and 3, which are free.
    table = _i32([[2, 0], [2, 3], [2, pages], [2, -1], [2, 2]])
    child = torch.full((5, 2), -7, dtype=torch.int32, device="cuda")
    k, v, refs = pool.k.clone(), pool.v.clone(), pool.refs.clone()
    say(f"[case] fork of free tails, {pages} pages")
    pool.fork(table, _i32([0, 1, 2, 3, 4]), _i32([6, 7, 5, 6, 7]), child)
    assert _err(pool) == B.CR_ERR_PAGE
    assert child.tolist() == [[2, 0], [2, 1], [2, 3], [2, 4], [2, 5]]
    refs[2] += 5
    refs[[0, 1, 3, 4, 5]] = 1
    assert torch.equal(pool.refs, refs)
    k[:, 5, :, :3], v[:, 5, :, :3] = k[:, 2, :, :3], v[:, 2, :, :3]
    assert torch.equal(pool.k, k) and torch.equal(pool.v, v)


@pytest.mark.parametrize("later", [40, 31_000], ids=["same", "grown"])
def test_a_graph_keeps_its_workspace(later):
    """A captured call's workspace stays the pool's when later calls have more sequences, whether they fit it or
    not: a replay writes into nobody else's memory."""
    pool = _pool(PAGES)
    live = torch.randperm(PAGES, generator=torch.Generator().manual_seed(5))[:9000].sort().values.cuda()
    table, length = live[::300].to(torch.int32).reshape(1, -1).contiguous(), _i32([4 * 30])
    out, counts = torch.empty_like(table), torch.empty_like(pool.refs)
    pool.refs[live] = 1
    pool.compact(table, length, table_out=out, refs_out=counts)
    want, want_counts = out.clone(), counts.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pool.compact(table, length, table_out=out, refs_out=counts)
    size = pool._ws.numel()
    say(f"[case] compaction in a graph, then {later} sequences")
    free = torch.full((later, 1), -1, dtype=torch.int32, device="cuda")
    pool.extend(free, None, torch.zeros(later, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(6)]
    for _ in range(3):
        out.zero_(), counts.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(counts, want_counts)
        assert all(bool((x == 0x5A).all()) for x in others)
    assert _err(pool) == 0


def _scattered(pages, live, seed):
    """Counts with `live` of the pages in use, scattered."""
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:live]] = 1
    return refs.tolist()


CACHES = [
    # pages, live, sequences: free pages of several chunks, few and many sequences; a small cache with too many for one block
    (20_000, 17_000, 30), (70_000, 300, 1), (70_000, 69_000, 700), (16_385, 10_000, 1025), (600, 100, 1100),
]


@pytest.mark.parametrize("pages,live,n", CACHES, ids=[f"{p}-{l}-{n}seq" for p, l, n in CACHES])
def test_extend_fork_free(pages, live, n):
    pt = 4
    pool = _pool(pages, pt, layers=2)
    refs = _scattered(pages, live, n)
    pool.refs.copy_(_i32(refs))
    ref = so.Pages(refs, pt)
    room = pages - live
    g = torch.Generator().manual_seed(pages)
    # a first extension and a second one that together take about half of what is free
    most = max(1, room // (2 * n))
    first = torch.randint(0, pt * max(1, most // 2) + 1, (n,), generator=g).tolist()
    if n > room // 2:
        first = [x if i % 8 == 0 else 0 for i, x in enumerate(first)]
    then = [x + d if x else 0 for x, d in zip(first, torch.randint(0, pt * most // 2 + 1, (n,), generator=g).tolist())]
    width = -(-max(then) // pt) + 1
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    rows = table.tolist()
    for old, new in ((None, first), (first, then)):
        say(f"[case] extend {pages} pages, {n} sequences")
        pool.extend(table, None if old is None else _i32(old), _i32(new))
        rows, ok = ref.extend(rows, old or [0] * n, new)
        assert ok and table.tolist() == rows and pool.refs.tolist() == ref.refs
    m = min(2 * n, len([r for r in ref.refs if r == 0]))
    parent = torch.randint(0, n, (m,), generator=g).tolist()
    length = [int(x * then[p]) for x, p in zip(torch.rand(m, generator=g).tolist(), parent)]
    child = torch.full((m, width), -9, dtype=torch.int32, device="cuda")
    k, v = pool.k.cpu(), pool.v.cpu()
    say(f"[case] fork {pages} pages, {m} children")
    pool.fork(table, _i32(parent), _i32(length), child)
    crow, copies, ok = ref.fork(rows, parent, length, width)
    assert ok and child.tolist() == crow and pool.refs.tolist() == ref.refs
    for x, y in ((pool.k, k), (pool.v, v)):
        for s, d, t in copies:
            y[:, d, :, :t] = y[:, s, :, :t]
        assert torch.equal(x.cpu(), y)
    say(f"[case] free {pages} pages")
    pool.free(child, _i32(length))
    pool.free(table, _i32(then))
    assert pool.refs.tolist() == refs and _err(pool) == 0


@pytest.mark.parametrize("pages", [10, PAGES])
def test_errors_are_the_same_in_both_forms(pages):
    """A cache whose pages 0 to 5 are named and all but 6 to 9 of the others taken: what 10 pages give, 20,000 give."""
    pool = _pool(pages)
    pool.refs.fill_(1)
    pool.refs[6:10] = 0
    before = pool.refs.tolist()
    table = _i32([[0, 1, 2], [3, 4, 5]])
    say(f"[case] errors, {pages} pages")
    big = torch.full((1, 9), -1, dtype=torch.int32, device="cuda")
    pool.extend(big, None, _i32([20]))
    assert _err(pool) == B.CR_ERR_PAGES_OUT and big.tolist() == [[-1] * 9] and pool.refs.tolist() == before
    child = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    k = pool.k.clone()
    pool.fork(table, _i32([0, 0, 1, 1, 1]), _i32([9, 1, 1, 1, 5]), child)
    assert _err(pool) == B.CR_ERR_PAGES_OUT and child.tolist() == [[-1] * 3] * 5 and pool.refs.tolist() == before
    pool.extend(big, _i32([8]), _i32([4]))
    assert _err(pool) == B.CR_ERR_SEQ and pool.refs.tolist() == before
    two = torch.full((2, 2), -1, dtype=torch.int32, device="cuda")
    pool.extend(two, None, _i32([9, 5]))  # the first passes the table, the second is served
    assert _err(pool) == B.CR_ERR_SEQ and two.tolist() == [[-1, -1], [6, 7]]
    pool.free(two, _i32([0, 5]))
    assert torch.equal(pool.k, k) and pool.refs.tolist() == before
    child = torch.zeros(3, 3, dtype=torch.int32, device="cuda")
    pool.fork(table, _i32([2, 0, 1]), _i32([1, 13, 5]), child)
    assert _err(pool) == B.CR_ERR_SEQ and child.tolist() == [[-1] * 3, [-1] * 3, [3, 6, -1]]
    k[:, 6, :, :1] = k[:, 4, :, :1]
    assert torch.equal(pool.k, k)
    pool.free(child, _i32([0, 0, 5]))
    assert pool.refs.tolist() == before and _err(pool) == 0
    child = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    pool.fork(_i32([[9, 1, pages]]), _i32([0]), _i32([12]), child)
    before[1] += 1
    assert _err(pool) == B.CR_ERR_PAGE and child.tolist() == [[-1, 1, -1]] and pool.refs.tolist() == before
    pool.free(_i32([[9, 0, pages]]), _i32([12]))
    before[0] -= 1
    assert _err(pool) == B.CR_ERR_PAGE and pool.refs.tolist() == before


def test_the_last_free_page():
    """As many pages as are free, the last page of the last chunk among them, and one more."""
    pool = _pool(PAGES, pt=1)
    pool.refs.fill_(1)
    free = [0, 4095, 4096, 8191, 16384, PAGES - 1]
    pool.refs[free] = 0
    table = torch.full((3, 3), -1, dtype=torch.int32, device="cuda")
    say("[case] extend to the last free page")
    pool.extend(table, None, _i32([3, 3, 1]))
    assert _err(pool) == B.CR_ERR_PAGES_OUT and table.tolist() == [[-1] * 3] * 3
    pool.extend(table, None, _i32([2, 3, 1]))
    assert _err(pool) == 0 and table.tolist() == [[0, 4095, -1], [4096, 8191, 16384], [PAGES - 1, -1, -1]]
    assert bool((pool.refs == 1).all())


def test_a_fork_in_a_graph():
    """By many blocks, replayed with other calls between."""
    pool = _pool(PAGES)
    pool.refs[100:140] = 1
    table = torch.arange(100, 140, dtype=torch.int32, device="cuda")[None]
    parent, length = _i32([0] * 6), _i32([29, 8, 0, 17, 32, 1])
    child = torch.empty(6, 10, dtype=torch.int32, device="cuda")
    pool.fork(table, parent, length, child)
    want, refs = child.tolist(), pool.refs.tolist()
    pool.free(child, length)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    say("[case] fork by many blocks in a graph")
    with torch.cuda.graph(graph):
        pool.fork(table, parent, length, child)
    for i in range(3):
        child.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert child.tolist() == want and pool.refs.tolist() == refs
        pool.free(child, length)
        other = torch.full((1, 3), -1, dtype=torch.int32, device="cuda")
        pool.extend(other, None, _i32([9]))
        pool.free(other, _i32([9]))
    assert _err(pool) == 0


@pytest.mark.parametrize("pages", [60, PAGES])
def test_several_tables_are_compacted_one_after_the_other(pages):
    """One call per table with the counts put elsewhere, the last (without a table) puts them in place."""
    pool = _pool(pages)
    live = [pages - 1, 3, pages - 7, 20, pages - 2]
    pool.refs[live] = _i32([1, 2, 1, 1, 1])
    ref = so.Pages(pool.refs.tolist(), 4)
    tables, lengths = [_i32([live[:2]]), _i32([live[2:], live[1:4]])], [[8], [9, 3]]
    want = []
    for t, n in zip(tables, lengths):
        want.append(so.Pages(ref.refs, 4).compact(t.tolist(), n)[0])
    k = pool.k.clone()
    _, moves = ref.compact([], [])
    for s, d in moves:
        k[:, d] = k[:, s]
    say(f"[case] two tables, {pages} pages")
    aside = torch.empty_like(pool.refs)
    for t, n in zip(tables, lengths):
        pool.compact(t, _i32(n), refs_out=aside)
    pool.compact(None, None)
    assert [t.tolist() for t in tables] == want and pool.refs.tolist() == ref.refs and torch.equal(pool.k, k) and _err(pool) == 0


@pytest.mark.parametrize("pages", [60, PAGES])
def test_children_in_rows_of_the_parents_table(pages):
    """Rows that no parent names take children of the same table."""
    pool = _pool(pages)
    pool.refs[:3] = 1
    table = _i32([[0, 1, 2], [-7] * 3, [-7] * 3])
    say(f"[case] children beside their parent, {pages} pages")
    pool.fork(table, _i32([0, 0]), _i32([9, 4]), table[1:])
    assert _err(pool) == 0 and table.tolist() == [[0, 1, 2], [0, 1, 3], [0, -1, -1]]
    assert pool.refs[:5].tolist() == [3, 2, 1, 1, 0]
